// A drafted tree's accepted path taken over into the budgeted cache, in two launches.
//
//   tree_statistics : up to 1024 slots per workgroup.  The accepted rows' probabilities are formed again, exp(logit - lse), from one pass over K
//                     alone: half of what the attention has read, where probabilities left behind by the attention would be 4 bytes per
//                     slot, head and node, of which the accepted ones are known only now.  Their sums go to the workspace.  Beside these
//                     workgroups, and before them, one per unit chooses the victims, E = max(0, n + a - budget) of them by the statistics
//                     as they stand (two exact searches, as in block_prepare), and the slots that the accepted tokens take.  Neither changes
//                     what the other reads.
//   tree_apply      : the sums added to the statistics, the accepted tokens' rows, positions and statistics to their slots.
//
// (One after the other, choice and sums took 14 + 45 us on 512 units x 2048 slots of bf16 / 128, together 53; on 16 x 500 9 + 7, together 7.4.  The search of a
// large budget needs more threads and LDS than the sums leave it: above kMostChosenBeside slots it is a launch of its own.  Commits of six tokens, us,
// beside / of its own: 8 units x 4000 slots 20.6 / 22.2, 64 x 4000 23.5 / 31.7, 512 x 4000 110 / 120; 64 x 6000 36.7 / 39.3, but 192 x 6000 58.6 / 57.9,
// 512 x 6000 182 / 178, 8 x 8000 30.1 / 26.9, 512 x 8000 241 / 235, 64 x 12000 81 / 59, 512 x 12000 491 / 351.)
#include <algorithm>
#include <type_traits>

#include "profile.hpp"
#include "tree.hpp"

namespace roco {
namespace {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

using namespace tree;

constexpr int kMostChosenBeside = 4096;

__device__ __forceinline__ int path_length(const CommitArgs& a, int request, int budget) {
  return min(max(a.n_path[request], 0), min(a.max_path, budget));
}
__device__ __forceinline__ int path_node(const CommitArgs& a, int request, int k) {
  return min(max(a.path[static_cast<size_t>(request) * a.max_path + k], 0), a.nodes - 1);
}

// The victims and the slots of the accepted tokens: CommitArgs::taken and the records of what is evicted.  All threads of the workgroup.
// sel_sh: SelectLds<1>::kWords words; list_sh: kListWords; keys: [2][B].
constexpr int kListWords = (1 + kMaxTreeNodes + 3) / 4 * 4;
template <int NT> __device__ __forceinline__ void choose_slots(const CommitArgs& a, int u, uint32_t* sel_sh, uint32_t* list_sh, uint32_t* keys) {
  const int tid = threadIdx.x, B = a.B;
  const int request = u / a.heads;
  const int budget = budget_of(a.pages, B, request);
  const int n = min(max(a.n_used[u], 0), budget);
  const int len = path_length(a, request, budget);
  const int n_new = min(budget, n + len), E = n + len - n_new;
  int32_t* const taken = a.taken + static_cast<size_t>(u) * kTakenWords;
  if (tid < a.max_path && tid >= len) {
    if (a.evicted_slot != nullptr) a.evicted_slot[static_cast<size_t>(u) * a.max_path + tid] = -1;
    if (a.evicted_pos != nullptr) a.evicted_pos[static_cast<size_t>(u) * a.max_path + tid] = -1;
  }
  if (tid == 0) {
    taken[1] = len;
    taken[2] = n_new;
    list_sh[0] = 0u;
  }
  if (len == 0) return;
  const float* const acc = a.stats + static_cast<size_t>(u) * 3 * B;
  const float* const acc2 = acc + B;
  const float* const cnt = acc2 + B;
  const int32_t* const pos = a.pos + static_cast<size_t>(u) * B;
  uint32_t *const var_key = keys, *const mas_key = keys + B;
  uint32_t* const found = list_sh + 1;  // the accepted tokens' slots, in any order
  const auto keep = [&](int j) {
    const uint32_t at = atomicAdd(&list_sh[0], 1u);
    if (at < static_cast<uint32_t>(len)) found[at] = static_cast<uint32_t>(j);
  };
  if (E == 0) {
    __syncthreads();  // list_sh[0] is there
  } else {
    // (kEach slots of a thread at a time, so that their loads are in flight together: one by one the keys took half of a choice)
    constexpr int kEach = 4;
#pragma unroll 1
    for (int i0 = tid; i0 < n; i0 += kEach * NT) {
      float first[kEach], second[kEach], count[kEach];
      int at[kEach];
      uint32_t mas[kEach], var[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = min(i0 + e * NT, n - 1);
        first[e] = acc[i];
        second[e] = acc2[i];
        count[e] = cnt[i];
        at[e] = pos[i];
      }
      ranking_keys<kEach>(first, second, count, at, a.pol, mas, var);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = min(i0 + e * NT, n - 1);
        mas_key[i] = mas[e];
        var_key[i] = var[e];
      }
    }
    __syncthreads();
    const uint32_t m = min(static_cast<uint32_t>(n), static_cast<uint32_t>(a.pol.scope_size(min(a.scope, budget), n)) + static_cast<uint32_t>(E) - 1u);
    KSmallest r = {0u, 0u};
#pragma unroll 1
    for (int phase = 0; phase < 2; ++phase) {
      const uint32_t* const key = phase == 0 ? var_key : mas_key;
      r = select_k_smallest<NT, 1, NT <= 256 ? 4 : 1>([&](int i) -> uint32_t { return key[i]; }, n, phase == 0 ? m : static_cast<uint32_t>(E),
                                                      phase == 0 && a.pol.scope_is_window(), sel_sh, phase == 0 || a.pol.spreads_importance());
#pragma unroll 1
      for (int i0 = tid; i0 < n; i0 += kEach * NT) {
        bool in[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int i = i0 + e * NT;
          in[e] = r.has(key[min(i, n - 1)], i);
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int i = i0 + e * NT;
          if (i >= n) break;
          if (phase == 0 && !in[e]) mas_key[i] = 0xffffffffu;
          if (phase == 1 && in[e]) keep(i);
        }
      }
      __syncthreads();
    }
  }
  if (tid < n_new - n) keep(n + tid);
  __syncthreads();
  if (tid >= len) return;
  const int j = static_cast<int>(found[tid]);
  int k = 0;
  for (int i = 0; i < len; ++i) k += static_cast<int>(found[i]) < j ? 1 : 0;
  taken[4 + k] = j;
  const bool held = j < n;  // by a token that is now evicted
  if (a.evicted_slot != nullptr) a.evicted_slot[static_cast<size_t>(u) * a.max_path + k] = held ? j : -1;
  if (a.evicted_pos != nullptr) a.evicted_pos[static_cast<size_t>(u) * a.max_path + k] = held ? pos[j] : -1;
}

// LDS: the ranking keys are in LDS (B <= kMaxDecodeBudgetLds).
constexpr int kChooseThreads = 1024;
template <bool LDS> __global__ __launch_bounds__(kChooseThreads, 8) void tree_choose(CommitArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds_keys[];  // [2][B]
  __shared__ __attribute__((aligned(16))) uint32_t sel_sh[SelectLds<1>::kWords];
  __shared__ uint32_t list_sh[kListWords];
  choose_slots<kChooseThreads>(a, blockIdx.x, sel_sh, list_sh, LDS ? lds_keys : a.keys + static_cast<size_t>(blockIdx.x) * 2 * a.B);
}

constexpr int kStatWaves = 4;
constexpr int kStatThreads = kStatWaves * kWave;
constexpr int kChoiceWords = kListWords + (SelectLds<1>::kWords + 3) / 4 * 4;  // of a choice among the sums, before its keys
// Bytes of a wave's tile: small ones, so that four workgroups are on a compute unit and one's sums over its rows, or its way to the first tile,
// go beside the others' streams (8 KiB and two workgroups: 512 units x 2048 slots of bf16 / 128 75.1 us against 70.3, 192 x 4096 of
// bf16 / 64 51.1 / 46.6).  16 slots are the least.
template <int DT, int HD> constexpr int kStatTile = DT == kF32 && HD == 128 ? 8192 : 4096;
constexpr int kMostQueryLds = 40960;  // bytes of accepted query rows in LDS at a time: 64 heads of fp32 / 128 take 32 KiB for a token

// How the accepted rows lie in matrix tiles of 16: a token's heads side by side, filled up to a power of two, so that as few tiles as
// can be are formed (a row of no head, or of no token, has a normaliser of infinity and no probability), and the mean over the heads is a sum
// over registers (up to four heads), lane groups (up to 16) and tiles.
struct RowPlan {
  int heads_log2;  // of a token, filled up
  int per_pass;    // tokens whose rows are in LDS at a time, whole tiles of them
  __host__ __device__ int rows(int tokens) const { return ((tokens << heads_log2) + 15) / 16 * 16; }
};
inline RowPlan row_plan(int group, int max_path, int row_bytes) {
  RowPlan p;
  p.heads_log2 = 0;
  while ((1 << p.heads_log2) < group) ++p.heads_log2;
  const int tokens_per_tile = std::max(1, 16 >> p.heads_log2), most = kMostQueryLds / row_bytes >> p.heads_log2;
  p.per_pass = std::min((max_path + tokens_per_tile - 1) / tokens_per_tile * tokens_per_tile, most / tokens_per_tile * tokens_per_tile);
  return p;
}

// Q is the A operand here, so that a lane holds four rows of one slot.  The accepted tokens themselves are tiles of the last workgroup, gathered
// from k_new; token m is not seen by the rows before m.  More rows than the LDS takes: another pass over K (which the L2 mostly has).
// choosers: the first workgroups, one per unit, that choose its slots (0: they have been chosen).
// 512 units x 2048 slots of bf16 / 128 with up to six rows 53 us, 5 TB/s of K; 192 x 4096 of bf16 / 64 with up to 32 rows 23, vector issue.
template <int DT, int HD, bool STREAMING, bool WINDOW>
__global__ __launch_bounds__(kStatThreads, 4) void tree_statistics(CommitArgs a, RowPlan plan, int choosers) {
  constexpr int kTileBytes = kStatTile<DT, HD>;
  using T = Tile<DT, HD, kTileBytes>;
  constexpr int W = kStatWaves, G = T::kGroups;
  extern __shared__ __attribute__((aligned(1024))) char lds[];  // the waves' tiles, two each, then the query rows and their normalisers; or a choice's keys
  __shared__ int32_t pos_s[WINDOW ? kTreeChunk : 1];
  if (static_cast<int>(blockIdx.x) < choosers) {
    uint32_t* const words = reinterpret_cast<uint32_t*>(lds);
    choose_slots<kStatThreads>(a, blockIdx.x, words + kListWords, words, words + kChoiceWords);
    return;
  }
  const int id = blockIdx.x - choosers, u = id % a.units, split = id / a.units;
  const int request = u / a.heads;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int qi = lane & 15, g = lane >> 4;
  // (what has to come from memory before anything else is asked for together)
  const int my_node = path_node(a, request, min(lane, a.max_path - 1));
  const int budget = budget_of(a.pages, a.B, request), asked_len = a.n_path[request], held = a.n_used[u];
  const int n = __builtin_amdgcn_readfirstlane(min(max(held, 0), budget));
  const int len = __builtin_amdgcn_readfirstlane(min(max(asked_len, 0), min(a.max_path, budget)));
  const int used = splits_used(n, a.chunk);  // the last of them takes the accepted tokens too
  if (len == 0 || split >= used) return;
  const int row0 = split * a.chunk, row1 = min(n, row0 + a.chunk);
  const int fresh = split == used - 1 ? len : 0;

  Walk<DT, HD, W, kTileBytes> walk;
  walk.init(a.pages, a.B, a.heads, u, request, row0, row1, fresh, wave, static_cast<unsigned>(u) * 5u + static_cast<unsigned>(split) * 3u);
  const int mine = walk.mine;
  char* const tiles = lds + wave * 2 * kTileBytes;
  const uint32_t tiles_addr = lds_address(tiles);
  int koff[T::kGroupLoads];
  load_offsets<DT, HD, false>(koff);
  auto request_k = [&](int t) {
    const typename Walk<DT, HD, W, kTileBytes>::Place p = walk.place(t);
    const uint32_t dst = tiles_addr + (t & 1) * kTileBytes;
    if (!walk.is_nodes(t)) {
      request_tile<DT, HD, STREAMING>(a.K, p.row, p.there, dst, koff);
      return p.there;
    }
    // the accepted tokens' rows, each from its node's (what lies behind the last token is out of range)
    const v4i32 buf = make_buffer(static_cast<const char*>(a.k_new) + static_cast<size_t>(u) * a.nodes * T::kBytes, static_cast<uint32_t>(a.nodes) * T::kBytes);
    const int lane2 = late_thread_id() & (kWave - 1);
#pragma unroll
    for (int j = 0; j < T::kLoads; ++j) {
      const int r = T::kPerLoad * j + lane2 / T::kChunks, c = lane2 % T::kChunks, k = walk.first_node(t) + r;
      const int node = __shfl(my_node, min(k, kWave - 1), kWave);
      mfma::load16_to_lds(buf, dst + j * 1024, k < len ? node * T::kBytes + ((c ^ T::swizzle_k(r & 15)) << 4) : 0x7ffffff0, 0);
    }
    return p.there;
  };
  if (WINDOW)
    for (int j = tid; j < row1 - row0; j += kStatThreads) pos_s[WINDOW ? j : 0] = a.pos[static_cast<size_t>(u) * a.B + row0 + j];
  float* const sums = a.sums + static_cast<size_t>(u) * 2 * a.B + row0;
  float* const fresh_sums = a.fresh + static_cast<size_t>(u) * 2 * kMaxTreeNodes;

  const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f, share = 1.0f / static_cast<float>(a.group);
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[u] : 0;
  const int frag = qi * T::kBytes + ((g ^ T::swizzle_k(qi)) << 4);
  // of the lane's four rows of a tile, those whose register holds a token's sum over its heads in the end
  const int heads_log2 = plan.heads_log2;
  const int slices = 1 << max(heads_log2 - 4, 0);  // tiles of a token
  const bool squares = !a.pol.keeps_last_score() && !a.pol.counts_above_average();
  const bool filled_up = (1 << heads_log2) != a.group;
  char* const q_s = lds + W * 2 * kTileBytes;
  float* const lse_s = reinterpret_cast<float*>(q_s + static_cast<size_t>(plan.rows(plan.per_pass)) * T::kBytes);  // base 2
#pragma unroll 1
  for (int first = 0; first < len; first += plan.per_pass) {
    const int tokens = min(plan.per_pass, len - first), rows = plan.rows(tokens);
    __syncthreads();  // nobody reads the rows of the pass before
    uint32_t there0 = 0, there1 = 0;
    if (first > 0) walk.look_ahead(0);
    if (mine > 0) there0 = request_k(0);
    if (mine > 1) there1 = request_k(1);
    // row i: token first + i >> heads_log2, with its heads beyond 16 in tiles of their own
#pragma unroll 1
    for (int i = tid; i < rows * T::kChunks; i += kStatThreads) {
      const int row = i / T::kChunks, c = i % T::kChunks;
      const int k = row >> heads_log2, h = row & ((1 << heads_log2) - 1);
      const bool real = k < tokens && h < a.group;
      const size_t at = (static_cast<size_t>(u) * a.nodes + __shfl(my_node, min(first + k, kWave - 1), kWave)) * a.group + h;
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (real) v = load16(static_cast<const char*>(a.q) + at * T::kBytes + c * 16);
      *reinterpret_cast<uint4*>(q_s + row * T::kBytes + ((c ^ T::swizzle_k(row & 15)) << 4)) = v;
      if (c == 0) lse_s[row] = real ? a.lse[at] * kLog2e : INFINITY;
    }
    __syncthreads();
#pragma unroll 1
    for (int t = 0; t < mine; ++t) {
      const char* const tile = tiles + (t & 1) * kTileBytes;
      // (newer than the tile's loads: those of the tile after it, and the stores of the two before)
      if (t + 1 >= mine) wait_loads<0>();
      else if (t == 0) wait_loads<T::kLoads>();
      else wait_loads<T::kLoads + G>();
      uint4 kf[G][T::kSteps];
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int kk = 0; kk < T::kSteps; ++kk) kf[i][kk] = *reinterpret_cast<const uint4*>(tile + i * 16 * T::kBytes + (frag ^ (kk << 6)));
      reads_done();
      uint32_t there2 = 0;
      if (t + 2 < mine) there2 = request_k(t + 2);
      const bool of_fresh = walk.is_nodes(t);
      const int j0 = of_fresh ? walk.first_node(t) : walk.first_slot(t) - row0;
      float sum[G], sum2[G];
      int own[G], at[G];  // the first row that sees the slot, or the token; its position
#pragma unroll
      for (int i = 0; i < G; ++i) {
        sum[i] = sum2[i] = 0.0f;
        const int j = j0 + 16 * i + qi;
        own[i] = of_fresh ? j : 0;
        at[i] = !WINDOW ? 0 : of_fresh ? qp0 + j : pos_s[WINDOW ? min(j, kTreeChunk - 1) : 0];
      }
      // (a copy for each way in which heads share a tile: a dozen branches per tile of rows otherwise)
      const auto add_rows = [&](auto in_tile_of) {
        constexpr int in_tile = decltype(in_tile_of)::value, stride = 1 << (in_tile < 2 ? in_tile : 2);
        const bool holds = in_tile < 3 || (g & ((1 << (in_tile < 3 ? 0 : in_tile - 2)) - 1)) == 0;
#pragma unroll 1
        for (int tile0 = 0; tile0 < rows; tile0 += 16 * slices) {
          const int token0 = first + (tile0 >> heads_log2);
          f32x4 p[G];
#pragma unroll
          for (int i = 0; i < G; ++i) p[i] = f32x4{0};
#pragma unroll 1
          for (int row = tile0; row < tile0 + 16 * slices; row += 16) {
            const f32x4 lse = *reinterpret_cast<const f32x4*>(lse_s + row + 4 * g);
            const char* const q = q_s + row * T::kBytes;
            f32x4 s[G];
#pragma unroll
            for (int kk = 0; kk < T::kSteps; ++kk) {
              const uint4 qf = *reinterpret_cast<const uint4*>(q + (frag ^ (kk << 6)));
#pragma unroll
              for (int i = 0; i < G; ++i) s[i] = score_step<DT>(qf, kf[i][kk], kk == 0 ? f32x4{0} : s[i]);
            }
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float x = fmaf(s[i][e], sc, -lse[e]);
                if (WINDOW) x += static_cast<unsigned>(qp0 + token0 + ((4 * g + e) >> in_tile) - at[i]) < static_cast<unsigned>(w) ? bias : 0.0f;
                const float v = fast_exp2(x);
                p[i][e] += filled_up && lse[e] == INFINITY ? 0.0f : v;  // (0 times an infinite key is NaN)
              }
          }
#pragma unroll
          for (int i = 0; i < G; ++i) {
            if (in_tile >= 1) { p[i][0] += p[i][1]; p[i][2] += p[i][3]; }
            if (in_tile >= 2) p[i][0] += p[i][2];
            if (in_tile >= 3) p[i][0] += __shfl_xor(p[i][0], 16, kWave);
            if (in_tile >= 4) p[i][0] += __shfl_xor(p[i][0], 32, kWave);
          }
#pragma unroll
          for (int e = 0; e < 4; e += stride) {
            const int k = token0 + ((4 * g + e) >> in_tile);  // sees the tokens before it, and itself
            float second[G];
#pragma unroll
            for (int i = 0; i < G; ++i) {
              p[i][e] *= share;
              second[i] = p[i][e] * p[i][e];
            }
            if (!squares) {
#pragma unroll
              for (int i = 0; i < G; ++i)
                second[i] = a.pol.keeps_last_score() ? (k == len - 1 ? p[i][e] : 0.0f) : a.pol.second_statistic(0.0f, p[i][e], static_cast<float>(n + k + 1));
            }
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const bool counts = holds && k < len && k >= own[i];
              sum[i] += counts ? p[i][e] : 0.0f;
              sum2[i] += counts ? second[i] : 0.0f;
            }
          }
        }
      };
      switch (min(heads_log2, 4)) {
        case 0: add_rows(std::integral_constant<int, 0>()); break;
        case 1: add_rows(std::integral_constant<int, 1>()); break;
        case 2: add_rows(std::integral_constant<int, 2>()); break;
        case 3: add_rows(std::integral_constant<int, 3>()); break;
        default: add_rows(std::integral_constant<int, 4>()); break;
      }
#pragma unroll
      for (int i = 0; i < G; ++i) {
        sum[i] += __shfl_xor(sum[i], 16, kWave);
        sum[i] += __shfl_xor(sum[i], 32, kWave);
        sum2[i] += __shfl_xor(sum2[i], 16, kWave);
        sum2[i] += __shfl_xor(sum2[i], 32, kWave);
        // A slot's sums are its wave's alone: they go to memory at once (8 KiB of LDS for them would cost a workgroup per compute unit), as one
        // store of a count that the waits rely on: the first 16 lanes' Acc, the next 16 lanes' Acc2, the others' out of range.
        const int j = j0 + 16 * i + qi, step = of_fresh ? kMaxTreeNodes : a.B;
        float* const to = of_fresh ? fresh_sums : sums;
        float v = qi < static_cast<int>((there0 >> (8 * i)) & 0xffu) ? g == 0 ? sum[i] : sum2[i] : -1.0f;  // (below zero: a slot of no page, not seen)
        const bool there = g < 2 && j < (of_fresh ? len : row1 - row0);
        if (first > 0 && there) v += to[g * step + j];
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), __builtin_amdgcn_make_buffer_rsrc(to, 0, (step + (of_fresh ? len : row1 - row0)) * 4, 0x00020000),
                                              there ? (g * step + j) * 4 : 0x7ffffff0, 0, 0);
      }
      there0 = there1;
      there1 = there2;
    }
  }
}

// ------------------------------------------------------------------------------------------------
// 512 units x 2048 slots 7 us, 5 TB/s of the planes read and written (slot by slot, each with its own trip to memory, 9.7).
constexpr int kApplyThreads = 256;
constexpr int kApplySlots = kTreeChunk;  // of a workgroup
__global__ __launch_bounds__(kApplyThreads) void tree_apply(CommitArgs a, int row_bytes) {
  constexpr int kEach = kApplySlots / kApplyThreads;
  static_assert(kEach == 4, "a word of token_s per thread");
  __shared__ uint32_t token_s[kApplyThreads];  // a byte per slot: the accepted token that it takes, or 255
  const int u = blockIdx.x % a.units, row0 = blockIdx.x / a.units * kApplySlots;
  const int request = u / a.heads;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int32_t* const taken = a.taken + static_cast<size_t>(u) * kTakenWords;
  // (asked for together, a trip to memory: what lies behind the unit's last slot is the array's, and not used)
  const int len = taken[1], n_new = taken[2];
  const int my_slot = taken[4 + lane], my_node = path_node(a, request, min(lane, a.max_path - 1)), position = a.qpos0[u];
  float* const acc = a.stats + static_cast<size_t>(u) * 3 * a.B;
  float* const acc2 = acc + a.B;
  float* const cnt = acc2 + a.B;
  const float* const sums = a.sums + static_cast<size_t>(u) * 2 * a.B;
  const float* const fresh = a.fresh + static_cast<size_t>(u) * 2 * kMaxTreeNodes;
  float first[kEach], second[kEach], count[kEach], more[kEach], more2[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int j = min(row0 + tid + e * kApplyThreads, a.B - 1);
    first[e] = acc[j];
    second[e] = acc2[j];
    count[e] = cnt[j];
    more[e] = sums[j];
    more2[e] = sums[a.B + j];
  }
  const int row1 = min(n_new, row0 + kApplySlots);
  if (len == 0 || row0 >= row1) return;
  token_s[tid] = 0xffffffffu;
  __syncthreads();
  if (tid < len && my_slot >= row0 && my_slot < row1) {
    reinterpret_cast<uint8_t*>(token_s)[my_slot - row0] = static_cast<uint8_t>(tid);
    a.pos[static_cast<size_t>(u) * a.B + my_slot] = position + tid;
  }
  if (tid == 0 && row0 == 0) a.n_used[u] = n_new;
  __syncthreads();
  // the rows of the tokens whose slots are among these, 16 bytes per thread
  const int chunks = row_bytes / 16;
#pragma unroll 1
  for (int i = 0; i < len * chunks; i += kApplyThreads) {
    const int k = (i + tid) / chunks, c = (i + tid) - k * chunks;
    const int slot = __shfl(my_slot, k & (kWave - 1), kWave), node = __shfl(my_node, k & (kWave - 1), kWave);
    if (k >= len || slot < row0 || slot >= row1) continue;
    size_t row = static_cast<size_t>(u) * a.B + slot;
    if (a.pages.table != nullptr) {
      const int page = a.pages.table[static_cast<size_t>(request) * a.pages.max_pages + (slot >> a.pages.page_log2)];
      if (page < 0 || page >= a.pages.n_pages) continue;
      row = ((static_cast<size_t>(page) * a.heads + (u - request * a.heads)) << a.pages.page_log2) + (slot & ((1 << a.pages.page_log2) - 1));
    }
    const size_t src = (static_cast<size_t>(u) * a.nodes + node) * row_bytes + c * 16, dst = row * row_bytes + c * 16;
    const uint4 key = load16(static_cast<const char*>(a.k_new) + src), value = load16(static_cast<const char*>(a.v_new) + src);
    *reinterpret_cast<uint4*>(static_cast<char*>(a.K) + dst) = key;
    *reinterpret_cast<uint4*>(static_cast<char*>(a.V) + dst) = value;
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int j = tid + e * kApplyThreads;
    if (row0 + j >= row1) break;
    const int k = reinterpret_cast<const uint8_t*>(token_s)[j];
    const bool taken_over = k < kMaxTreeNodes;
    if (!taken_over && more[e] < 0.0f) continue;  // not seen: as it was
    acc[row0 + j] = taken_over ? fresh[k] : first[e] + more[e];
    acc2[row0 + j] = taken_over ? fresh[kMaxTreeNodes + k] : (a.pol.keeps_last_score() ? 0.0f : second[e]) + more2[e];
    cnt[row0 + j] = taken_over ? static_cast<float>(len - k) : count[e] + static_cast<float>(len);
  }
}

#pragma clang diagnostic pop

template <int DT, int HD, bool STREAMING, bool WINDOW> hipError_t launch_statistics(const CommitArgs& a, hipStream_t s) {
  ProfScope ps(kProfTreeStatistics, s);
  constexpr int kRowBytes = Tile<DT, HD>::kBytes, kTiles = kStatWaves * 2 * kStatTile<DT, HD>;
  constexpr int kMostStat = kTiles + kMostQueryLds / kRowBytes * (kRowBytes + 4), kMostChoice = (kChoiceWords + 2 * kMostChosenBeside) * 4;
  const RowPlan plan = row_plan(a.group, a.max_path, kRowBytes);
  const int choosers = a.B <= kMostChosenBeside ? a.units : 0;
  const void* const fn = reinterpret_cast<const void*>(tree_statistics<DT, HD, STREAMING, WINDOW>);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, std::max(kMostStat, kMostChoice)) != hipSuccess) return hipErrorInvalidValue;
  const int stat = kTiles + plan.rows(plan.per_pass) * (kRowBytes + 4), choice = choosers > 0 ? (kChoiceWords + 2 * a.B) * 4 : 0;
  hipLaunchKernelGGL((tree_statistics<DT, HD, STREAMING, WINDOW>), dim3(static_cast<unsigned>(choosers) + static_cast<unsigned>(a.units) * a.splits), dim3(kStatThreads),
                     std::max(stat, choice), s, a, plan, choosers);
  return hipGetLastError();
}

template <int DT, int HD> hipError_t launch_commit(const CommitArgs& a, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.B > kMostChosenBeside) {
    ProfScope ps(kProfTreeChoose, s);
    const size_t key_lds = key_lds_bytes(a.B);
    if (!allow_key_lds(reinterpret_cast<const void*>(tree_choose<true>), key_lds)) return hipErrorInvalidValue;
    if (key_lds == 0) hipLaunchKernelGGL((tree_choose<false>), dim3(a.units), dim3(kChooseThreads), 0, s, a);
    else hipLaunchKernelGGL((tree_choose<true>), dim3(a.units), dim3(kChooseThreads), key_lds, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.recency_window > 0) e = a.streaming ? launch_statistics<DT, HD, true, true>(a, s) : launch_statistics<DT, HD, false, true>(a, s);
  else e = a.streaming ? launch_statistics<DT, HD, true, false>(a, s) : launch_statistics<DT, HD, false, false>(a, s);
  if (e != hipSuccess) return e;
  ProfScope ps(kProfTreeApply, s);
  const unsigned chunks = static_cast<unsigned>((a.B + kApplySlots - 1) / kApplySlots);
  hipLaunchKernelGGL(tree_apply, dim3(static_cast<unsigned>(a.units) * chunks), dim3(kApplyThreads), 0, s, a, Tile<DT, HD>::kBytes);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_commit(int dtype, int head_dim, const CommitArgs& a, hipStream_t s) {
  if (dtype == kBF16) return head_dim == 128 ? launch_commit<kBF16, 128>(a, s) : launch_commit<kBF16, 64>(a, s);
  return head_dim == 128 ? launch_commit<kF32, 128>(a, s) : launch_commit<kF32, 64>(a, s);
}

}  // namespace roco
