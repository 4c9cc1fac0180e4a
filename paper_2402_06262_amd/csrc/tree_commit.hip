// A drafted tree's accepted path taken over into the budgeted cache.
//
//   tree_take       : one workgroup per unit.  E = max(0, n + a - budget) victims by the statistics as they stand (two exact searches, as
//                     in block_prepare), the accepted tokens to the freed and the empty slots in order, their K / V rows into the cache.
//   tree_statistics : up to 1024 slots per workgroup.  The accepted rows' probabilities are formed again, exp(logit - lse), from one pass
//                     over K alone: half of what the attention has read, where probabilities left behind by the attention would be 4 bytes
//                     per slot, head and node, of which the accepted ones are known only now.
#include <algorithm>

#include "profile.hpp"
#include "tree.hpp"

namespace roco {
namespace {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

using namespace tree;

__device__ __forceinline__ int path_length(const CommitArgs& a, int request, int budget) {
  return min(max(a.n_path[request], 0), min(a.max_path, budget));
}
__device__ __forceinline__ int path_node(const CommitArgs& a, int request, int k) {
  return min(max(a.path[static_cast<size_t>(request) * a.max_path + k], 0), a.nodes - 1);
}

// LDS: the ranking keys are in LDS (B <= kMaxDecodeBudgetLds).
template <int NT, bool LDS> __global__ __launch_bounds__(NT, 8) void tree_take(CommitArgs a, int row_bytes) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds_keys[];  // [2][B]
  __shared__ __attribute__((aligned(16))) uint32_t sel_sh[SelectLds<1>::kWords];
  __shared__ uint32_t scan_sh[NT / kWave + 1];
  __shared__ int slot_of[kMaxTreeNodes];
  const int u = blockIdx.x, tid = threadIdx.x, B = a.B;
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
    taken[0] = n;
    taken[1] = len;
    taken[2] = n_new;
  }
  if (len == 0) return;
  const float* const acc = a.stats + static_cast<size_t>(u) * 3 * B;
  const float* const acc2 = acc + B;
  const float* const cnt = acc2 + B;
  int32_t* const pos = a.pos + static_cast<size_t>(u) * B;
  uint32_t* const var_key = LDS ? lds_keys : a.keys + static_cast<size_t>(u) * 2 * B;
  uint32_t* const mas_key = var_key + B;
  KSmallest scope = {0u, 0u}, out = {0u, 0u};
  if (E > 0) {
#pragma unroll 1
    for (int i = tid; i < n; i += NT) ranking_keys(acc[i], acc2[i], cnt[i], pos[i], a.pol, mas_key[i], var_key[i]);
    __syncthreads();
    const uint32_t m = min(static_cast<uint32_t>(n), static_cast<uint32_t>(a.pol.scope_size(min(a.scope, budget), n)) + static_cast<uint32_t>(E) - 1u);
#pragma unroll 1
    for (int phase = 0; phase < 2; ++phase) {
      const KSmallest r = select_k_smallest<NT, 1, 1>(
          [&](int i) -> uint32_t {
            const uint32_t vk = var_key[i];
            return phase == 0 ? vk : scope.has(vk, i) ? mas_key[i] : 0xffffffffu;
          },
          n, phase == 0 ? m : static_cast<uint32_t>(E), phase == 0 && a.pol.scope_is_window(), sel_sh, phase == 0 || a.pol.spreads_importance());
      if (phase == 0) scope = r;
      else out = r;
    }
  }
  auto is_target = [&](int j) -> bool {
    if (j >= n) return j < n_new;
    if (E == 0) return false;
    return out.has(scope.has(var_key[j], j) ? mas_key[j] : 0xffffffffu, j);
  };
  // thread t owns the slots [t c, (t + 1) c); the i-th target takes the i-th token
  const int c = (n_new + NT - 1) / NT;
  const int lo = min(n_new, tid * c), hi = min(n_new, lo + c);
  uint32_t mine = 0;
#pragma unroll 1
  for (int j = lo; j < hi; ++j) mine += is_target(j) ? 1u : 0u;
  uint32_t total;
  uint32_t rank = block_exclusive_scan<NT>(mine, scan_sh, total);
#pragma unroll 1
  for (int j = lo; j < hi; ++j) {
    if (!is_target(j) || rank >= static_cast<uint32_t>(len)) continue;
    const int k = static_cast<int>(rank++);
    slot_of[k] = j;
    taken[4 + k] = j;
    const bool held = j < n;  // by a token that is now evicted
    if (a.evicted_slot != nullptr) a.evicted_slot[static_cast<size_t>(u) * a.max_path + k] = held ? j : -1;
    if (a.evicted_pos != nullptr) a.evicted_pos[static_cast<size_t>(u) * a.max_path + k] = held ? pos[j] : -1;
    pos[j] = a.qpos0[u] + k;
  }
  __syncthreads();
  if (tid == 0) a.n_used[u] = n_new;
  const int lanes = row_bytes / 16;
#pragma unroll 1
  for (int i = tid; i < len * lanes; i += NT) {
    const int k = i / lanes, col = i % lanes * 16, slot = slot_of[k];
    const size_t src = (static_cast<size_t>(u) * a.nodes + path_node(a, request, k)) * row_bytes + col;
    size_t row = static_cast<size_t>(u) * B + slot;
    if (a.pages.table != nullptr) {
      const int page = a.pages.table[static_cast<size_t>(request) * a.pages.max_pages + (slot >> a.pages.page_log2)];
      if (page < 0 || page >= a.pages.n_pages) continue;
      row = ((static_cast<size_t>(page) * a.heads + (u - request * a.heads)) << a.pages.page_log2) + (slot & ((1 << a.pages.page_log2) - 1));
    }
    *reinterpret_cast<uint4*>(static_cast<char*>(a.K) + row * row_bytes + col) = load16(static_cast<const char*>(a.k_new) + src);
    *reinterpret_cast<uint4*>(static_cast<char*>(a.V) + row * row_bytes + col) = load16(static_cast<const char*>(a.v_new) + src);
  }
}

constexpr int kStatWaves = 4;
constexpr int kStatThreads = kStatWaves * kWave;
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

// Q is the A operand here, so that a lane holds four rows of one slot.  The accepted tokens' K rows have been written to their slots: a slot of
// token m is one that the rows before m do not see.  More rows than the LDS takes: another pass over K (which the L2 mostly has).
template <int DT, int HD, bool STREAMING, bool WINDOW>
__global__ __launch_bounds__(kStatThreads, 4) void tree_statistics(CommitArgs a, RowPlan plan) {
  constexpr int kTileBytes = kStatTile<DT, HD>;
  using T = Tile<DT, HD, kTileBytes>;
  constexpr int W = kStatWaves, G = T::kGroups;
  extern __shared__ __attribute__((aligned(1024))) char lds[];  // the waves' tiles, two each; then the query rows and their normalisers
  __shared__ float sum_s[kTreeChunk], sum2_s[kTreeChunk];
  __shared__ signed char token_s[kTreeChunk];  // accepted token that a slot has taken, or -1
  __shared__ int32_t pos_s[WINDOW ? kTreeChunk : 1];
  const int u = blockIdx.x % a.units, split = blockIdx.x / a.units;
  const int request = u / a.heads;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int qi = lane & 15, g = lane >> 4;
  const int32_t* const taken = a.taken + static_cast<size_t>(u) * kTakenWords;
  // (what has to come from memory before anything else is asked for together)
  const int my_slot = taken[4 + lane], my_node = path_node(a, request, min(lane, a.max_path - 1));
  const int n = __builtin_amdgcn_readfirstlane(taken[0]), len = __builtin_amdgcn_readfirstlane(taken[1]), n_new = __builtin_amdgcn_readfirstlane(taken[2]);
  const int row0 = split * a.chunk, row1 = min(n_new, row0 + a.chunk);
  if (len == 0 || row0 >= row1) return;

  Walk<DT, HD, W, kTileBytes> walk;
  walk.init(a.pages, a.B, a.heads, u, request, row0, row1, 0, wave, static_cast<unsigned>(u) * 5u + static_cast<unsigned>(split) * 3u);
  const int mine = walk.mine;
  char* const tiles = lds + wave * 2 * kTileBytes;
  const uint32_t tiles_addr = lds_address(tiles);
  int koff[T::kGroupLoads];
  load_offsets<DT, HD, false>(koff);
  auto request_k = [&](int t) {
    const typename Walk<DT, HD, W, kTileBytes>::Place p = walk.place(t);
    request_tile<DT, HD, STREAMING>(a.K, p.row, p.there, tiles_addr + (t & 1) * kTileBytes, koff);
    return p.there;
  };
  for (int j = tid; j < row1 - row0; j += kStatThreads) {
    token_s[j] = -1;
    sum_s[j] = sum2_s[j] = 0.0f;
    if (WINDOW) pos_s[WINDOW ? j : 0] = a.pos[static_cast<size_t>(u) * a.B + row0 + j];
  }
  __syncthreads();
  if (tid < len && my_slot >= row0 && my_slot < row1) token_s[my_slot - row0] = static_cast<signed char>(tid);

  const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f, share = 1.0f / static_cast<float>(a.group);
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[u] : 0;
  const int frag = qi * T::kBytes + ((g ^ T::swizzle_k(qi)) << 4);
  // of the lane's four rows of a tile, those whose register holds a token's sum over its heads in the end
  const int heads_log2 = plan.heads_log2, in_tile = min(heads_log2, 4);
  const int slices = 1 << (heads_log2 - in_tile);  // tiles of a token
  const bool filled_up = (1 << heads_log2) != a.group;
  const int stride = 1 << min(in_tile, 2);
  const bool holds = in_tile < 3 || (g & ((1 << (in_tile - 2)) - 1)) == 0;
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
      if (t + 1 < mine) wait_loads<T::kLoads>();
      else wait_loads<0>();
      uint4 kf[G][T::kSteps];
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int kk = 0; kk < T::kSteps; ++kk) kf[i][kk] = *reinterpret_cast<const uint4*>(tile + i * 16 * T::kBytes + (frag ^ (kk << 6)));
      reads_done();
      uint32_t there2 = 0;
      if (t + 2 < mine) there2 = request_k(t + 2);
      const int j0 = walk.first_slot(t) - row0;
      float sum[G], sum2[G];
      int own[G], at[G];
#pragma unroll
      for (int i = 0; i < G; ++i) {
        sum[i] = sum2[i] = 0.0f;
        const int j = min(j0 + 16 * i + qi, row1 - row0 - 1);
        own[i] = token_s[j];
        at[i] = WINDOW ? pos_s[WINDOW ? j : 0] : 0;
      }
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
        for (int e = 0; e < 4; ++e) {
          if ((e & (stride - 1)) != 0) continue;
          const int k = token0 + ((4 * g + e) >> in_tile);  // sees the tokens before it, and itself
#pragma unroll
          for (int i = 0; i < G; ++i) {
            const float v = p[i][e] * share;
            const bool counts = holds && k < len && k >= own[i];
            const float second = a.pol.keeps_last_score() ? (k == len - 1 ? v : 0.0f) : a.pol.second_statistic(0.0f, v, static_cast<float>(n + k + 1));
            sum[i] += counts ? v : 0.0f;
            sum2[i] += counts ? second : 0.0f;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < G; ++i) {
        sum[i] += __shfl_xor(sum[i], 16, kWave);
        sum[i] += __shfl_xor(sum[i], 32, kWave);
        sum2[i] += __shfl_xor(sum2[i], 16, kWave);
        sum2[i] += __shfl_xor(sum2[i], 32, kWave);
        if (g == 0 && qi < static_cast<int>((there0 >> (8 * i)) & 0xffu)) {  // (slots of no page have received nothing)
          sum_s[j0 + 16 * i + qi] += sum[i];
          sum2_s[j0 + 16 * i + qi] += sum2[i];
        }
      }
      there0 = there1;
      there1 = there2;
    }
  }
  __syncthreads();
  // ---- the slots' statistics: added to those of older tokens, the first ones of the accepted
  float* const acc = a.stats + static_cast<size_t>(u) * 3 * a.B + row0;
  float* const acc2 = acc + a.B;
  float* const cnt = acc2 + a.B;
  for (int j = tid; j < row1 - row0; j += kStatThreads) {
    const int k = token_s[j];
    const bool old = k < 0;
    acc[j] = (old ? acc[j] : 0.0f) + sum_s[j];
    acc2[j] = (old && !a.pol.keeps_last_score() ? acc2[j] : 0.0f) + sum2_s[j];
    cnt[j] = old ? cnt[j] + static_cast<float>(len) : static_cast<float>(len - k);
  }
}

#pragma clang diagnostic pop

template <int DT, int HD, bool STREAMING, bool WINDOW> hipError_t launch_statistics(const CommitArgs& a, hipStream_t s) {
  constexpr int kRowBytes = Tile<DT, HD>::kBytes, kTiles = kStatWaves * 2 * kStatTile<DT, HD>, kMost = kTiles + kMostQueryLds / kRowBytes * (kRowBytes + 4);
  const RowPlan plan = row_plan(a.group, a.max_path, kRowBytes);
  const void* const fn = reinterpret_cast<const void*>(tree_statistics<DT, HD, STREAMING, WINDOW>);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kMost) != hipSuccess) return hipErrorInvalidValue;
  const size_t lds = kTiles + static_cast<size_t>(plan.rows(plan.per_pass)) * (kRowBytes + 4);
  hipLaunchKernelGGL((tree_statistics<DT, HD, STREAMING, WINDOW>), dim3(static_cast<unsigned>(a.units) * a.splits), dim3(kStatThreads), lds, s, a, plan);
  return hipGetLastError();
}

template <int DT, int HD> hipError_t launch_commit(const CommitArgs& a, hipStream_t s) {
  constexpr int kRowBytes = Tile<DT, HD>::kBytes;
  const size_t key_lds = key_lds_bytes(a.B);
  if (!allow_key_lds(reinterpret_cast<const void*>(tree_take<512, true>), key_lds) ||
      !allow_key_lds(reinterpret_cast<const void*>(tree_take<1024, true>), key_lds))
    return hipErrorInvalidValue;
  {
    ProfScope ps(kProfTreeTake, s);
    if (key_lds == 0) hipLaunchKernelGGL((tree_take<1024, false>), dim3(a.units), dim3(1024), 0, s, a, kRowBytes);
    else if (a.units > 256) hipLaunchKernelGGL((tree_take<512, true>), dim3(a.units), dim3(512), key_lds, s, a, kRowBytes);
    else hipLaunchKernelGGL((tree_take<1024, true>), dim3(a.units), dim3(1024), key_lds, s, a, kRowBytes);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope ps(kProfTreeStatistics, s);
  if (a.recency_window > 0) return a.streaming ? launch_statistics<DT, HD, true, true>(a, s) : launch_statistics<DT, HD, false, true>(a, s);
  return a.streaming ? launch_statistics<DT, HD, true, false>(a, s) : launch_statistics<DT, HD, false, false>(a, s);
}

}  // namespace

hipError_t launch_tree_commit(int dtype, int head_dim, const CommitArgs& a, hipStream_t s) {
  if (dtype == kBF16) return head_dim == 128 ? launch_commit<kBF16, 128>(a, s) : launch_commit<kBF16, 64>(a, s);
  return head_dim == 128 ? launch_commit<kF32, 128>(a, s) : launch_commit<kF32, 64>(a, s);
}

}  // namespace roco
