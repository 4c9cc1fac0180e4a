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
constexpr size_t kMostQueryLds = 40960;  // bytes of accepted query rows that are kept in LDS

// The accepted rows in tiles of 16 tokens of one head.  A head's probabilities are formed a tile at a time and added up over the heads
// in registers: Q is the A operand here, so that a lane holds four tokens of one slot and the sum over the tokens is over its registers
// and two exchanges.  STAGED: the query rows are in LDS (they fit), else read where they are.
template <int DT, int HD, bool STREAMING, bool WINDOW, bool STAGED>
__global__ __launch_bounds__(kStatThreads, 2) void tree_statistics(CommitArgs a) {
  using T = Tile<DT, HD>;
  constexpr int W = kStatWaves, G = T::kGroups, kTileBytes = 8192;
  extern __shared__ __attribute__((aligned(1024))) char lds[];  // the waves' tiles, two each; then the query rows
  __shared__ float sum_s[kTreeChunk], sum2_s[kTreeChunk];
  __shared__ signed char token_s[kTreeChunk];  // accepted token that a slot has taken, or -1
  __shared__ int32_t pos_s[WINDOW ? kTreeChunk : 1];
  __shared__ int node_s[kMaxTreeNodes];
  const int u = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const int request = u / a.heads;
  const int32_t* const taken = a.taken + static_cast<size_t>(u) * kTakenWords;
  const int n = __builtin_amdgcn_readfirstlane(taken[0]), len = __builtin_amdgcn_readfirstlane(taken[1]), n_new = __builtin_amdgcn_readfirstlane(taken[2]);
  if (len == 0) return;
  constexpr int kStep = T::kSlots * W;
  static_assert(kTreeChunk % kStep == 0, "a chunk of whole tiles");
  const int chunk = ((n_new + a.splits - 1) / a.splits + kStep - 1) / kStep * kStep;
  const int row0 = min(n_new, split * chunk), row1 = min(n_new, row0 + chunk);
  if (row0 >= row1) return;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int qi = lane & 15, g = lane >> 4;

  Walk<DT, HD, W> walk;
  walk.init(a.pages, a.B, a.heads, u, request, row0, row1, 0, wave, static_cast<unsigned>(u) * 5u + static_cast<unsigned>(split) * 3u);
  const int mine = walk.mine;
  char* const tiles = lds + wave * 2 * kTileBytes;
  const uint32_t tiles_addr = lds_address(tiles);
  int koff[T::kGroupLoads];
  load_offsets<DT, HD, false>(koff);
  typedef typename Walk<DT, HD, W>::Place Place;
  uint32_t there[3] = {0, 0, 0};
  auto request_k = [&](int t) {
    const Place p = walk.place(t);
    request_tile<DT, HD, STREAMING>(a.K, p.row, p.there, tiles_addr + (t & 1) * kTileBytes, koff);
    return p.there;
  };
  if (mine > 0) there[0] = request_k(0);
  if (mine > 1) there[1] = request_k(1);

  // ---- the accepted rows
  const int token_tiles = (len + 15) / 16, padded = token_tiles * 16;
  char* const q_s = lds + W * 2 * kTileBytes;
  float* const lse_s = reinterpret_cast<float*>(q_s + (STAGED ? static_cast<size_t>(a.group) * padded * T::kBytes : 0));  // [group][padded], base 2
  if (tid < len) node_s[tid] = path_node(a, request, tid);
  for (int j = tid; j < kTreeChunk; j += kStatThreads) {
    token_s[j] = -1;
    if (WINDOW && row0 + j < row1) pos_s[WINDOW ? j : 0] = a.pos[static_cast<size_t>(u) * a.B + row0 + j];
  }
  __syncthreads();
  if (tid < len) {
    const int j = taken[4 + tid] - row0;
    if (j >= 0 && j < row1 - row0) token_s[j] = static_cast<signed char>(tid);
  }
  for (int i = tid; i < a.group * padded; i += kStatThreads) {
    const int h = i / padded, k = i % padded;
    lse_s[i] = k < len ? a.lse[(static_cast<size_t>(u) * a.nodes + node_s[k]) * a.group + h] * kLog2e : 0.0f;
  }
  if (STAGED) {
    for (int i = tid; i < a.group * padded * T::kChunks; i += kStatThreads) {
      const int row = i / T::kChunks, c = i % T::kChunks, h = row / padded, k = row % padded;
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (k < len) v = load16(static_cast<const char*>(a.q) + ((static_cast<size_t>(u) * a.nodes + node_s[k]) * a.group + h) * T::kBytes + c * 16);
      *reinterpret_cast<uint4*>(q_s + row * T::kBytes + ((c ^ T::swizzle_k(row & 15)) << 4)) = v;
    }
  }
  __syncthreads();

  const float sc = a.scale_log2, rb = a.recency_bias_log2, share = 1.0f / static_cast<float>(a.group);
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[u] : 0;
  const int frag = qi * T::kBytes + ((g ^ T::swizzle_k(qi)) << 4);
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
    if (t + 2 < mine) there[2] = request_k(t + 2);
    const int j0 = walk.first_slot(t) - row0;
    float sum[G], sum2[G];
    int own[G], at[G];
#pragma unroll
    for (int i = 0; i < G; ++i) {
      sum[i] = sum2[i] = 0.0f;
      own[i] = token_s[j0 + 16 * i + qi];
      at[i] = WINDOW ? pos_s[WINDOW ? j0 + 16 * i + qi : 0] : 0;
    }
#pragma unroll 1
    for (int tt = 0; tt < token_tiles; ++tt) {
      f32x4 p[G];
#pragma unroll
      for (int i = 0; i < G; ++i) p[i] = f32x4{0};
#pragma unroll 1
      for (int h = 0; h < a.group; ++h) {
        const int row = h * padded + 16 * tt;
        const f32x4 lse = *reinterpret_cast<const f32x4*>(lse_s + row + 4 * g);
        const char* const q = STAGED ? q_s + row * T::kBytes
                                     : static_cast<const char*>(a.q) + ((static_cast<size_t>(u) * a.nodes + node_s[min(16 * tt + qi, len - 1)]) * a.group + h) * T::kBytes;
        f32x4 s[G];
#pragma unroll
        for (int kk = 0; kk < T::kSteps; ++kk) {
          const uint4 qf = STAGED ? *reinterpret_cast<const uint4*>(q + (frag ^ (kk << 6))) : load16(q + kk * 64 + g * 16);
#pragma unroll
          for (int i = 0; i < G; ++i) s[i] = score_step<DT>(qf, kf[i][kk], kk == 0 ? f32x4{0} : s[i]);
        }
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = fmaf(s[i][e], sc, -lse[e]);
            if (WINDOW) {
              const int away = qp0 + 16 * tt + 4 * g + e - at[i];
              if (away >= 0 && away < w) x += rb;
            }
            p[i][e] += fast_exp2(x);
          }
      }
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = 16 * tt + 4 * g + e;  // sees the tokens before it, and itself
          const float v = p[i][e] * share;
          if (k < len && k >= own[i]) {
            sum[i] += v;
            sum2[i] += a.pol.keeps_last_score() ? (k == len - 1 ? v : 0.0f) : a.pol.second_statistic(0.0f, v, static_cast<float>(n + k + 1));
          }
        }
    }
#pragma unroll
    for (int i = 0; i < G; ++i) {
      sum[i] += __shfl_xor(sum[i], 16, kWave);
      sum[i] += __shfl_xor(sum[i], 32, kWave);
      sum2[i] += __shfl_xor(sum2[i], 16, kWave);
      sum2[i] += __shfl_xor(sum2[i], 32, kWave);
      const bool real = qi < static_cast<int>((there[0] >> (8 * i)) & 0xffu);  // slots of no page have received nothing
      if (g == 0) {
        sum_s[j0 + 16 * i + qi] = real ? sum[i] : 0.0f;
        sum2_s[j0 + 16 * i + qi] = real ? sum2[i] : 0.0f;
      }
    }
    there[0] = there[1];
    there[1] = there[2];
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

template <int DT, int HD, bool STREAMING, bool WINDOW, bool STAGED> hipError_t launch_statistics(const CommitArgs& a, size_t lds, hipStream_t s) {
  constexpr int kMost = kStatWaves * 2 * 8192 + static_cast<int>(kMostQueryLds) + kMaxTreeNodes * kMaxTreeGroup * 4;
  const void* const fn = reinterpret_cast<const void*>(tree_statistics<DT, HD, STREAMING, WINDOW, STAGED>);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kMost) != hipSuccess) return hipErrorInvalidValue;
  hipLaunchKernelGGL((tree_statistics<DT, HD, STREAMING, WINDOW, STAGED>), dim3(static_cast<unsigned>(a.units) * a.splits), dim3(kStatThreads), lds, s, a);
  return hipGetLastError();
}

template <int DT, int HD, bool STREAMING> hipError_t launch_statistics_form(const CommitArgs& a, bool staged, size_t lds, hipStream_t s) {
  if (a.recency_window > 0)
    return staged ? launch_statistics<DT, HD, STREAMING, true, true>(a, lds, s) : launch_statistics<DT, HD, STREAMING, true, false>(a, lds, s);
  return staged ? launch_statistics<DT, HD, STREAMING, false, true>(a, lds, s) : launch_statistics<DT, HD, STREAMING, false, false>(a, lds, s);
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
  const size_t rows = static_cast<size_t>(a.group) * ((a.max_path + 15) / 16 * 16);
  const bool staged = rows * kRowBytes <= kMostQueryLds;
  const size_t lds = kStatWaves * 2 * 8192 + (staged ? rows * kRowBytes : 0) + rows * 4;
  return a.streaming ? launch_statistics_form<DT, HD, true>(a, staged, lds, s) : launch_statistics_form<DT, HD, false>(a, staged, lds, s);
}

}  // namespace

hipError_t launch_tree_commit(int dtype, int head_dim, const CommitArgs& a, hipStream_t s) {
  if (dtype == kBF16) return head_dim == 128 ? launch_commit<kBF16, 128>(a, s) : launch_commit<kBF16, 64>(a, s);
  return head_dim == 128 ? launch_commit<kF32, 128>(a, s) : launch_commit<kF32, 64>(a, s);
}

}  // namespace roco
