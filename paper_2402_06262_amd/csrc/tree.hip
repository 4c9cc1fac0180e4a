// Drafted trees: the joining of the splits' shares, and which form of tree_attend a call takes.
#include <stdlib.h>

#include <algorithm>

#include "profile.hpp"
#include "tree.hpp"

namespace roco {

hipError_t launch_tree_attend_bf16_128(const TreeArgs& a, hipStream_t s);  // a file each
hipError_t launch_tree_attend_bf16_64(const TreeArgs& a, hipStream_t s);
hipError_t launch_tree_attend_f32_128(const TreeArgs& a, hipStream_t s);
hipError_t launch_tree_attend_f32_64(const TreeArgs& a, hipStream_t s);

namespace {

constexpr int kJoinThreads = 256;

// A wave per query row: its splits' maxima and sums, a lane each, then their outputs, weighted, in the order of the splits.
template <int DT, int HD> __global__ __launch_bounds__(kJoinThreads) void tree_join(TreeArgs a) {
  constexpr int E = HD / kWave;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int all = a.nodes * a.group;
  const long long id = static_cast<long long>(blockIdx.x) * (kJoinThreads / kWave) + wave;
  const int u = static_cast<int>(id / all), row = static_cast<int>(id % all);
  if (u >= a.units) return;
  const int request = u / a.heads;
  const int nodes = a.n_nodes != nullptr ? min(max(a.n_nodes[request], 0), a.nodes) : a.nodes;
  if (row >= nodes * a.group) return;
  const int splits = tree::splits_used(min(max(a.n_used[u], 0), tree::budget_of(a.pages, a.B, request)), a.chunk);
  if (splits == 1) return;  // has written its rows
  const size_t first = static_cast<size_t>(u) * a.splits * all + row;  // of split 0; the others `all` further each
  float m = -INFINITY, l = 0.0f;
  if (lane < splits) {
    m = a.part_m[first + static_cast<size_t>(lane) * all];
    l = a.part_l[first + static_cast<size_t>(lane) * all];
  }
  const float M = group_max<kWave>(m);
  const float w = m > -INFINITY ? fast_exp2(m - M) : 1.0f;  // (a split of no maximum has a sum of zero, or NaN)
  const float sum = group_sum<kWave>(l * w);
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.0f;
  for (int i0 = 0; i0 < splits; i0 += 4) {  // four at a time: behind the last split its outputs again, with nothing of them
    float v[4][E];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float* const p = a.part_o + (first + static_cast<size_t>(min(i0 + k, splits - 1)) * all) * HD + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = p[e];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float wk = __shfl(w, min(i0 + k, kWave - 1), kWave);
      if (i0 + k >= splits) break;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(wk, v[k][e], o[e]);
    }
  }
  const float scale = 1.0f / sum;
  const size_t at = static_cast<size_t>(u) * all + row;
#pragma unroll
  for (int e = 0; e < E; ++e) store_elem<DT>(a.out, at * HD + lane * E + e, o[e] * scale);
  if (a.lse != nullptr && lane == 0) a.lse[at] = 0.6931471805599453f * (M + __log2f(sum));
}

template <int DT, int HD> hipError_t launch_join(const TreeArgs& a, hipStream_t s) {
  ProfScope ps(kProfTreeJoin, s);
  const long long rows = static_cast<long long>(a.units) * a.nodes * a.group;
  const unsigned blocks = static_cast<unsigned>((rows + kJoinThreads / kWave - 1) / (kJoinThreads / kWave));
  hipLaunchKernelGGL((tree_join<DT, HD>), dim3(blocks), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Query rows of a workgroup: 64, or of bf16 192 (128 with a recency window, whose code has no registers for the third tile of a wave).
int tree_attend_row_tiles(int dtype, int rows, bool window) {
  const int most = dtype != kBF16 || rows <= 64 ? 64 : window ? 128 : 192;
  return (rows + most - 1) / most;
}

// Two workgroups on every compute unit, while each has 64 slots (with more than 64 rows of bf16 192: its share of the outputs is larger).
TreeSplits tree_attend_splits(int dtype, int units, int rows, int B, bool window) {
  const char* const asked = getenv("ROCO_TREE_SPLITS");
  int want = asked != nullptr ? atoi(asked) : 0;
  if (want <= 0) {
    const long long groups = static_cast<long long>(units) * tree_attend_row_tiles(dtype, rows, window);
    want = static_cast<int>((512 + groups - 1) / groups);
    if (dtype == kBF16 && rows > 64) want = std::min(want, (B + 191) / 192);
  }
  want = std::max(1, std::min({want, kMaxTreeSplits, (B + 63) / 64}));
  TreeSplits s;
  s.chunk = ((B + want - 1) / want + 63) / 64 * 64;
  s.splits = (B + s.chunk - 1) / s.chunk;
  return s;
}

hipError_t launch_tree_attend(int dtype, int head_dim, const TreeArgs& a, hipStream_t s) {
  hipError_t e;
  {
    ProfScope ps(kProfTreeAttend, s);
    if (dtype == kBF16) e = head_dim == 128 ? launch_tree_attend_bf16_128(a, s) : launch_tree_attend_bf16_64(a, s);
    else e = head_dim == 128 ? launch_tree_attend_f32_128(a, s) : launch_tree_attend_f32_64(a, s);
  }
  if (e != hipSuccess || a.splits == 1) return e;
  if (dtype == kBF16) return head_dim == 128 ? launch_join<kBF16, 128>(a, s) : launch_join<kBF16, 64>(a, s);
  return head_dim == 128 ? launch_join<kF32, 128>(a, s) : launch_join<kF32, 64>(a, s);
}

}  // namespace roco
