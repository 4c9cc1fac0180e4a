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
constexpr int kJoinAhead = 4;  // of a lane's loads

// WAVES waves per query row: its splits' maxima and sums, a lane each, then their outputs, weighted.  HD / 4 lanes take a split's 16 bytes at a
// time, so that a wave has 2 or 4 splits in hand; the sums over the lanes and the waves have a fixed order.  What bounds it is the
// latency of its loads: one wave per row with two of a split's elements per lane took 14 us for 1024 rows of 32 splits.
template <int DT, int HD, int WAVES> __global__ __launch_bounds__(kJoinThreads) void tree_join(TreeArgs a) {
  constexpr int LANES = HD / 4, PER = kWave / LANES, STEP = PER * WAVES * kJoinAhead;
  constexpr int ROWS = kJoinThreads / kWave / WAVES;  // of a workgroup
  __shared__ __attribute__((aligned(16))) float other_s[WAVES > 1 ? ROWS * WAVES : 1][WAVES > 1 ? HD : 1];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int part = wave % WAVES;
  const int all = a.nodes * a.group;
  const long long id = static_cast<long long>(blockIdx.x) * ROWS + wave / WAVES;
  const int u = static_cast<int>(id / all), row = static_cast<int>(id % all);
  if (u >= a.units) return;  // (a row's waves go together: with several of them a workgroup has one row)
  const int request = u / a.heads;
  const int nodes = a.n_nodes != nullptr ? min(max(a.n_nodes[request], 0), a.nodes) : a.nodes;
  const int splits = tree::splits_used(min(max(a.n_used[u], 0), tree::budget_of(a.pages, a.B, request)), a.chunk);
  if (row >= nodes * a.group || splits == 1) return;  // (the only split has written its rows)
  const size_t first = static_cast<size_t>(u) * a.splits * all + row;  // of split 0; the others `all` further each
  float m = -INFINITY, l = 0.0f;
  if (lane < splits) {
    m = a.part_m[first + static_cast<size_t>(lane) * all];
    l = a.part_l[first + static_cast<size_t>(lane) * all];
  }
  const int col = lane % LANES * 4, mine = lane / LANES * WAVES + part;  // this lane's splits: mine, mine + PER * WAVES, ...
  tree::f32x4 o = tree::f32x4{0};
  float M = 0.0f, w = 0.0f;
#pragma unroll 1
  for (int i0 = 0; i0 < splits; i0 += STEP) {
    tree::f32x4 v[kJoinAhead];
#pragma unroll
    for (int k = 0; k < kJoinAhead; ++k) {
      const int i = min(i0 + mine + k * PER * WAVES, splits - 1);
      v[k] = *reinterpret_cast<const tree::f32x4*>(a.part_o + (first + static_cast<size_t>(i) * all) * HD + col);
    }
    if (i0 == 0) {
      M = group_max<kWave>(m);
      w = m > -INFINITY ? fast_exp2(m - M) : 1.0f;  // (a split of no maximum has a sum of zero, or NaN)
    }
#pragma unroll
    for (int k = 0; k < kJoinAhead; ++k) {
      const int i = i0 + mine + k * PER * WAVES;
      const float wk = __shfl(w, min(i, kWave - 1), kWave);
      if (i < splits) o += v[k] * wk;
    }
  }
#pragma unroll
  for (int step = LANES; step < kWave; step *= 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], step, kWave);
  }
  if (WAVES > 1) {
    if (lane < LANES) *reinterpret_cast<tree::f32x4*>(&other_s[wave][WAVES > 1 ? col : 0]) = o;
    __syncthreads();
    if (part != 0) return;
    o = tree::f32x4{0};
#pragma unroll
    for (int k = 0; k < WAVES; ++k) o += *reinterpret_cast<const tree::f32x4*>(&other_s[WAVES > 1 ? wave + k : 0][WAVES > 1 ? col : 0]);
  }
  const float sum = group_sum<kWave>(l * w);
  const size_t at = static_cast<size_t>(u) * all + row;
  if (lane < LANES) tree::store4<DT>(a.out, at * HD + col, o * (1.0f / sum));
  if (a.lse != nullptr && lane == 0) a.lse[at] = 0.6931471805599453f * (M + __log2f(sum));
}

// Few splits of many rows: HD / 4 lanes and their 16 bytes have kJoinRows rows each, so that the loads of all of them are in flight (a wave per row
// took 21 us for 65536 rows of two splits, 63 MB, and these 9.8; 1260 rows 4.8 and 6.2).  The sums over the splits are in their order.
// The borders, whole attentions in us: 16384 rows of two and four splits 29.1 and 27.5, by a wave per row 32.5 and 29.9, but 4096 rows 32.5 and 26.8 by
// these, 32.7 and 26.6 by a wave per row.  Eight splits of 65536 and 8192 rows 175 and 45, by four waves per row 214 and 50; 16 splits of 65536 rows
// 320 by these, 305 by four waves per row.
constexpr int kJoinRows = 4, kFewSplits = 8, kManyRows = 16384;
template <int DT, int HD> __global__ __launch_bounds__(kJoinThreads) void tree_join_few(TreeArgs a, int groups) {
  constexpr int LANES = HD / 4, STEP = kJoinThreads / LANES;
  const int u = blockIdx.x / groups, row0 = blockIdx.x % groups * (STEP * kJoinRows);
  const int request = u / a.heads, all = a.nodes * a.group;
  const int nodes = a.n_nodes != nullptr ? min(max(a.n_nodes[request], 0), a.nodes) : a.nodes;
  const int rows = nodes * a.group;
  const int splits = tree::splits_used(min(max(a.n_used[u], 0), tree::budget_of(a.pages, a.B, request)), a.chunk);
  if (row0 >= rows || splits == 1) return;  // (the only split has written its rows)
  const int sub = threadIdx.x % LANES, col = sub * 4;
  int row[kJoinRows];
  size_t first[kJoinRows];
  float m[kJoinRows], l[kJoinRows], M[kJoinRows], sum[kJoinRows];
  tree::f32x4 o[kJoinRows];
#pragma unroll
  for (int r = 0; r < kJoinRows; ++r) {
    row[r] = row0 + r * STEP + static_cast<int>(threadIdx.x) / LANES;
    first[r] = static_cast<size_t>(u) * a.splits * all + min(row[r], rows - 1);
    const size_t at = first[r] + static_cast<size_t>(min(sub, splits - 1)) * all;
    m[r] = a.part_m[at];
    l[r] = a.part_l[at];
    o[r] = tree::f32x4{0};
  }
#pragma unroll 1
  for (int i = 0; i < splits; i += 2) {
    tree::f32x4 v[2][kJoinRows];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int r = 0; r < kJoinRows; ++r) v[k][r] = *reinterpret_cast<const tree::f32x4*>(a.part_o + (first[r] + static_cast<size_t>(min(i + k, splits - 1)) * all) * HD + col);
    if (i == 0) {
#pragma unroll
      for (int r = 0; r < kJoinRows; ++r) {
        M[r] = -INFINITY;
#pragma unroll
        for (int k = 0; k < kFewSplits; ++k) M[r] = fmaxf(M[r], __shfl(m[r], k, LANES));  // (lanes behind the last split have the last one's)
        m[r] = m[r] > -INFINITY ? fast_exp2(m[r] - M[r]) : 1.0f;  // a split's weight (one of no maximum has a sum of zero, or NaN)
        sum[r] = 0.0f;
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int r = 0; r < kJoinRows; ++r) {
        const float w = __shfl(m[r], i + k, LANES), s = __shfl(l[r], i + k, LANES);
        if (i + k >= splits) continue;
        o[r] += v[k][r] * w;
        sum[r] += s * w;
      }
  }
#pragma unroll
  for (int r = 0; r < kJoinRows; ++r) {
    if (row[r] >= rows) continue;
    const size_t at = static_cast<size_t>(u) * all + row[r];
    tree::store4<DT>(a.out, at * HD + col, o[r] * (1.0f / sum[r]));
    if (a.lse != nullptr && sub == 0) a.lse[at] = 0.6931471805599453f * (M[r] + __log2f(sum[r]));
  }
}

template <int DT, int HD, int WAVES> hipError_t launch_join_waves(const TreeArgs& a, hipStream_t s) {
  constexpr int kRows = kJoinThreads / kWave / WAVES;
  const long long rows = static_cast<long long>(a.units) * a.nodes * a.group;
  hipLaunchKernelGGL((tree_join<DT, HD, WAVES>), dim3(static_cast<unsigned>((rows + kRows - 1) / kRows)), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}
// A wave per row, or four where the splits are many: then the rows are few.
template <int DT, int HD> hipError_t launch_join(const TreeArgs& a, hipStream_t s) {
  ProfScope ps(kProfTreeJoin, s);
  if (a.splits > kFewSplits) return launch_join_waves<DT, HD, 4>(a, s);
  if (static_cast<long long>(a.units) * a.nodes * a.group < kManyRows) return launch_join_waves<DT, HD, 1>(a, s);
  constexpr int kRows = kJoinThreads / (HD / 4) * kJoinRows;
  const int groups = (a.nodes * a.group + kRows - 1) / kRows;
  hipLaunchKernelGGL((tree_join_few<DT, HD>), dim3(static_cast<unsigned>(a.units) * groups), dim3(kJoinThreads), 0, s, a, groups);
  return hipGetLastError();
}

}  // namespace

// Query rows of a workgroup: 64, or of bf16 192 (128 with a recency window, whose code has no registers for the third tile of a wave).
int tree_attend_row_tiles(int dtype, int rows, bool window) {
  const int most = dtype != kBF16 || rows <= 64 ? 64 : window ? 128 : 192;
  return (rows + most - 1) / most;
}

// Two workgroups on every compute unit, while each has 64 slots.  With more than 64 rows of bf16, where a workgroup's products bound it and not the
// memory: the splits, of 192 slots at least, whose rounds of 512 workgroups are shortest, a workgroup being as long as its tiles of 32 and 8
// more for its start and its share of the outputs (128 units x 4096 slots x 512 rows: four splits 273 us, two 271, three 288; with requests of
// different lengths, which fewer splits leave waiting for the longest, 194, 205 and 206; 192 units x 2048 x 160 rows: two splits 98 us, three 115,
// one 117; 512 x 4096 x 384 rows: one 673, two 729; 32 x 8192 x 128 rows: the rule's sixteen 57, six 71).
TreeSplits tree_attend_splits(int dtype, int units, int rows, int B, bool window) {
  const char* const asked = getenv("ROCO_TREE_SPLITS");
  int want = asked != nullptr ? atoi(asked) : 0;
  const long long groups = static_cast<long long>(units) * tree_attend_row_tiles(dtype, rows, window);
  if (want <= 0) {
    want = static_cast<int>((512 + groups - 1) / groups);
    if (dtype == kBF16 && rows > 64) {
      long long least = -1;
      for (int splits = 1; splits <= std::max(1, std::min(kMaxTreeSplits, B / 192)); ++splits) {
        const long long cost = (groups * splits + 511) / 512 * ((B + splits - 1) / splits + 8 * 32);
        if (least < 0 || cost < least) {
          least = cost;
          want = splits;
        }
      }
    }
  }
  // (what a launch of the attention takes, and of the joining with a workgroup per row)
  want = std::min<long long>(want, (kMostWorkgroups - 1) / (groups + 7ll * tree_attend_row_tiles(dtype, rows, window)));
  if (static_cast<long long>(units) * rows >= kMostWorkgroups) want = std::min(want, kFewSplits);
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
