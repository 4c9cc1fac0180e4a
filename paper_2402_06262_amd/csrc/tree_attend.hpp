// Attention of drafted trees over the budgeted cache: out = softmax(scale q . [K of the cache; k of the nodes seen]) [V; v], and
// ln of the softmax's sum, without a change to the cache.
//
// One pass over K and V with a running maximum and sum.  A wave streams tiles of 8 KiB of either through LDS of its own, two of each,
// filled by loads that go straight there and ordered by the wave's own load counter: no barrier, and three operand tiles of a wave on
// their way at any time.  Scores = K . Q^T on the matrix cores, so that a lane holds four slots of one query; the outputs' products
// O^T = V^T . P^T take these registers as they are.  A tree's nodes are tiles of the last split like any others, but for their mask.
// The running maximum follows a tile's only when that is more than 2^8 above it: no rescaling, and no exchange between lanes, for most
// tiles, and the sums stay far from the ends of fp32.
// Up to 64 rows the memory bounds it: 512 units x 2048 slots of bf16 / 128 with 16 rows 84 us, 6.5 TB/s of K and V; 16 x 65536 with 64 rows 102 us with the
// joining of their splits, 5.3.
// fp32's matrix instructions share that place from 17 rows on: 60 x 1501 slots of 128 with 21 rows (32 are formed) 30 us for 92 MB.
#pragma once
#include <type_traits>

#include "tree.hpp"
#include "profile.hpp"

namespace roco {
namespace tree {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

constexpr int kAttendWaves = 2;
constexpr int kAttendThreads = kAttendWaves * kWave;
constexpr float kSlack = 8.0f;  // base-2 logits that a tile may lie above the running maximum
constexpr float kLn2 = 0.6931471805599453f;

// Whether 16 bytes of values hold an infinite one or NaN.
template <int DT> __device__ __forceinline__ bool holds_special(const uint4& v) {
  // (the exponent's bits set: adding one to them carries)
  const auto one = [](uint32_t x) {
    if (DT == kBF16) return ((x & 0x7f800000u) + 0x00800000u) | (((x & 0x7f80u) + 0x80u) << 16);
    return (x & 0x7f800000u) + 0x00800000u;
  };
  return ((one(v.x) | one(v.y) | one(v.z) | one(v.w)) & 0x80000000u) != 0;
}
// What is derived from these is computed where it is used, not kept in registers through the loop: for what only some tiles need.
struct LateLane {
  int lane, qi, g;
  __device__ __forceinline__ LateLane() : lane(late_thread_id() & (kWave - 1)), qi(lane & 15), g(lane >> 4) {}
};
__device__ __forceinline__ int late(int v) {
  asm volatile("" : "+s"(v));
  return v;
}

template <int DT> __device__ __forceinline__ float load_elem(const void* base, size_t idx) {
  if constexpr (DT == kBF16) return bf16_to_f32(static_cast<const uint16_t*>(base)[idx]);
  else return static_cast<const float*>(base)[idx];
}

// The nodes whose values are not finite, added to the rows that see them: `count` rows from `first` on, which the wave has written without
// them, a row at a time, HD / 64 of its elements per lane.  max_s, scale_s: the rows' maxima, and what they were multiplied by.  (Final rows
// of bf16 are rounded twice where they see such a node.)
template <int DT, int HD, bool WINDOW>
__device__ __forceinline__ void add_special_nodes(const TreeArgs& a, int u, size_t out_row, size_t part_row, int first, int count, int used, uint64_t seen,
                                                  uint64_t special, const float* max_s, const float* scale_s) {
  constexpr int E = HD / kWave;
  __threadfence_block();
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll 1
  for (int q = 0; q < count; ++q) {
    const uint64_t sees = from_lane(seen, (first + q) / a.group);
    if ((sees & special) == 0) continue;
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = used == 1 ? load_elem<DT>(a.out, (out_row + q) * HD + lane * E + e) : a.part_o[(part_row + q) * HD + lane * E + e];
#pragma unroll 1
    for (uint64_t left = sees & special; left != 0; left &= left - 1) {
      const int j = __builtin_ctzll(left);
      const size_t node = (static_cast<size_t>(u) * a.nodes + j) * HD + lane * E;
      float dot = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) dot = fmaf(load_elem<DT>(a.q, (out_row + q) * HD + lane * E + e), load_elem<DT>(a.k_new, node + e), dot);
      float x = group_sum<kWave>(dot) * a.scale_log2;
      if (WINDOW && __builtin_popcountll(sees) - __builtin_popcountll(from_lane(seen, j)) < a.recency_window) x += a.recency_bias_log2;
      const float p = fast_exp2(x - (max_s[q] > -INFINITY ? max_s[q] : 0.0f)) * scale_s[q];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = fmaf(p, load_elem<DT>(a.v_new, node + e), v[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (used == 1) store_elem<DT>(a.out, (out_row + q) * HD + lane * E + e, v[e]);
      else a.part_o[(part_row + q) * HD + lane * E + e] = v[e];
    }
  }
}

// NQ tiles of 16 query rows; a row is a node and a head of the group.  WINDOW: a recency bias is in force.
// A launch begins with a cold instruction cache, a third of a microsecond per KiB, so that nothing is unrolled that need not be, and what is
// rare loops over rows.
// One wave on a SIMD (the registers are filled up to that): the two workgroups that LDS lets on a compute unit otherwise share two of its SIMDs,
// and leave two idle (512 units x 2048 slots of bf16 92.2 us against 84.4, 60 units x 1501 of fp32 with 21 rows 40.5 / 31.1).
template <int DT, int HD, int NQ, bool STREAMING, bool WINDOW>
__global__ __launch_bounds__(kAttendThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void tree_attend(TreeArgs a) {
  using T = Tile<DT, HD>;
  constexpr int W = kAttendWaves, G = T::kGroups, QR = 16 * NQ;
  constexpr int kTileBytes = 8192, kWaveBytes = 4 * kTileBytes;  // K, V, K, V
  constexpr int kAhead = 2;
  constexpr int kSide = WINDOW ? 1 : 0;                          // the positions of a K tile's slots come along
  // the queries come through the place of the second V tile, or of the second tiles, or before any tile
  constexpr int kQueryBytes = QR * T::kBytes;
  constexpr bool kBehindK = kQueryBytes <= kTileBytes, kBeforeK = !kBehindK && kQueryBytes <= 2 * kTileBytes;
  extern __shared__ __attribute__((aligned(1024))) char lds[];   // the waves' tiles; then a wave's outputs
  __shared__ __attribute__((aligned(256))) int32_t pos_s[WINDOW ? W : 1][2][kWave];
  __shared__ float merge_m[QR], merge_l[QR];
  __shared__ uint64_t special_s[W];
  // the row tiles of a split go to one die: eight dies take the workgroups in turn
  const int per = 8 * a.row_tiles, id = blockIdx.x;
  const int us = id / per * 8 + id % 8, row_tile = id % per / 8;
  if (us >= a.units * a.splits) return;
  const int u = us % a.units, split = us / a.units;  // (the later splits, which not every unit needs, come last and to all dies)
  const int request = u / a.heads;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int qi = lane & 15, g = lane >> 4;
  // (what has to come from memory before anything else is asked for together)
  int parent = lane - 1;
  if (a.parent != nullptr) parent = a.parent[static_cast<size_t>(request) * a.nodes + min(lane, a.nodes - 1)];
  const int asked_nodes = a.n_nodes != nullptr ? a.n_nodes[request] : a.nodes, held = a.n_used[u], budget = budget_of(a.pages, a.B, request);
  const int nodes = __builtin_amdgcn_readfirstlane(min(max(asked_nodes, 0), a.nodes));
  const int n = __builtin_amdgcn_readfirstlane(min(max(held, 0), budget));
  const int rows = nodes * a.group, first_row = row_tile * QR;
  const int used = splits_used(n, a.chunk);  // the last of them takes the nodes too
  if (first_row >= rows || split >= used) return;
  const int row0 = split * a.chunk, row1 = min(n, row0 + a.chunk);
  Walk<DT, HD, W> walk;
  walk.init(a.pages, a.B, a.heads, u, request, row0, row1, split == used - 1 ? nodes : 0, wave, static_cast<unsigned>(u) * 5u + static_cast<unsigned>(split) * 3u);
  const int mine = walk.mine;

  char* const tiles = lds + wave * kWaveBytes;
  const uint32_t tiles_addr = lds_address(tiles), pos_addr = lds_address(&pos_s[WINDOW ? wave : 0][0][0]);
  int koff[T::kGroupLoads], voff[T::kGroupLoads];
  load_offsets<DT, HD, false>(koff);
  load_offsets<DT, HD, true>(voff);
  // B operand: the queries, a load's 16 rows of a tile as those of K (rows behind the last are zeros; their results are dropped)
  const size_t row_base = static_cast<size_t>(u) * a.nodes * a.group;
  const int kfrag = qi * T::kBytes + ((g ^ T::swizzle_k(qi)) << 4);
  uint4 own[NQ][T::kSteps];
  constexpr int kQueryPlace = kBehindK ? 3 * kTileBytes : kBeforeK ? 2 * kTileBytes : 0;
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {
    const int row = first_row + 16 * t2;
    const v4i32 buf = make_buffer(static_cast<const char*>(a.q) + (row_base + row) * T::kBytes, static_cast<uint32_t>(min(max(rows - row, 0), 16)) * T::kBytes);
#pragma unroll
    for (int j = 0; j < T::kGroupLoads; ++j) load16_to_lds(buf, tiles_addr + kQueryPlace + (t2 * T::kGroupLoads + j) * 1024, koff[j], 0);
  }
  auto read_queries = [&]() {
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2)
#pragma unroll
      for (int kk = 0; kk < T::kSteps; ++kk)
        own[t2][kk] = *reinterpret_cast<const uint4*>(tiles + kQueryPlace + t2 * 16 * T::kBytes + (kfrag ^ (kk << 6)));
    reads_done();
  };
  if (!kBehindK && !kBeforeK) {
    wait_loads<0>();
    read_queries();
  }

  const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f;  // (without a bias, products are multiplied by sc where they become exponents)
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[u] : 0;
  const auto token_of = [&](int t2, int q) { return min(first_row + 16 * t2 + q, rows - 1) / late(a.group); };
  const auto see = [&]() { return seen_nodes(parent, nodes, LateLane().lane); };
  uint64_t seen = 0, special = 0;  // by node `lane`; nodes whose values are not finite
  int qp[NQ];
  if (WINDOW) {
    seen = see();
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) qp[t2] = qp0 + __shfl(__builtin_popcountll(seen), token_of(t2, qi), kWave) - 1;
  }
  float m[NQ], l[NQ];
  f32x4 o[NQ][T::kBlocks];
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {
    m[t2] = -INFINITY;
    l[t2] = 0.0f;
#pragma unroll
    for (int db = 0; db < T::kBlocks; ++db) o[t2][db] = f32x4{0};
  }
  const v4i32 pbuf = make_buffer(a.pos + static_cast<size_t>(u) * a.B, WINDOW ? static_cast<uint32_t>(a.B) * 4u : 0u);
  const size_t new_rows = static_cast<size_t>(u) * a.nodes * T::kBytes;
  // bf16: V^T of dimensions 0..15, rows 4 g + lane / 4 % 4, 8 bytes from column 4 (lane % 4) on; fp32: row 4 g, column lane % 16
  const int vrow = DT == kBF16 ? 4 * g + (qi >> 2) : 4 * g;
  const int vfrag = vrow * T::kBytes + (T::swizzle_v(vrow) << 4) + (DT == kBF16 ? (qi & 3) * 8 : qi * 4);

  typedef typename Walk<DT, HD, W>::Place Place;
  const auto request_k = [&](const Place& p, bool of_nodes, int t) {
    request_tile<DT, HD, STREAMING>(of_nodes ? static_cast<const char*>(a.k_new) + new_rows : static_cast<const char*>(a.K), p.row, p.there, tiles_addr + (t & 1) * 2 * kTileBytes, koff);
    // (a wave-wide load of 64 words, whatever the tile; behind the unit's last slot, and for nodes, zeros)
    if (WINDOW) mfma::load4_to_lds(pbuf, pos_addr + (t & 1) * (kWave * 4), of_nodes ? 0x7ffffffc : (walk.first_slot(t) + lane) * 4, 0);
  };
  const auto request_v = [&](const Place& p, bool of_nodes, int t) {
    request_tile<DT, HD, STREAMING>(of_nodes ? static_cast<const char*>(a.v_new) + new_rows : static_cast<const char*>(a.V), p.row, p.there, tiles_addr + (t & 1) * 2 * kTileBytes + kTileBytes, voff);
  };
  Place second;
  bool second_nodes = false;
  uint32_t there0 = 0, there1 = 0, there2 = 0;  // of this tile and the two behind it
  // (the first requests are not a part of the loop over the tiles, though that is code again: with the queries read inside it their registers were copied
  // on its way round, 120 instructions per tile of fp32 / 128, and 32 rows took 43 us where they take 34)
#pragma unroll 1
  for (int t = 0; t < 2; ++t) {
    if (kBeforeK && t == 1) {
      if (mine > 0) wait_loads<2 * T::kLoads + kSide>();
      else wait_loads<0>();
      read_queries();
    }
    if (t < mine) {
      const Place next = walk.place(t);
      const bool next_nodes = walk.is_nodes(t);
      if (t == 0) there0 = next.there;
      else there1 = next.there;
      request_k(next, next_nodes, t);
      if (!kBehindK || t == 0) request_v(next, next_nodes, t);
      else second = next, second_nodes = next_nodes;
    }
  }
  if (kBehindK) {
    if (mine > 1) wait_loads<3 * T::kLoads + 2 * kSide>();
    else if (mine > 0) wait_loads<2 * T::kLoads + kSide>();
    else wait_loads<0>();
    read_queries();
    if (mine > 1) request_v(second, second_nodes, 1);
  }
#pragma unroll 1
  for (int t = 0; t < mine; ++t) {
    char* const tileK = tiles + (t & 1) * 2 * kTileBytes;
    char* const tileV = tileK + kTileBytes;
    f32x4 s[NQ][G];
    int ps[G][4];
    // K(t) has landed; V(t), and K and V of the next tile, may still be on their way
    if (t + 1 < mine) wait_loads<3 * T::kLoads + kSide>();
    else wait_loads<T::kLoads>();
    // (fragments are read kAhead steps ahead: left to itself the compiler reads each one right before its use, and waits for it)
    uint4 kf[kAhead + 1][G];
    const auto read_k = [&](int kk) {
#pragma unroll
      for (int i = 0; i < G; ++i) kf[kk % (kAhead + 1)][i] = *reinterpret_cast<const uint4*>(tileK + i * 16 * T::kBytes + (kfrag ^ (kk << 6)));
    };
#pragma unroll
    for (int kk = 0; kk < kAhead; ++kk) read_k(kk);
#pragma unroll
    for (int kk = 0; kk < T::kSteps; ++kk) {
      if (kk + kAhead < T::kSteps) read_k(kk + kAhead);
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int t2 = 0; t2 < NQ; ++t2) s[t2][i] = score_step<DT>(kf[kk % (kAhead + 1)][i], own[t2][kk], kk == 0 ? f32x4{0} : s[t2][i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (WINDOW) {
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const int4 p4 = *reinterpret_cast<const int4*>(&pos_s[WINDOW ? wave : 0][t & 1][16 * i + 4 * g]);
        ps[i][0] = p4.x; ps[i][1] = p4.y; ps[i][2] = p4.z; ps[i][3] = p4.w;
      }
    }
    reads_done();
    Place next;
    bool next_nodes = false;
    if (t + 2 < mine) {
      next = walk.place(t + 2);
      there2 = next.there;
      next_nodes = walk.is_nodes(t + 2);
      request_k(next, next_nodes, t + 2);
    }
    const bool of_nodes = walk.is_nodes(t);
    constexpr uint32_t kWhole = G == 1 ? 0x10u : G == 2 ? 0x1010u : 0x10101010u;
    if (of_nodes) {
      if (!WINDOW) seen = see();
      const int j0 = walk.first_node(t);
      const LateLane L;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        if (WINDOW) {
#pragma unroll
          for (int e = 0; e < 4; ++e) ps[i][e] = qp0 + __shfl(__builtin_popcountll(seen), min(j0 + 16 * i + 4 * L.g + e, kWave - 1), kWave) - 1;
        }
      }
#pragma unroll
      for (int t2 = 0; t2 < NQ; ++t2) {
        const uint64_t sees = from_lane(seen, token_of(t2, L.qi)) >> (j0 + 4 * L.g);
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t2][i][e] = (sees >> (16 * i + e)) & 1 ? s[t2][i][e] : -INFINITY;
      }
    } else if (there0 != kWhole) {
      const LateLane L;
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool visible = 4 * L.g + e < static_cast<int>((there0 >> (8 * i)) & 0xffu);
#pragma unroll
          for (int t2 = 0; t2 < NQ; ++t2) s[t2][i][e] = visible ? s[t2][i][e] : -INFINITY;
        }
    }
    // ---- probabilities; what a row does not see is -inf
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) {
      float most = -INFINITY;
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (WINDOW) {
            const int away = qp[t2] - ps[i][e];
            s[t2][i][e] = fmaf(s[t2][i][e], sc, static_cast<unsigned>(away) < static_cast<unsigned>(w) ? bias : 0.0f);
          }
          most = fmaxf(most, s[t2][i][e]);
        }
      if (!WINDOW) most *= sc;
      if (__any(most > m[t2] + kSlack)) {
        most = fmaxf(most, __shfl_xor(most, 16, kWave));
        most = fmaxf(most, __shfl_xor(most, 32, kWave));
        const float m_new = most > m[t2] + kSlack ? most : m[t2];  // (a row's bits do not depend on the rows beside it)
        const float alpha = m[t2] > -INFINITY ? fast_exp2(m[t2] - m_new) : 0.0f;
        l[t2] *= alpha;
#pragma unroll
        for (int db = 0; db < T::kBlocks; ++db) o[t2][db] *= alpha;
        m[t2] = m_new;
      }
      const float ref = m[t2] > -INFINITY ? m[t2] : 0.0f;  // nothing seen yet: every term is 2^-inf = 0
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[t2][i][e] = fast_exp2(WINDOW ? s[t2][i][e] - ref : fmaf(s[t2][i][e], sc, -ref));
          sum += s[t2][i][e];
        }
      l[t2] += sum;
    }
    // ---- O^T += V^T . P^T
    if (t + 2 < mine) wait_loads<3 * T::kLoads + 2 * kSide>();
    else if (t + 1 < mine) wait_loads<2 * T::kLoads + kSide>();
    else wait_loads<0>();
    if (of_nodes) {
      // A node's value that is infinite or NaN must not reach the rows that do not see the node, and 0 times it would: such nodes
      // are zero in the products, and added in the end to the rows that see them.
      bool any = false;
      const LateLane L;
#pragma unroll
      for (int i = 0; i < 8; ++i) any |= holds_special<DT>(*reinterpret_cast<const uint4*>(tileV + i * 1024 + L.lane * 16));
      if (__any(any)) {
        const int j0 = walk.first_node(t);
#pragma unroll 1
        for (int j = 0; j < min(T::kSlots, nodes - j0); ++j) {
          uint4* const row = reinterpret_cast<uint4*>(tileV + j * T::kBytes) + L.lane % T::kChunks;
          if (!__any(holds_special<DT>(*row))) continue;
          special |= 1ull << (j0 + j);
          *row = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      reads_done();
    }
    if constexpr (DT == kBF16) {
      // The probabilities as sums of two bf16 numbers: rounded to one they would make as much of the output's error as its own
      // rounding (2.3e-3 against 1.7e-3 of its norm); the matrix cores have the time.
      uint4 vf[kAhead + 1];
      const auto read_v = [&](int at) {
        const char* const vt = tileV + at / T::kBlocks * 2 * 16 * T::kBytes + (vfrag ^ (at % T::kBlocks << 5));
        const uint2 lo = lds_read_transposed(vt), hi = lds_read_transposed(vt + 16 * T::kBytes);
        vf[at % (kAhead + 1)] = make_uint4(lo.x, lo.y, hi.x, hi.y);
      };
#pragma unroll
      for (int at = 0; at < kAhead; ++at) read_v(at);
#pragma unroll
      for (int i = 0; i < G; i += 2) {
        uint4 p[NQ][2];
#pragma unroll
        for (int t2 = 0; t2 < NQ; ++t2) {
          const f32x4 pair[2] = {s[t2][i], s[t2][i + 1]};
          fused::split_positive(pair, p[t2]);
        }
#pragma unroll
        for (int db = 0; db < T::kBlocks; ++db) {
          const int at = i / 2 * T::kBlocks + db;
          if (at + kAhead < G / 2 * T::kBlocks) read_v(at + kAhead);
          const uint4 v = vf[at % (kAhead + 1)];
#pragma unroll
          for (int k = 1; k >= 0; --k)
#pragma unroll
            for (int t2 = 0; t2 < NQ; ++t2) o[t2][db] = fused::mfma16(v, p[t2][k], o[t2][db]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
      float vf[kAhead + 1][4];
      const auto read_v = [&](int at) {
        const char* const vt = tileV + at / T::kBlocks * 16 * T::kBytes + (vfrag ^ (at % T::kBlocks << 6));
#pragma unroll
        for (int e = 0; e < 4; ++e) vf[at % (kAhead + 1)][e] = *reinterpret_cast<const float*>(vt + e * T::kBytes);
      };
#pragma unroll
      for (int at = 0; at < kAhead; ++at) read_v(at);
#pragma unroll
      for (int at = 0; at < G * T::kBlocks; ++at) {
        if (at + kAhead < G * T::kBlocks) read_v(at + kAhead);
        const int i = at / T::kBlocks, db = at % T::kBlocks;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int t2 = 0; t2 < NQ; ++t2) o[t2][db] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[at % (kAhead + 1)][e], s[t2][i][e], o[t2][db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    reads_done();
    if (t + 2 < mine) request_v(next, next_nodes, t);
    there0 = there1;
    there1 = there2;
  }
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {  // the lane groups have summed different slots
    l[t2] += __shfl_xor(l[t2], 16, kWave);
    l[t2] += __shfl_xor(l[t2], 32, kWave);
  }

  // ---- the second wave's share is added to the first one's, which writes the rows
  constexpr int kOut = HD + 4;
  __syncthreads();
  float* const outs = reinterpret_cast<float*>(lds);
  if (lane == 0) special_s[wave] = special;
  if (wave == 1) {
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) {
      const int q = 16 * t2 + qi;
      if (g == 0) { merge_m[q] = m[t2]; merge_l[q] = l[t2]; }
#pragma unroll
      for (int db = 0; db < T::kBlocks; ++db) *reinterpret_cast<f32x4*>(outs + q * kOut + 16 * db + 4 * g) = o[t2][db];
    }
  }
  __syncthreads();
  if (wave != 0) return;
  special = special_s[0] | special_s[1];
  const size_t part_base = (static_cast<size_t>(u) * a.splits + split) * a.nodes * a.group;
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {
    const int q = 16 * t2 + qi, row = first_row + q;
    const float m1 = merge_m[q], l1 = merge_l[q];
    // (a maximum is -inf where a wave has seen nothing, or nothing but logits of -inf or NaN: NaN sums stay)
    const float M = fmaxf(m[t2], m1);
    const float w0 = m[t2] > -INFINITY ? fast_exp2(m[t2] - M) : 1.0f, w1 = m1 > -INFINITY ? fast_exp2(m1 - M) : 1.0f;
    const float sum = l[t2] * w0 + l1 * w1;
    const float scale = used == 1 ? 1.0f / sum : 1.0f;
    if (g == 0 && row < rows) {
      if (used == 1) {
        if (a.lse != nullptr) a.lse[row_base + row] = kLn2 * (M + __log2f(sum));
      } else {
        a.part_m[part_base + row] = M;
        a.part_l[part_base + row] = sum;
      }
      merge_m[q] = M;
      merge_l[q] = scale;
    }
#pragma unroll
    for (int db = 0; db < T::kBlocks; ++db) {
      const f32x4 v = (o[t2][db] * w0 + *reinterpret_cast<const f32x4*>(outs + q * kOut + 16 * db + 4 * g) * w1) * scale;
      if (row < rows && used == 1) store4<DT>(a.out, (row_base + row) * HD + 16 * db + 4 * g, v);
      else if (row < rows) *reinterpret_cast<f32x4*>(a.part_o + (part_base + row) * HD + 16 * db + 4 * g) = v;
    }
  }
  if (special != 0)
    add_special_nodes<DT, HD, WINDOW>(a, u, row_base + first_row, part_base + first_row, first_row, min(QR, rows - first_row), used, see(), special, merge_m, merge_l);
}

// More than 64 query rows of bf16: four waves with 16 NQ rows each share the tiles, which come two at a time, K or V of one by each
// wave, while the two before them are used; one barrier for two tiles.  Two workgroups on a compute unit, so that one wave's exponentials run beside another's products: with 64
// rows to a workgroup and the rest in others, every row tile fetched K and V again, and a wave had its matrix cores to itself.
// Probabilities are sums of two bf16 numbers as with fewer rows, so that a tree's outputs do not lose bits to the rows beside it in a call: one number,
// half a step of 2^-8 off, takes a quarter less time (152 us for 194 on the trees below, whose outputs are then 2.3e-3 of their norm off instead of 1.7e-3,
// their own rounding).
// 512 units x 4096 slots with 384 rows 673 us, 610 TFLOP/s, 920 with the second numbers' products; 128 units of 919 to 4096 slots with 256 to 496 rows
// 194 us, 16 of them to join splits, whose products would take 49: exponentials, products and fragments' reads follow each other in a wave, and two
// waves on a SIMD cover a part of it.
constexpr int kWideWaves = 4;
constexpr int kWideThreads = kWideWaves * kWave;

template <int HD, int NQ, bool WINDOW>
__global__ __launch_bounds__(kWideThreads, 2) void tree_attend_wide(TreeArgs a) {
  constexpr int DT = kBF16;
  using T = Tile<DT, HD>;
  constexpr int W = kWideWaves, G = T::kGroups, QR = 16 * NQ;  // query rows of a wave
  constexpr int kTileBytes = 8192, kPairBytes = 2 * kTileBytes;  // a tile of K and one of V
  static_assert(W == 4, "two waves ask for K, two for V");
  extern __shared__ __attribute__((aligned(1024))) char lds[];  // four pairs of tiles: two in use, two on their way
  __shared__ __attribute__((aligned(256))) int32_t pos_s[WINDOW ? 4 : 1][kWave];
  __shared__ float max_s[W][QR], scale_s[W][QR];
  __shared__ uint32_t there_s[4];  // Place::there of the tiles
  const int per = 8 * a.row_tiles, id = blockIdx.x;
  const int us = id / per * 8 + id % 8, row_tile = id % per / 8;
  if (us >= a.units * a.splits) return;
  const int u = us % a.units, split = us / a.units;  // (the later splits, which not every unit needs, come last and to all dies)
  const int request = u / a.heads;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int qi = lane & 15, g = lane >> 4;
  const int asked_nodes = a.n_nodes != nullptr ? a.n_nodes[request] : a.nodes, held = a.n_used[u], budget = budget_of(a.pages, a.B, request);
  const int nodes = __builtin_amdgcn_readfirstlane(min(max(asked_nodes, 0), a.nodes));
  const int n = __builtin_amdgcn_readfirstlane(min(max(held, 0), budget));
  const int rows = nodes * a.group, first_row = row_tile * W * QR + wave * QR;
  const int used = splits_used(n, a.chunk);
  if (row_tile * W * QR >= rows || split >= used) return;
  const int row0 = split * a.chunk, row1 = min(n, row0 + a.chunk);
  Walk<DT, HD, 1, kTileBytes, 2> walk;
  walk.init(a.pages, a.B, a.heads, u, request, row0, row1, split == used - 1 ? nodes : 0, 0, static_cast<unsigned>(u) * 5u + static_cast<unsigned>(split) * 3u);
  const int tiles = walk.mine;
  if ((wave >> 1) < tiles) walk.look_ahead(wave >> 1);

  int koff[T::kGroupLoads];
  load_offsets<DT, HD, false>(koff);
  const size_t row_base = static_cast<size_t>(u) * a.nodes * a.group;
  const int kfrag = qi * T::kBytes + ((g ^ T::swizzle_k(qi)) << 4);
  // the wave's queries come through a pair's place, before any tile
  uint4 own[NQ][T::kSteps];
  {
    static_assert(QR * T::kBytes <= kPairBytes, "a pair's place");
    char* const place = lds + wave * kPairBytes;
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) {
      const int row = first_row + 16 * t2;
      const v4i32 buf = make_buffer(static_cast<const char*>(a.q) + (row_base + min(row, rows - 1)) * T::kBytes, static_cast<uint32_t>(min(max(rows - row, 0), 16)) * T::kBytes);
#pragma unroll
      for (int j = 0; j < T::kGroupLoads; ++j) load16_to_lds(buf, lds_address(place) + (t2 * T::kGroupLoads + j) * 1024, koff[j], 0);
    }
    wait_loads<0>();
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2)
#pragma unroll
      for (int kk = 0; kk < T::kSteps; ++kk) own[t2][kk] = *reinterpret_cast<const uint4*>(place + t2 * 16 * T::kBytes + (kfrag ^ (kk << 6)));
    reads_done();
    __syncthreads();
  }
  const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f;
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[u] : 0;
  const auto token_of = [&](int t2, int q) { return min(first_row + 16 * t2 + q, rows - 1) / late(a.group); };
  uint64_t seen = 0, special = 0;
  const auto see = [&]() {
    const int node = LateLane().lane;
    return seen_nodes(a.parent != nullptr ? a.parent[static_cast<size_t>(request) * a.nodes + min(node, a.nodes - 1)] : node - 1, nodes, node);
  };
  int qp[NQ];
  if (WINDOW) {
    seen = see();
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) qp[t2] = qp0 + __shfl(__builtin_popcountll(seen), token_of(t2, qi), kWave) - 1;
  }
  float m[NQ], l[NQ];
  f32x4 o[NQ][T::kBlocks];
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {
    m[t2] = -INFINITY;
    l[t2] = 0.0f;
#pragma unroll
    for (int db = 0; db < T::kBlocks; ++db) o[t2][db] = f32x4{0};
  }
  const v4i32 pbuf = make_buffer(a.pos + static_cast<size_t>(u) * a.B, WINDOW ? static_cast<uint32_t>(a.B) * 4u : 0u);
  const uint32_t pos_addr = lds_address(&pos_s[0][0]), ring_addr = lds_address(lds);
  const size_t new_rows = static_cast<size_t>(u) * a.nodes * T::kBytes;

  // K (even waves) or V of a tile
  const auto request_operand = [&](auto of_v, const typename Walk<DT, HD, 1, kTileBytes, 2>::Place& next, bool of_nodes, const void* cache, const void* fresh, uint32_t dst) {
    constexpr bool kOfV = decltype(of_v)::value;
    const int lane2 = LateLane().lane;
    int off[T::kGroupLoads];
#pragma unroll
    for (int j = 0; j < T::kGroupLoads; ++j) {
      const int r = T::kPerLoad * j + lane2 / T::kChunks, c = lane2 % T::kChunks;
      off[j] = r * T::kBytes + ((c ^ (kOfV ? T::swizzle_v(r) : T::swizzle_k(r))) << 4);
    }
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const size_t at = (of_nodes ? new_rows : 0) + static_cast<size_t>(next.row[i]) * T::kBytes;
      const v4i32 buf = make_buffer(static_cast<const char*>(of_nodes ? fresh : cache) + at, ((next.there >> (8 * i)) & 0xffu) * T::kBytes);
#pragma unroll
      for (int j = 0; j < T::kGroupLoads; ++j) load16_to_lds(buf, dst + (i * T::kGroupLoads + j) * 1024, off[j], 0);
    }
  };
#pragma unroll 1
  for (int t0 = -2; t0 < tiles; t0 += 2) {
    if (t0 >= 0) {  // these tiles have landed, and nobody reads those before them any more
      wait_loads<0>();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    if (const int t = t0 + 2 + (wave >> 1); t < tiles) {
      const typename Walk<DT, HD, 1, kTileBytes, 2>::Place next = walk.place(t);
      const bool next_nodes = walk.is_nodes(t);
      const uint32_t pair = ring_addr + static_cast<uint32_t>(t & 3) * kPairBytes;
      if (wave & 1) {
        request_operand(std::true_type(), next, next_nodes, a.V, a.v_new, pair + kTileBytes);
      } else {
        request_operand(std::false_type(), next, next_nodes, a.K, a.k_new, pair);
        if (WINDOW) mfma::load4_to_lds(pbuf, pos_addr + (t & 3) * (kWave * 4), next_nodes ? 0x7ffffffc : (walk.first_slot(t) + lane) * 4, 0);
        if (LateLane().lane == 0) there_s[t & 3] = next.there;
      }
    }
#pragma unroll 1
    for (int sub = 0; sub < 2; ++sub) {
      const int t = t0 + sub;
      if (t < 0 || t >= tiles) break;
      if (first_row >= rows && !walk.is_nodes(t)) continue;  // no rows of this wave's (a tile of nodes may have everybody wait)
      char* const tileV = lds + (t & 3) * kPairBytes + kTileBytes;
      // (the tiles lie at multiples of 1 KiB: the chunk's exclusive or can be taken of the address)
      const LateLane F;
      const int vrow = 4 * F.g + (F.qi >> 2);
      const uint32_t pair = ring_addr + static_cast<uint32_t>(t & 3) * kPairBytes;
      const uint32_t k_at = pair + F.qi * T::kBytes + ((F.g ^ T::swizzle_k(F.qi)) << 4);
      const uint32_t v_at = pair + kTileBytes + vrow * T::kBytes + (T::swizzle_v(vrow) << 4) + (F.qi & 3) * 8;
      // (fragments are read a step ahead and no further: the scheduler would take all registers for them, and more)
      f32x4 s[NQ][G];
      uint4 kf[2][G];
      const auto read_k = [&](int kk) {
#pragma unroll
        for (int i = 0; i < G; ++i) kf[kk & 1][i] = lds_read16((k_at ^ (kk << 6)) + i * 16 * T::kBytes);
      };
      read_k(0);
#pragma unroll
      for (int kk = 0; kk < T::kSteps; ++kk) {
        if (kk + 1 < T::kSteps) read_k(kk + 1);
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int t2 = 0; t2 < NQ; ++t2) s[t2][i] = score_step<DT>(kf[kk & 1][i], own[t2][kk], kk == 0 ? f32x4{0} : s[t2][i]);
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool of_nodes = walk.is_nodes(t);
      constexpr uint32_t kWhole = G == 1 ? 0x10u : G == 2 ? 0x1010u : 0x10101010u;
      const uint32_t here = __builtin_amdgcn_readfirstlane(there_s[t & 3]);
      if (WINDOW) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const int4 p4 = *reinterpret_cast<const int4*>(&pos_s[WINDOW ? t & 3 : 0][16 * i + 4 * g]);
          int ps[4] = {p4.x, p4.y, p4.z, p4.w};
          if (of_nodes) {
#pragma unroll
            for (int e = 0; e < 4; ++e) ps[e] = qp0 - 1 + __shfl(__builtin_popcountll(seen), min(walk.first_node(t) + 16 * i + 4 * g + e, kWave - 1), kWave);
          }
#pragma unroll
          for (int t2 = 0; t2 < NQ; ++t2)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t2][i][e] = fmaf(s[t2][i][e], sc, static_cast<unsigned>(qp[t2] - ps[e]) < static_cast<unsigned>(w) ? bias : 0.0f);
        }
      }
      if (of_nodes || here != kWhole) {
        const LateLane L;
        const int j0 = walk.first_node(t);
        if (of_nodes && !WINDOW) seen = see();
        uint64_t there4 = 0;  // bit 16 i + e: slot 4 g + e of group i is there
#pragma unroll
        for (int i = 0; i < G; ++i) there4 |= static_cast<uint64_t>(0xffffu >> (16 - ((here >> (8 * i)) & 0xffu))) << (16 * i);
        there4 >>= 4 * L.g;
#pragma unroll
        for (int t2 = 0; t2 < NQ; ++t2) {
          uint64_t visible = there4;
          if (of_nodes) visible &= from_lane(seen, token_of(t2, L.qi)) >> (j0 + 4 * L.g);
#pragma unroll
          for (int i = 0; i < G; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t2][i][e] = (visible >> (16 * i + e)) & 1 ? s[t2][i][e] : -INFINITY;
        }
        if (of_nodes) {  // (see tree_attend; the rows are everybody's)
          bool any = false;
#pragma unroll
          for (int i = 0; i < 8; ++i) any |= holds_special<DT>(*reinterpret_cast<const uint4*>(tileV + i * 1024 + L.lane * 16));
          if (__any(any)) {
#pragma unroll 1
            for (int j = 0; j < min(T::kSlots, nodes - j0); ++j)
              if (__any(holds_special<DT>(*(reinterpret_cast<const uint4*>(tileV + j * T::kBytes) + L.lane % T::kChunks)))) special |= 1ull << (j0 + j);
            __syncthreads();
            if (wave == 0) {
#pragma unroll 1
              for (int j = 0; j < min(T::kSlots, nodes - j0); ++j)
                if ((special >> (j0 + j)) & 1) reinterpret_cast<uint4*>(tileV + j * T::kBytes)[L.lane % T::kChunks] = make_uint4(0u, 0u, 0u, 0u);
            }
            __syncthreads();
          }
        }
      }
#pragma unroll
      for (int t2 = 0; t2 < NQ; ++t2) {
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) most = fmaxf(most, s[t2][i][e]);
        if (!WINDOW) most *= sc;
        if (__any(most > m[t2] + kSlack)) {
          most = fmaxf(most, __shfl_xor(most, 16, kWave));
          most = fmaxf(most, __shfl_xor(most, 32, kWave));
          const float m_new = most > m[t2] + kSlack ? most : m[t2];
          const float alpha = m[t2] > -INFINITY ? fast_exp2(m[t2] - m_new) : 0.0f;
          l[t2] *= alpha;
#pragma unroll
          for (int db = 0; db < T::kBlocks; ++db) o[t2][db] *= alpha;
          m[t2] = m_new;
        }
        const float ref = m[t2] > -INFINITY ? m[t2] : 0.0f;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[t2][i][e] = fast_exp2(WINDOW ? s[t2][i][e] - ref : fmaf(s[t2][i][e], sc, -ref));
            sum += s[t2][i][e];
          }
        l[t2] += sum;
      }
#pragma unroll
      for (int i = 0; i < G; i += 2) {
        uint4 p[NQ][2];
#pragma unroll
        for (int t2 = 0; t2 < NQ; ++t2) {
          const f32x4 pair[2] = {s[t2][i], s[t2][i + 1]};
          fused::split_positive(pair, p[t2]);
        }
        uint4 vf[2];
        const auto read_v = [&](int db) {
          const uint32_t vt = (v_at ^ (db << 5)) + i * 16 * T::kBytes;
          const uint2 lo = lds_read_transposed_at(vt), hi = lds_read_transposed_at(vt + 16 * T::kBytes);
          vf[db & 1] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        };
        read_v(0);
#pragma unroll
        for (int db = 0; db < T::kBlocks; ++db) {
          if (db + 1 < T::kBlocks) read_v(db + 1);
#pragma unroll
          for (int k = 1; k >= 0; --k)
#pragma unroll
            for (int t2 = 0; t2 < NQ; ++t2) o[t2][db] = fused::mfma16(vf[db & 1], p[t2][k], o[t2][db]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  const LateLane L;
  const size_t part_base = (static_cast<size_t>(u) * a.splits + split) * a.nodes * a.group;
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {
    const int row = first_row + 16 * t2 + L.qi;
    float sum = l[t2];
    sum += __shfl_xor(sum, 16, kWave);
    sum += __shfl_xor(sum, 32, kWave);
    const float scale = used == 1 ? 1.0f / sum : 1.0f;
    if (L.g == 0) {
      if (row < rows) {
        if (used == 1) {
          if (a.lse != nullptr) a.lse[row_base + row] = kLn2 * (m[t2] + __log2f(sum));
        } else {
          a.part_m[part_base + row] = m[t2];
          a.part_l[part_base + row] = sum;
        }
      }
      max_s[wave][16 * t2 + L.qi] = m[t2];
      scale_s[wave][16 * t2 + L.qi] = scale;
    }
#pragma unroll
    for (int db = 0; db < T::kBlocks; ++db) {
      const f32x4 v = o[t2][db] * scale;
      if (row < rows && used == 1) store4<DT>(a.out, (row_base + row) * HD + 16 * db + 4 * L.g, v);
      else if (row < rows) *reinterpret_cast<f32x4*>(a.part_o + (part_base + row) * HD + 16 * db + 4 * L.g) = v;
    }
  }
  if (special != 0)
    add_special_nodes<DT, HD, WINDOW>(a, u, row_base + first_row, part_base + first_row, first_row, min(QR, rows - first_row), used, see(), special, max_s[wave], scale_s[wave]);
}

#pragma clang diagnostic pop

template <int DT, int HD, int NQ, bool STREAMING, bool WINDOW> hipError_t launch_attend(const TreeArgs& a, hipStream_t s) {
  constexpr int kLds = kAttendWaves * 4 * 8192;
  static_assert(16 * NQ * (HD + 4) * 4 <= kLds, "a wave's outputs take the tiles' place");
  const void* const fn = reinterpret_cast<const void*>(tree_attend<DT, HD, NQ, STREAMING, WINDOW>);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) return hipErrorInvalidValue;
  const int per = 8 * a.row_tiles;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(a.units) * a.splits + 7) / 8 * per);
  hipLaunchKernelGGL((tree_attend<DT, HD, NQ, STREAMING, WINDOW>), dim3(blocks), dim3(kAttendThreads), kLds, s, a);
  return hipGetLastError();
}

template <int HD, int NQ, bool WINDOW> hipError_t launch_attend_wide(const TreeArgs& a, hipStream_t s) {
  constexpr int kLds = 4 * 2 * 8192;
  const void* const fn = reinterpret_cast<const void*>(tree_attend_wide<HD, NQ, WINDOW>);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) return hipErrorInvalidValue;
  const int per = 8 * a.row_tiles;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(a.units) * a.splits + 7) / 8 * per);
  hipLaunchKernelGGL((tree_attend_wide<HD, NQ, WINDOW>), dim3(blocks), dim3(kWideThreads), kLds, s, a);
  return hipGetLastError();
}

template <int DT, int HD, int NQ> hipError_t launch_attend_form(const TreeArgs& a, hipStream_t s) {
  if (a.recency_window > 0) return a.streaming ? launch_attend<DT, HD, NQ, true, true>(a, s) : launch_attend<DT, HD, NQ, false, true>(a, s);
  return a.streaming ? launch_attend<DT, HD, NQ, true, false>(a, s) : launch_attend<DT, HD, NQ, false, false>(a, s);
}
// Query rows of a workgroup: up to 64, in tiles of 16; bf16 with more: up to 192.
template <int DT, int HD> hipError_t launch_attend_rows(const TreeArgs& a, hipStream_t s) {
  const int rows = a.nodes * a.group;
  if constexpr (DT == kBF16) {
    if (rows > 64) {
      const bool three = (rows + a.row_tiles - 1) / a.row_tiles > 128;
      if (a.recency_window > 0) return launch_attend_wide<HD, 2, true>(a, s);
      return three ? launch_attend_wide<HD, 3, false>(a, s) : launch_attend_wide<HD, 2, false>(a, s);
    }
  }
  return rows <= 16 ? launch_attend_form<DT, HD, 1>(a, s) : rows <= 32 ? launch_attend_form<DT, HD, 2>(a, s) : launch_attend_form<DT, HD, 4>(a, s);
}

}  // namespace tree
}  // namespace roco
