// Attention of drafted trees over the budgeted cache: out = softmax(scale q . [K of the cache; k of the nodes seen]) [V; v], and
// ln of the softmax's sum, without a change to the cache.
//
// One pass over K and V with a running maximum and sum.  A wave streams tiles of 8 KiB of either through LDS of its own, two of each,
// filled by loads that go straight there and ordered by the wave's own load counter: no barrier, and three operand tiles of a wave on
// their way at any time.  Scores = K . Q^T on the matrix cores, so that a lane holds four slots of one query; the outputs' products
// O^T = V^T . P^T take these registers as they are.  A tree's nodes are tiles of the last split like any others, but for their mask.
// The running maximum follows a tile's only when that is more than 2^8 above it: no rescaling, and no exchange between lanes, for most
// tiles, and the sums stay far from the ends of fp32.
#pragma once
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

template <int DT> __device__ __forceinline__ void store4(void* base, size_t idx, const f32x4& v) {
  if constexpr (DT == kBF16) {
    uint2 r;
    r.x = f32_to_bf16(v.x) | static_cast<uint32_t>(f32_to_bf16(v.y)) << 16;
    r.y = f32_to_bf16(v.z) | static_cast<uint32_t>(f32_to_bf16(v.w)) << 16;
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + idx) = r;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(base) + idx) = v;
  }
}

// Whether 16 bytes of values hold an infinite one or NaN.
template <int DT> __device__ __forceinline__ bool holds_special(const uint4& v) {
  // (the exponent's bits set: adding one to them carries)
  const auto one = [](uint32_t x) {
    if (DT == kBF16) return ((x & 0x7f800000u) + 0x00800000u) | (((x & 0x7f80u) + 0x80u) << 16);
    return (x & 0x7f800000u) + 0x00800000u;
  };
  return ((one(v.x) | one(v.y) | one(v.z) | one(v.w)) & 0x80000000u) != 0;
}
template <int DT> __device__ __forceinline__ float load_elem(const void* base, size_t idx) {
  if constexpr (DT == kBF16) return bf16_to_f32(static_cast<const uint16_t*>(base)[idx]);
  else return static_cast<const float*>(base)[idx];
}

// NQ tiles of 16 query rows; a row is a node and a head of the group.  WINDOW: a recency bias is in force.
// A launch begins with a cold instruction cache, a third of a microsecond per KiB, so that nothing is unrolled that need not be: the
// loop over the tiles begins two tiles early, with the requests alone, and what is rare loops over rows.
template <int DT, int HD, int NQ, bool STREAMING, bool WINDOW>
__global__ __launch_bounds__(kAttendThreads, 1) void tree_attend(TreeArgs a) {
  using T = Tile<DT, HD>;
  constexpr int W = kAttendWaves, G = T::kGroups, QR = 16 * NQ;
  constexpr int kTileBytes = 8192, kWaveBytes = 4 * kTileBytes;  // K, V, K, V
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
  const int u = us / a.splits, split = us % a.splits;
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

  const float sc = a.scale_log2, rb = a.recency_bias_log2;
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[u] : 0;
  const auto token_of = [&](int t2) { return min(first_row + 16 * t2 + qi, rows - 1) / a.group; };
  const auto see = [&]() { return seen_nodes(parent, nodes, lane); };
  uint64_t seen = 0, special = 0;  // by node `lane`; nodes whose values are not finite
  int qp[NQ];
  if (WINDOW) {
    seen = see();
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) qp[t2] = qp0 + __shfl(__builtin_popcountll(seen), token_of(t2), kWave) - 1;
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

  uint32_t there0 = 0, there1 = 0, there2 = 0;  // of this tile and the two behind it
#pragma unroll 1
  for (int t = -2; t < mine; ++t) {
    char* const tileK = tiles + (t & 1) * 2 * kTileBytes;
    char* const tileV = tileK + kTileBytes;
    f32x4 s[NQ][G];
    int ps[G][4];
    if (t >= 0) {
      // K(t) has landed; V(t), and K and V of the next tile, may still be on their way
      if (t + 1 < mine) wait_loads<3 * T::kLoads + kSide>();
      else wait_loads<T::kLoads>();
#pragma unroll
      for (int kk = 0; kk < T::kSteps; ++kk) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const uint4 kf = *reinterpret_cast<const uint4*>(tileK + i * 16 * T::kBytes + (kfrag ^ (kk << 6)));
#pragma unroll
          for (int t2 = 0; t2 < NQ; ++t2) s[t2][i] = score_step<DT>(kf, own[t2][kk], kk == 0 ? f32x4{0} : s[t2][i]);
        }
      }
      if (WINDOW) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const int4 p4 = *reinterpret_cast<const int4*>(&pos_s[WINDOW ? wave : 0][t & 1][16 * i + 4 * g]);
          ps[i][0] = p4.x; ps[i][1] = p4.y; ps[i][2] = p4.z; ps[i][3] = p4.w;
        }
      }
      reads_done();
    } else if (kBeforeK && t == -1) {
      if (mine > 0) wait_loads<2 * T::kLoads + kSide>();
      else wait_loads<0>();
      read_queries();
    }
    typename Walk<DT, HD, W>::Place next;
    bool next_nodes = false;
    if (t + 2 < mine) {
      next = walk.place(t + 2);
      there2 = next.there;
      next_nodes = walk.is_nodes(t + 2);
      request_tile<DT, HD, STREAMING>(next_nodes ? static_cast<const char*>(a.k_new) + new_rows : static_cast<const char*>(a.K), next.row, next.there, lds_address(tileK), koff);
      // (a wave-wide load of 64 words, whatever the tile; behind the unit's last slot, and for nodes, zeros)
      if (WINDOW) mfma::load4_to_lds(pbuf, pos_addr + (t & 1) * (kWave * 4), next_nodes ? 0x7ffffffc : (walk.first_slot(t + 2) + lane) * 4, 0);
    }
    if (t >= 0) {
      const bool of_nodes = walk.is_nodes(t);
      constexpr uint32_t kWhole = G == 1 ? 0x10u : G == 2 ? 0x1010u : 0x10101010u;
      if (of_nodes) {
        if (!WINDOW) seen = see();
        const int j0 = walk.first_node(t);
#pragma unroll
        for (int i = 0; i < G; ++i) {
          if (WINDOW) {
#pragma unroll
            for (int e = 0; e < 4; ++e) ps[i][e] = qp0 + __shfl(__builtin_popcountll(seen), min(j0 + 16 * i + 4 * g + e, kWave - 1), kWave) - 1;
          }
        }
#pragma unroll
        for (int t2 = 0; t2 < NQ; ++t2) {
          const uint64_t sees = from_lane(seen, token_of(t2)) >> j0;
#pragma unroll
          for (int i = 0; i < G; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t2][i][e] = (sees >> (16 * i + 4 * g + e)) & 1 ? s[t2][i][e] : -INFINITY;
        }
      } else if (there0 != kWhole) {
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool visible = 4 * g + e < static_cast<int>((there0 >> (8 * i)) & 0xffu);
#pragma unroll
            for (int t2 = 0; t2 < NQ; ++t2) s[t2][i][e] = visible ? s[t2][i][e] : -INFINITY;
          }
      }
      // ---- base-2 logits and probabilities; what a row does not see is -inf
#pragma unroll
      for (int t2 = 0; t2 < NQ; ++t2) {
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = s[t2][i][e] * sc;
            if (WINDOW) {
              const int away = qp[t2] - ps[i][e];
              if (away >= 0 && away < w) x += rb;
            }
            s[t2][i][e] = x;
            most = fmaxf(most, x);
          }
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
            s[t2][i][e] = fast_exp2(s[t2][i][e] - ref);
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
#pragma unroll
        for (int i = 0; i < 8; ++i) any |= holds_special<DT>(*reinterpret_cast<const uint4*>(tileV + i * 1024 + lane * 16));
        if (__any(any)) {
          const int j0 = walk.first_node(t);
#pragma unroll 1
          for (int j = 0; j < min(T::kSlots, nodes - j0); ++j) {
            uint4* const row = reinterpret_cast<uint4*>(tileV + j * T::kBytes) + lane % T::kChunks;
            if (!__any(holds_special<DT>(*row))) continue;
            special |= 1ull << (j0 + j);
            *row = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        reads_done();
      }
      if constexpr (DT == kBF16) {
        // The probabilities as sums of two bf16 numbers: rounded to one they would make as much of the output's error as its own
        // rounding (2.4e-3 against 1.7e-3 of its norm); the matrix cores have the time.
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
            const char* const vt = tileV + i * 16 * T::kBytes + (vfrag ^ (db << 5));
            const uint2 lo = lds_read_transposed(vt), hi = lds_read_transposed(vt + 16 * T::kBytes);
            const uint4 vf = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
            for (int k = 1; k >= 0; --k)
#pragma unroll
              for (int t2 = 0; t2 < NQ; ++t2) o[t2][db] = fused::mfma16(vf, p[t2][k], o[t2][db]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int db = 0; db < T::kBlocks; ++db) {
            const char* const vt = tileV + i * 16 * T::kBytes + (vfrag ^ (db << 6));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = *reinterpret_cast<const float*>(vt + e * T::kBytes);
#pragma unroll
              for (int t2 = 0; t2 < NQ; ++t2) o[t2][db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[t2][i][e], o[t2][db], 0, 0, 0);
            }
          }
      }
      reads_done();
    }
    if (kBehindK && t == -1) {
      if (mine > 1) wait_loads<3 * T::kLoads + 2 * kSide>();
      else if (mine > 0) wait_loads<2 * T::kLoads + kSide>();
      else wait_loads<0>();
      read_queries();
    }
    if (t + 2 < mine) request_tile<DT, HD, STREAMING>(next_nodes ? static_cast<const char*>(a.v_new) + new_rows : static_cast<const char*>(a.V), next.row, next.there, lds_address(tileV), voff);
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
  const bool any_special = special != 0;
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
      float* const at = outs + q * kOut + 16 * db + 4 * g;
      const f32x4 v = (o[t2][db] * w0 + *reinterpret_cast<const f32x4*>(at) * w1) * scale;
      if (any_special) *reinterpret_cast<f32x4*>(at) = v;
      else if (row < rows && used == 1) store4<DT>(a.out, (row_base + row) * HD + 16 * db + 4 * g, v);
      else if (row < rows) *reinterpret_cast<f32x4*>(a.part_o + (part_base + row) * HD + 16 * db + 4 * g) = v;
    }
  }
  if (!any_special) return;
  seen = see();
  // a row at a time, HD / 64 of its elements per lane: what the nodes add that were left out
  constexpr int E = HD / kWave;
#pragma unroll 1
  for (int q = 0; q < min(QR, rows - first_row); ++q) {
    const int row = first_row + q, token = row / a.group;
    const uint64_t sees = from_lane(seen, token);
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = outs[q * kOut + lane * E + e];
#pragma unroll 1
    for (uint64_t left = sees & special; left != 0; left &= left - 1) {
      const int j = __builtin_ctzll(left);
      const size_t node = (static_cast<size_t>(u) * a.nodes + j) * HD + lane * E;
      float dot = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) dot = fmaf(load_elem<DT>(a.q, (row_base + row) * HD + lane * E + e), load_elem<DT>(a.k_new, node + e), dot);
      float x = group_sum<kWave>(dot) * sc;
      if (WINDOW && __builtin_popcountll(sees) - __builtin_popcountll(from_lane(seen, j)) < w) x += rb;
      const float p = fast_exp2(x - (merge_m[q] > -INFINITY ? merge_m[q] : 0.0f)) * merge_l[q];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = fmaf(p, load_elem<DT>(a.v_new, node + e), v[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (used == 1) store_elem<DT>(a.out, (row_base + row) * HD + lane * E + e, v[e]);
      else a.part_o[(part_base + row) * HD + lane * E + e] = v[e];
    }
  }
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

template <int DT, int HD, int NQ> hipError_t launch_attend_form(const TreeArgs& a, hipStream_t s) {
  if (a.recency_window > 0) return a.streaming ? launch_attend<DT, HD, NQ, true, true>(a, s) : launch_attend<DT, HD, NQ, false, true>(a, s);
  return a.streaming ? launch_attend<DT, HD, NQ, true, false>(a, s) : launch_attend<DT, HD, NQ, false, false>(a, s);
}
// Query rows of a workgroup: up to 64, in tiles of 16.
template <int DT, int HD> hipError_t launch_attend_rows(const TreeArgs& a, hipStream_t s) {
  const int rows = a.nodes * a.group;
  return rows <= 16 ? launch_attend_form<DT, HD, 1>(a, s) : rows <= 32 ? launch_attend_form<DT, HD, 2>(a, s) : launch_attend_form<DT, HD, 4>(a, s);
}

}  // namespace tree
}  // namespace roco
