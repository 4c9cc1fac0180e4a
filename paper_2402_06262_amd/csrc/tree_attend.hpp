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

// NQ tiles of 16 query rows; a row is a node and a head of the group.  WINDOW: a recency bias is in force.
template <int DT, int HD, int NQ, bool WINDOW>
__global__ __launch_bounds__(kAttendThreads, 1) void tree_attend(TreeArgs a) {
  using T = Tile<DT, HD>;
  constexpr int W = kAttendWaves, G = T::kGroups, QR = 16 * NQ;
  constexpr int kTileBytes = 8192, kWaveBytes = 4 * kTileBytes;  // K, K, V, V
  constexpr int kSide = WINDOW ? 1 : 0;                          // the positions of a K tile's slots come along
  extern __shared__ __attribute__((aligned(1024))) char lds[];   // the waves' tiles; then a wave's outputs
  __shared__ __attribute__((aligned(256))) int32_t pos_s[WINDOW ? W : 1][2][kWave];
  __shared__ float merge_m[QR], merge_l[QR];
  // the row tiles of a split go to one die: eight dies take the workgroups in turn
  const int per = 8 * a.row_tiles, id = blockIdx.x;
  const int us = id / per * 8 + id % 8, row_tile = id % per / 8;
  if (us >= a.units * a.splits) return;
  const int u = us / a.splits, split = us % a.splits;
  const int request = u / a.heads;
  const int nodes = __builtin_amdgcn_readfirstlane(a.n_nodes != nullptr ? min(max(a.n_nodes[request], 0), a.nodes) : a.nodes);
  const int rows = nodes * a.group, first_row = row_tile * QR;
  if (first_row >= rows) return;
  const int n = __builtin_amdgcn_readfirstlane(min(max(a.n_used[u], 0), budget_of(a.pages, a.B, request)));
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int qi = lane & 15, g = lane >> 4;

  constexpr int kStep = T::kSlots * W;
  const int chunk = ((n + a.splits - 1) / a.splits + kStep - 1) / kStep * kStep;
  const int row0 = min(n, split * chunk), row1 = min(n, row0 + chunk);
  Walk<DT, HD, W> walk;
  walk.init(a.pages, a.B, a.heads, u, request, row0, row1, split == a.splits - 1 ? nodes : 0, wave, static_cast<unsigned>(u) * 5u + static_cast<unsigned>(split) * 3u);
  const int mine = walk.mine;

  char* const tiles = lds + wave * kWaveBytes;
  const uint32_t tiles_addr = lds_address(tiles), pos_addr = lds_address(&pos_s[WINDOW ? wave : 0][0][0]);
  int koff[T::kGroupLoads], voff[T::kGroupLoads];
  load_offsets<DT, HD, false>(koff);
  load_offsets<DT, HD, true>(voff);
  const v4i32 pbuf = make_buffer(a.pos + static_cast<size_t>(u) * a.B, WINDOW ? static_cast<uint32_t>(a.B) * 4u : 0u);
  const char* const new_k = static_cast<const char*>(a.k_new) + static_cast<size_t>(u) * a.nodes * T::kBytes;
  const char* const new_v = static_cast<const char*>(a.v_new) + static_cast<size_t>(u) * a.nodes * T::kBytes;
  typedef typename Walk<DT, HD, W>::Place Place;
  auto request_k = [&](int t, const Place& p) {
    const bool of_nodes = walk.is_nodes(t);
    request_tile<DT, HD>(of_nodes ? new_k : static_cast<const char*>(a.K), p.row, p.there, tiles_addr + (t & 1) * kTileBytes, koff);
    // (a wave-wide load of 64 words, whatever the tile; behind the unit's last slot, and for nodes, zeros)
    if (WINDOW) mfma::load4_to_lds(pbuf, pos_addr + (t & 1) * (kWave * 4), of_nodes ? 0x7ffffffc : (walk.first_slot(t) + lane) * 4, 0);
  };
  auto request_v = [&](int t, const Place& p) {
    request_tile<DT, HD>(walk.is_nodes(t) ? new_v : static_cast<const char*>(a.V), p.row, p.there, tiles_addr + (2 + (t & 1)) * kTileBytes, voff);
  };

  // B operand: the queries (lanes behind the last row repeat it; their results are dropped)
  uint4 own[NQ][T::kSteps];
  int token[NQ];
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {
    const int row = min(first_row + 16 * t2 + qi, rows - 1);
    token[t2] = row / a.group;
    const char* const q = static_cast<const char*>(a.q) + (static_cast<size_t>(u) * a.nodes * a.group + row) * T::kBytes;
#pragma unroll
    for (int kk = 0; kk < T::kSteps; ++kk) own[t2][kk] = load16(q + kk * 64 + g * 16);
  }
  uint32_t there[3] = {0, 0, 0};  // of this tile and the two behind it
  if (mine > 0) {
    const Place p = walk.place(0);
    there[0] = p.there;
    request_k(0, p);
    request_v(0, p);
  }
  if (mine > 1) {
    const Place p = walk.place(1);
    there[1] = p.there;
    request_k(1, p);
    request_v(1, p);
  }
  const float sc = a.scale_log2, rb = a.recency_bias_log2;
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[u] : 0;
  int qp[NQ];
  uint64_t seen = 0;  // by node `lane`
  if (WINDOW) {
    seen = seen_nodes(a.parent != nullptr ? a.parent + static_cast<size_t>(request) * a.nodes : nullptr, nodes, lane);
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) qp[t2] = qp0 + __shfl(__builtin_popcountll(seen), token[t2], kWave) - 1;
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
  const int kfrag = qi * T::kBytes + ((g ^ T::swizzle_k(qi)) << 4);
  // bf16: V^T of dimensions 0..15, rows 4 g + lane / 4 % 4, 8 bytes from column 4 (lane % 4) on; fp32: row 4 g, column lane % 16
  const int vrow = DT == kBF16 ? 4 * g + (qi >> 2) : 4 * g;
  const int vfrag = DT == kBF16 ? vrow * T::kBytes + (T::swizzle_v(vrow) << 4) + (qi & 3) * 8 : vrow * T::kBytes + (T::swizzle_v(vrow) << 4) + qi * 4;

#pragma unroll 1
  for (int t = 0; t < mine; ++t) {
    const char* const tileK = tiles + (t & 1) * kTileBytes;
    char* const tileV = tiles + (2 + (t & 1)) * kTileBytes;
    const bool of_nodes = walk.is_nodes(t);
    if (t + 1 < mine) wait_loads<3 * T::kLoads + kSide>();
    else wait_loads<T::kLoads>();
    f32x4 s[NQ][G];
#pragma unroll
    for (int kk = 0; kk < T::kSteps; ++kk) {
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const uint4 kf = *reinterpret_cast<const uint4*>(tileK + i * 16 * T::kBytes + (kfrag ^ (kk << 6)));
#pragma unroll
        for (int t2 = 0; t2 < NQ; ++t2) s[t2][i] = score_step<DT>(kf, own[t2][kk], kk == 0 ? f32x4{0} : s[t2][i]);
      }
    }
    int ps[G][4];
    if (WINDOW) {
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const int4 p4 = *reinterpret_cast<const int4*>(&pos_s[WINDOW ? wave : 0][t & 1][16 * i + 4 * g]);
        ps[i][0] = p4.x; ps[i][1] = p4.y; ps[i][2] = p4.z; ps[i][3] = p4.w;
      }
    }
    reads_done();
    Place next;
    if (t + 2 < mine) {
      next = walk.place(t + 2);
      there[2] = next.there;
      request_k(t + 2, next);
    }
    // ---- base-2 logits; what a row does not see, or is not there, is -inf
    if (of_nodes) {
      if (!WINDOW) seen = seen_nodes(a.parent != nullptr ? a.parent + static_cast<size_t>(request) * a.nodes : nullptr, nodes, lane);
      const int j0 = walk.first_node(t);
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (WINDOW) ps[i][e] = qp0 + __shfl(__builtin_popcountll(seen), min(j0 + 16 * i + 4 * g + e, kWave - 1), kWave) - 1;
        }
    }
    constexpr uint32_t kWhole = G == 1 ? 0x10u : G == 2 ? 0x1010u : 0x10101010u;
    const bool whole = there[0] == kWhole && !of_nodes;
#pragma unroll
    for (int t2 = 0; t2 < NQ; ++t2) {
      uint64_t sees = ~0ull;
      if (of_nodes) sees = from_lane(seen, token[t2]);
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
          if (!whole) {
            const int at = 4 * g + e;
            const bool visible = at < static_cast<int>((there[0] >> (8 * i)) & 0xffu) &&
                                 (!of_nodes || ((sees >> (walk.first_node(t) + 16 * i + at)) & 1) != 0);
            x = visible ? x : -INFINITY;
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
      // A node's value that is infinite or NaN must not reach the rows that do not see the node, and 0 times it would: such rows are
      // added by themselves, to the rows that see them, and zero for the products.
      const auto special = [](const uint4& v) {
        const auto one = [](uint32_t x) {
          return (x & 0x7f800000u) == 0x7f800000u || (DT == kBF16 && (x & 0x7f80u) == 0x7f80u);
        };
        return one(v.x) || one(v.y) || one(v.z) || one(v.w);
      };
      bool any = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) any = any || special(*reinterpret_cast<const uint4*>(tileV + i * 1024 + lane * 16));
      if (__any(any)) {
        const int j0 = walk.first_node(t);
#pragma unroll 1
        for (int j = 0; j < min(T::kSlots, nodes - j0); ++j) {
          uint4* const row = reinterpret_cast<uint4*>(tileV + j * T::kBytes);
          if (!__any(special(row[lane % T::kChunks]))) continue;
#pragma unroll
          for (int t2 = 0; t2 < NQ; ++t2) {
            float p = 0.0f;
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (j >> 4 == i && (j & 3) == e) p = s[t2][i][e];
            p = __shfl(p, ((j >> 2) & 3) * 16 + qi, kWave);
            const bool visible = ((from_lane(seen, token[t2]) >> (j0 + j)) & 1) != 0;
#pragma unroll
            for (int db = 0; db < T::kBlocks; ++db) {
              f32x4 v;
              if constexpr (DT == kBF16) {
                const uint2 b = *reinterpret_cast<const uint2*>(tileV + j * T::kBytes + (((2 * db + (g >> 1)) ^ T::swizzle_v(j)) << 4) + (g & 1) * 8);
                v = f32x4{__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xffff0000u), __uint_as_float(b.y << 16), __uint_as_float(b.y & 0xffff0000u)};
              } else {
                v = *reinterpret_cast<const f32x4*>(tileV + j * T::kBytes + (((4 * db + g) ^ T::swizzle_v(j)) << 4));
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) o[t2][db][e] = visible ? fmaf(p, v[e], o[t2][db][e]) : o[t2][db][e];
            }
          }
          reads_done();
          if (lane < T::kChunks) row[lane] = make_uint4(0u, 0u, 0u, 0u);
          reads_done();
        }
      }
    }
    if constexpr (DT == kBF16) {
      // The probabilities as sums of two bf16 numbers: rounded to one they would make as much of the output's error as its own rounding
      // (2.4e-3 against 1.7e-3 of its norm); the matrix cores have the time.
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
    if (t + 2 < mine) request_v(t + 2, next);
    there[0] = there[1];
    there[1] = there[2];
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
#pragma unroll
  for (int t2 = 0; t2 < NQ; ++t2) {
    const int q = 16 * t2 + qi, row = first_row + q;
    if (row >= rows) continue;
    const float m1 = merge_m[q], l1 = merge_l[q];
    // (a maximum is -inf where a wave has seen nothing, or nothing but logits of -inf or NaN: NaN sums stay)
    const float M = fmaxf(m[t2], m1);
    const float w0 = m[t2] > -INFINITY ? fast_exp2(m[t2] - M) : 1.0f, w1 = m1 > -INFINITY ? fast_exp2(m1 - M) : 1.0f;
    const float sum = l[t2] * w0 + l1 * w1;
    const size_t at = static_cast<size_t>(u) * a.nodes * a.group + row;
    const size_t part = (static_cast<size_t>(u) * a.splits + split) * a.nodes * a.group + row;
    const float scale = a.splits == 1 ? 1.0f / sum : 1.0f;
    if (g == 0) {
      if (a.splits == 1) {
        if (a.lse != nullptr) a.lse[at] = kLn2 * (M + __log2f(sum));
      } else {
        a.part_m[part] = M;
        a.part_l[part] = sum;
      }
    }
#pragma unroll
    for (int db = 0; db < T::kBlocks; ++db) {
      const f32x4 other = *reinterpret_cast<const f32x4*>(outs + q * kOut + 16 * db + 4 * g);
      const f32x4 v = (o[t2][db] * w0 + other * w1) * scale;
      if (a.splits == 1) store4<DT>(a.out, at * HD + 16 * db + 4 * g, v);
      else *reinterpret_cast<f32x4*>(a.part_o + part * HD + 16 * db + 4 * g) = v;
    }
  }
}

#pragma clang diagnostic pop

template <int DT, int HD, int NQ, bool WINDOW> hipError_t launch_attend(const TreeArgs& a, hipStream_t s) {
  constexpr int kLds = kAttendWaves * 4 * 8192;
  static_assert(16 * NQ * (HD + 4) * 4 <= kLds, "a wave's outputs take the tiles' place");
  const void* const fn = reinterpret_cast<const void*>(tree_attend<DT, HD, NQ, WINDOW>);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) return hipErrorInvalidValue;
  const int per = 8 * a.row_tiles;
  const unsigned blocks = static_cast<unsigned>((static_cast<long long>(a.units) * a.splits + 7) / 8 * per);
  hipLaunchKernelGGL((tree_attend<DT, HD, NQ, WINDOW>), dim3(blocks), dim3(kAttendThreads), kLds, s, a);
  return hipGetLastError();
}

// Query rows of a workgroup: up to 64, in tiles of 16.
template <int DT, int HD> hipError_t launch_attend_rows(const TreeArgs& a, hipStream_t s) {
  const int rows = a.nodes * a.group;
  if (a.recency_window > 0)
    return rows <= 16 ? launch_attend<DT, HD, 1, true>(a, s) : rows <= 32 ? launch_attend<DT, HD, 2, true>(a, s) : launch_attend<DT, HD, 4, true>(a, s);
  return rows <= 16 ? launch_attend<DT, HD, 1, false>(a, s) : rows <= 32 ? launch_attend<DT, HD, 2, false>(a, s) : launch_attend<DT, HD, 4, false>(a, s);
}

}  // namespace tree
}  // namespace roco
