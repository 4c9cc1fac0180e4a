// Attention of a chunk of new tokens over the budgeted cache and itself:  out = softmax(scale q . [K of the cache; k of the tokens up to its own])
// [V; v], and ln of the softmax's sum, without a change to the cache.
//
// One pass over the keys with a running reference and sum.  A workgroup has 128 query rows of a unit, (token, head) pairs, 32 to a wave, in
// registers; keys and values come in tiles of 32 through a ring in LDS, filled by loads that go straight there, first the cache's, then the chunk's.
// Scores = K . Q^T on the matrix cores, so that a lane holds 16 keys of one query, and the outputs' products O^T = V^T . P^T take these
// registers as they are (of bf16, rounded to bf16).
#pragma once
#include "chunk.hpp"
#include "profile.hpp"

namespace roco {
namespace chunk {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

constexpr int kRowTile = 128;  // query rows of a workgroup
constexpr int kKeyTile = 32;   // keys of a stage
constexpr float kLn2 = 0.6931471805599453f;

template <int DT, int HD> struct AttendForm {
  using R = Rows<DT, HD>;
  static constexpr int kTileBytes = kKeyTile * R::kBytes;         // of K, then as many of V
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kStages = kStageBytes <= 16384 ? 3 : 2;
  static constexpr int kAhead = kStages - 1;                      // tiles that are asked for before their turn
  static constexpr int kLoads = 8 * R::kBytes / 1024;             // of a wave, for its eight rows of K or of V
  static constexpr int kWavesPerSimd = DT == kF32 ? 2 : HD == 128 ? 3 : 4;
};

// Whether 16 bytes hold an infinite value or NaN.
template <int DT> __device__ __forceinline__ bool holds_special(const uint4& v) {
  // (the exponent's bits set: adding one to them carries)
  const auto one = [](uint32_t x) {
    if (DT == kBF16) return ((x & 0x7f800000u) + 0x00800000u) | (((x & 0x7f80u) + 0x80u) << 16);
    return (x & 0x7f800000u) + 0x00800000u;
  };
  return ((one(v.x) | one(v.y) | one(v.z) | one(v.w)) & 0x80000000u) != 0;
}

template <int DT, int HD, bool WINDOW>
__global__ __launch_bounds__(kThreads, (AttendForm<DT, HD>::kWavesPerSimd)) void chunk_attend(ChunkArgs a, int row_tiles) {
  using R = Rows<DT, HD>;
  using F = AttendForm<DT, HD>;
  constexpr int kSide = WINDOW ? 1 : 0;  // the positions of a tile's slots come along
  constexpr int kTileLoads = 2 * F::kLoads + kSide;
  extern __shared__ __attribute__((aligned(1024))) char ring[];
  __shared__ __attribute__((aligned(256))) int32_t pos_s[WINDOW ? kWaves : 1][F::kStages][kWave];
  // (unit's head, split) pairs side by side on a die, the eight dies taking a contiguous share each; the later row tiles, which see more, first
  const int total = row_tiles * a.heads * a.splits, share = (total + 7) / 8;
  const int id = static_cast<int>(blockIdx.x % 8) * share + static_cast<int>(blockIdx.x / 8);
  if (static_cast<int>(blockIdx.x / 8) >= share || id >= total) return;
  const int pair = id / row_tiles, head = pair % a.heads, split = pair / a.heads;
  Located at;
  if (!locate_tile<kRowTile>(a, a.group, row_tiles - 1 - id % row_tiles, at)) return;
  const int rows = at.count * a.group, first_row = at.tile * kRowTile;
  if (first_row >= rows) return;
  const int u = at.request * a.heads + head;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int half = lane >> 5;
  const int n = __builtin_amdgcn_readfirstlane(min(max(a.n_used[u], 0), budget_of(a.pages, a.B, at.request)));
  // the tiles of keys that the row tile sees, and this workgroup's share of them
  const int cache_tiles = (n + kKeyTile - 1) / kKeyTile;
  const int tiles = __builtin_amdgcn_readfirstlane(cache_tiles + (min(rows, first_row + kRowTile) - 1) / a.group / kKeyTile + 1);
  const int per = __builtin_amdgcn_readfirstlane((tiles + a.splits - 1) / a.splits);
  const int t0 = __builtin_amdgcn_readfirstlane(split * per), t1 = min(tiles, t0 + per);
  const size_t all_rows = static_cast<size_t>(a.tokens) * a.heads * a.group;

  // this lane's query: row `row` of the request's, of token `token`
  const int wave_row = first_row + 32 * wave, row = wave_row + (lane & 31);
  const int token = min(row, rows - 1) / a.group;
  const int wave_first = wave_row / a.group, wave_last = (min(rows, wave_row + 32) - 1) / a.group;  // tokens of the wave's rows
  const bool idle = wave_row >= rows;
  // of the packed rows, [tokens][heads][group]
  const size_t out_row = (static_cast<size_t>(at.first + token) * a.heads + head) * a.group + (min(row, rows - 1) - token * a.group);

  float m = -INFINITY, l = 0.0f;
  f32x16 o[R::kBlocks];
#pragma unroll
  for (int db = 0; db < R::kBlocks; ++db) o[db] = f32x16{0};

  if (t0 < t1) {
    const Groups groups(a.pages, a.B, a.heads, at.request, head);
    const uint32_t ring_addr = lds_address(ring), pos_addr = lds_address(&pos_s[WINDOW ? wave : 0][0][0]);
    // this lane's chunks of a tile: the wave fetches rows 8 wave .. 8 wave + 7
    int koff[F::kLoads], voff[F::kLoads];
#pragma unroll
    for (int i = 0; i < F::kLoads; ++i) {
      const int r = R::kPerLoad * i + lane / R::kChunks, in_tile = 8 * wave + r;
      koff[i] = r * R::kBytes + (((lane % R::kChunks) ^ R::swizzle_k(in_tile)) << 4);
      voff[i] = r * R::kBytes + (((lane % R::kChunks) ^ R::swizzle_v(in_tile)) << 4);
    }
    const v4i32 pbuf = make_buffer(a.pos + static_cast<size_t>(u) * a.B, WINDOW ? static_cast<uint32_t>(n) * 4u : 0u);
    const char* const new_k = static_cast<const char*>(a.k_new) + static_cast<int64_t>(at.first) * a.kv_stride + static_cast<size_t>(head) * R::kBytes;
    const char* const new_v = static_cast<const char*>(a.v_new) + static_cast<int64_t>(at.first) * a.kv_stride + static_cast<size_t>(head) * R::kBytes;
    const int more_stride = static_cast<int>(a.kv_stride) - R::kBytes;  // of the chunk's rows
    int ahead[2] = {0, 0};  // pages of the two groups of the tile that is asked for next
    const auto look_ahead = [&](int t) {
      if (t >= min(t1, cache_tiles)) return;
#pragma unroll
      for (int i = 0; i < 2; ++i) ahead[i] = __builtin_amdgcn_readfirstlane(groups.page_of(min(t * kKeyTile + 16 * i, n - 1)));
    };
    // Asks for a tile; the result: how many slots of its groups are there, a byte each.
    const auto request = [&](int t, int stage) {
      const uint32_t dst = ring_addr + stage * F::kStageBytes + wave * 8 * R::kBytes;
      uint32_t there = 0x1010u;
      const int sub = 8 * (wave & 1);  // of the wave's rows in their group
      if (t < cache_tiles) {
        uint32_t row_at = 0;
        there = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int slot = t * kKeyTile + 16 * i;
          uint32_t r;
          int count = __builtin_amdgcn_readfirstlane(min(max(n - slot, 0), 16));
          if (!groups.row_of(slot, ahead[i], r)) count = 0;
          there |= static_cast<uint32_t>(count) << (8 * i);
          if (i == wave >> 1) row_at = count > 0 ? r : 0u;
        }
        const uint32_t mine = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(min(max(static_cast<int>((there >> (8 * (wave >> 1))) & 0xffu) - sub, 0), 8)));
        const size_t byte = static_cast<size_t>(row_at + (mine > 0 ? sub : 0)) * R::kBytes;
        const v4i32 kbuf = make_buffer(static_cast<const char*>(a.K) + byte, mine * R::kBytes), vbuf = make_buffer(static_cast<const char*>(a.V) + byte, mine * R::kBytes);
#pragma unroll
        for (int i = 0; i < F::kLoads; ++i) load16_to_lds(kbuf, dst + i * 1024, koff[i], 0);
#pragma unroll
        for (int i = 0; i < F::kLoads; ++i) load16_to_lds(vbuf, dst + F::kTileBytes + i * 1024, voff[i], 0);
        look_ahead(t + 1);
      } else {
        const int j = (t - cache_tiles) * kKeyTile + 8 * wave, mine = __builtin_amdgcn_readfirstlane(min(max(at.count - j, 0), 8));
        const int64_t byte = static_cast<int64_t>(mine > 0 ? j : 0) * a.kv_stride;
        const uint32_t size = mine > 0 ? static_cast<uint32_t>(mine - 1) * static_cast<uint32_t>(a.kv_stride) + R::kBytes : 0u;
        const v4i32 kbuf = make_buffer(new_k + byte, size), vbuf = make_buffer(new_v + byte, size);
#pragma unroll
        for (int i = 0; i < F::kLoads; ++i) {
          const int more = (R::kPerLoad * i + lane / R::kChunks) * more_stride;
          load16_to_lds(kbuf, dst + i * 1024, koff[i] + more, 0);
          load16_to_lds(vbuf, dst + F::kTileBytes + i * 1024, voff[i] + more, 0);
        }
      }
      // (a wave-wide load of 64 words; behind the unit's last slot, and for the chunk's tokens, zeros)
      if (WINDOW) mfma::load4_to_lds(pbuf, pos_addr + stage * (kWave * 4), t < cache_tiles ? (t * kKeyTile + lane) * 4 : 0x7ffffffc, 0);
      return there;
    };
    uint32_t there[F::kStages];  // of the tile in use and those behind it
    look_ahead(t0);
#pragma unroll
    for (int i = 0; i < F::kAhead; ++i) there[i] = t0 + i < t1 ? request(t0 + i, i) : 0u;
    uint4 own[R::kSteps];
    {
      const char* const q_row = static_cast<const char*>(a.q) + static_cast<int64_t>(at.first + token) * a.q_stride +
                                (static_cast<size_t>(head) * a.group + (min(row, rows - 1) - token * a.group)) * R::kBytes;
#pragma unroll
      for (int kk = 0; kk < R::kSteps; ++kk) own[kk] = load16(q_row + (2 * kk + half) * 16);
    }
    // The queries must have arrived before the loop: a wait for them inside it would also wait for the tiles requested last.
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)

    const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f;
    const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[at.request] : 0;
    // fragment reads: K row lane % 32, chunk 2 kk + half (the tiles lie at multiples of 1 KiB: the step is an exclusive or of the address);
    // V of bf16 transposed, rows 4 half + lane % 16 / 4 (+ 8), 8 bytes of columns 32 db + 16 (lane / 16 % 2) + 4 (lane % 4); of fp32
    // row 4 half (+ e + 8 i), column 32 db + lane % 32
    const uint32_t kfrag = (lane & 31) * R::kBytes + ((half ^ R::swizzle_k(lane & 31)) << 4);
    const int vrow = DT == kBF16 ? 4 * half + ((lane & 15) >> 2) : 4 * half;
    const uint32_t vfrag = F::kTileBytes + vrow * R::kBytes + (R::swizzle_v(vrow) << 4) +
                           (DT == kBF16 ? ((lane >> 4) & 1) * 32 + (lane & 3) * 8 : (lane & 31) * 4);
    int zeroed = 0x7fffffff;  // the first of the chunk's tokens whose value may have been taken out (see below)
    int stage = 0;
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
      if (t + F::kAhead - 1 < t1) wait_loads<(F::kAhead - 1) * kTileLoads>();  // the tiles behind it may still be on their way
      else wait_loads<0>();
      __syncthreads();  // tile t is in LDS, and everybody has issued its last read of tile t - 1
      const uint32_t here = there[0];
#pragma unroll
      for (int i = 0; i + 1 < F::kAhead; ++i) there[i] = there[i + 1];
      const int behind = stage == 0 ? F::kStages - 1 : stage - 1;
      there[F::kAhead - 1] = t + F::kAhead < t1 ? request(t + F::kAhead, behind) : 0u;
      const uint32_t st = ring_addr + stage * F::kStageBytes;
      const int32_t* const pos_t = &pos_s[WINDOW ? wave : 0][stage][0];
      stage = stage == F::kStages - 1 ? 0 : stage + 1;
      const bool of_new = t >= cache_tiles;
      const int j0 = (t - cache_tiles) * kKeyTile;  // the tile's first token
      if (of_new && j0 + kKeyTile - 1 > first_row / a.group) {
        // Some row does not see all of the tile's tokens.  A value that is infinite or NaN must not reach the rows that do not see its token,
        // and 0 times it would: such rows of V are zero in the products, and added in the end to the rows that see them.
        char* const tileV = ring + (st - ring_addr) + F::kTileBytes;
        bool any = false;
#pragma unroll 2
        for (int i = 0; i < F::kTileBytes / 1024; ++i) any |= holds_special<DT>(*reinterpret_cast<const uint4*>(tileV + i * 1024 + lane * 16));
        if (__any(any)) {  // (all waves look at the same tile)
          zeroed = min(zeroed, j0);
          __syncthreads();
#pragma unroll 1
          for (int j = 8 * wave; j < 8 * wave + 8; ++j) {
            uint4* const chunk = reinterpret_cast<uint4*>(tileV + j * R::kBytes) + lane % R::kChunks;
            if (__any(holds_special<DT>(*chunk))) *chunk = make_uint4(0u, 0u, 0u, 0u);
          }
          __syncthreads();
        }
      }
      if (idle || (of_new && j0 > wave_last)) continue;  // nothing that the wave's rows see
      // ---- scores of 32 keys x 32 queries
      f32x16 s = {0};
#pragma unroll
      for (int kk = 0; kk < R::kSteps; ++kk) s = score_step<DT>(tree::lds_read16((st + kfrag) ^ (kk << 5)), own[kk], s);
      // ---- probabilities against the reference m, and their sum
      const bool interior = !WINDOW && (of_new ? j0 + kKeyTile - 1 <= wave_first : here == 0x1010u);
      float sum = 0.0f;
      bool done = false;
      // (of bf16 rounded at once: eight registers, not sixteen)
      f32x16 p;
      bf16x8 pf[2];
      const auto keep = [&](int e, float v) {
        if (DT == kBF16) pf[e >> 3][e & 7] = static_cast<__bf16>(v);
        else p[e] = v;
        sum += v;
      };
      if (interior) {
        // The reference need not be the running maximum: the terms are taken against it as it stands, and only a tile whose sum leaves the safe
        // range -- the first one, whose reference is -inf, and scores that rise by more than 16 powers of two -- raises it below.
        const float neg = -m;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          keep(e, fast_exp2(fmaf(s[e], sc, neg)));
        }
        done = __builtin_amdgcn_ballot_w64(!(sum <= 0x1p16f)) == 0;
      }
      if (!done) {
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int k = 8 * (e >> 2) + 4 * half + (e & 3);  // of the tile's keys
          float x = s[e] * sc;
          if (WINDOW) {
            const int away = qp0 + token - (of_new ? qp0 + j0 + k : pos_t[k]);
            x += static_cast<unsigned>(away) < static_cast<unsigned>(w) ? bias : 0.0f;
          }
          if (!interior) {
            const bool seen = of_new ? j0 + k <= token : (k & 15) < static_cast<int>((here >> (k & 16 ? 8 : 0)) & 0xffu);
            x = seen ? x : -INFINITY;
          }
          s[e] = x;
          most = fmaxf(most, x);
        }
        most = fmaxf(most, __shfl_xor(most, 32, kWave));  // the two halves feed one product
        const float m_new = fmaxf(m, most);
        if (__any(m_new > m)) {
          const float alpha = m > -INFINITY ? fast_exp2(m - m_new) : 0.0f;
          l *= alpha;
#pragma unroll
          for (int db = 0; db < R::kBlocks; ++db) o[db] *= alpha;
        }
        m = m_new;
        const float ref = m > -INFINITY ? m : 0.0f;  // nothing seen yet: every term is 2^-inf = 0
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          keep(e, fast_exp2(s[e] - ref));
        }
      }
      l += sum;
      // ---- O^T += V^T . P^T
      const uint32_t vt = st + vfrag;
      if constexpr (DT == kBF16) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
          for (int db = 0; db < R::kBlocks; ++db) {
            const uint32_t v_at = (vt ^ (db << 6)) + ks * 16 * R::kBytes;
            const uint2 lo = tree::lds_read_transposed_at(v_at), hi = tree::lds_read_transposed_at(v_at + 8 * R::kBytes);
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y)), pf[ks], o[db], 0, 0, 0);
          }
        }
      } else {
        typedef const __attribute__((address_space(3))) float* LdsFloats;
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int db = 0; db < R::kBlocks; ++db) {
            const float v = *(LdsFloats)(static_cast<uintptr_t>((vt ^ (db << 7)) + (8 * (e >> 2) + (e & 3)) * R::kBytes));
            o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[e], o[db], 0, 0, 0);
          }
      }
    }
    if (zeroed != 0x7fffffff && !idle) {
      // the values that were taken out
#pragma unroll 1
      for (int j = zeroed; j < min((t1 - cache_tiles) * kKeyTile, wave_last + 1); ++j) {
        const char *const kj = new_k + static_cast<int64_t>(j) * a.kv_stride, *const vj = new_v + static_cast<int64_t>(j) * a.kv_stride;
        if (!__any(holds_special<DT>(load16(vj + lane % R::kChunks * 16)))) continue;
        float x = 0.0f;
#pragma unroll
        for (int kk = 0; kk < R::kSteps; ++kk) {
          float q8[8], k8[8];
          unpack16<DT>(own[kk], q8);
          unpack16<DT>(load16(kj + (2 * kk + half) * 16), k8);
#pragma unroll
          for (int e = 0; e < Elem<DT>::per16; ++e) x = fmaf(q8[e], k8[e], x);
        }
        x = (x + __shfl_xor(x, 32, kWave)) * sc;
        if (WINDOW && token - j < w) x += bias;
        const float pj = fast_exp2(x - (m > -INFINITY ? m : 0.0f));
        if (j > token) continue;
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db)
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            const int d0 = 32 * db + 8 * g4 + 4 * half;
            float v4[4];
            if constexpr (DT == kBF16) {
              const uint2 r = *reinterpret_cast<const uint2*>(vj + d0 * 2);
              v4[0] = __uint_as_float(r.x << 16); v4[1] = __uint_as_float(r.x & 0xffff0000u);
              v4[2] = __uint_as_float(r.y << 16); v4[3] = __uint_as_float(r.y & 0xffff0000u);
            } else {
              unpack16<kF32>(load16(vj + d0 * 4), v4);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][4 * g4 + e] = fmaf(pj, v4[e], o[db][4 * g4 + e]);
          }
      }
    }
  }
  if (row >= rows) return;
  l += __shfl_xor(l, 32, kWave);  // each half has summed different keys of the same query
  if (a.splits > 1) {
    const size_t part = static_cast<size_t>(split) * all_rows + out_row;
    if (half == 0) {
      a.part_m[part] = m;
      a.part_l[part] = l;
    }
    if (t0 >= t1) return;  // (a share without keys has no outputs either: m = -inf, l = 0)
#pragma unroll
    for (int db = 0; db < R::kBlocks; ++db)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<tree::f32x4*>(a.part_o + part * HD + 32 * db + 8 * g4 + 4 * half) =
            tree::f32x4{o[db][4 * g4], o[db][4 * g4 + 1], o[db][4 * g4 + 2], o[db][4 * g4 + 3]};
    return;
  }
  if (half == 0 && a.lse != nullptr) a.lse[out_row] = kLn2 * (m + __log2f(l));
  const float inv = 1.0f / l;
#pragma unroll
  for (int db = 0; db < R::kBlocks; ++db)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      tree::store4<DT>(a.out, out_row * HD + 32 * db + 8 * g4 + 4 * half,
                       tree::f32x4{o[db][4 * g4] * inv, o[db][4 * g4 + 1] * inv, o[db][4 * g4 + 2] * inv, o[db][4 * g4 + 3] * inv});
}

// The splits' shares of a row, HD / 4 lanes with 16 bytes each; in the order of the splits.
template <int DT, int HD> __global__ __launch_bounds__(kThreads) void chunk_join(ChunkArgs a) {
  constexpr int LANES = HD / 4, PER = kThreads / LANES;
  const size_t all_rows = static_cast<size_t>(a.tokens) * a.heads * a.group;
  const size_t row = static_cast<size_t>(blockIdx.x) * PER + threadIdx.x / LANES;
  // only the tokens that are some request's
  const int from = min(max(a.start[0], 0), a.tokens), to = min(max(a.start[a.requests], 0), a.tokens);
  const size_t per_token = static_cast<size_t>(a.heads) * a.group;
  if (row < from * per_token || row >= to * per_token) return;
  const int sub = threadIdx.x % LANES;
  float M = -INFINITY;
#pragma unroll 4
  for (int i = 0; i < a.splits; ++i) M = fmaxf(M, a.part_m[i * all_rows + row]);
  tree::f32x4 o = tree::f32x4{0};
  float sum = 0.0f;
#pragma unroll 4
  for (int i = 0; i < a.splits; ++i) {
    const float mi = a.part_m[i * all_rows + row], li = a.part_l[i * all_rows + row];
    if (mi == -INFINITY && li == 0.0f) continue;  // a share without keys
    const float w = mi > -INFINITY ? fast_exp2(mi - M) : 1.0f;  // (no maximum: a sum of zero, or NaN)
    o += *reinterpret_cast<const tree::f32x4*>(a.part_o + (i * all_rows + row) * HD + 4 * sub) * w;
    sum += li * w;
  }
  tree::store4<DT>(a.out, row * HD + 4 * sub, o * (1.0f / sum));
  if (a.lse != nullptr && sub == 0) a.lse[row] = kLn2 * (M + __log2f(sum));
}

#pragma clang diagnostic pop

template <int DT, int HD, bool WINDOW> hipError_t launch_attend_form(const ChunkArgs& a, hipStream_t s) {
  using F = AttendForm<DT, HD>;
  constexpr int kLds = F::kStages * F::kStageBytes;
  const void* const fn = reinterpret_cast<const void*>(chunk_attend<DT, HD, WINDOW>);
  if (kLds > 49152 && hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) return hipErrorInvalidValue;
  const int row_tiles = tiles_of(a.requests, a.tokens, a.group, kRowTile);
  const int total = row_tiles * a.heads * a.splits;
  {
    ProfScope ps(kProfChunkAttend, s);
    hipLaunchKernelGGL((chunk_attend<DT, HD, WINDOW>), dim3(static_cast<unsigned>((total + 7) / 8 * 8)), dim3(kThreads), kLds, s, a, row_tiles);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  ProfScope ps(kProfChunkJoin, s);
  constexpr int PER = kThreads / (HD / 4);
  const size_t rows = static_cast<size_t>(a.tokens) * a.heads * a.group;
  hipLaunchKernelGGL((chunk_join<DT, HD>), dim3(static_cast<unsigned>((rows + PER - 1) / PER)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
template <int DT, int HD> hipError_t launch_attend(const ChunkArgs& a, hipStream_t s) {
  return a.recency_window > 0 ? launch_attend_form<DT, HD, true>(a, s) : launch_attend_form<DT, HD, false>(a, s);
}

}  // namespace chunk
}  // namespace roco
