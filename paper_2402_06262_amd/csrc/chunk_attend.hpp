// Attention of a chunk of new tokens over the budgeted cache and itself:  out = softmax(scale q . [K of the cache; k of the tokens up to its own])
// [V; v], and ln of the softmax's sum, without a change to the cache.
//
// One pass over the keys with a running reference and sum.  Query rows, (token, head) pairs of a unit, lie in registers, 32 to a matrix tile; keys and values come
// through a ring in LDS, filled by loads that go straight there, first the cache's, then the chunk's.  Scores = K . Q^T on the matrix cores, so that a
// lane holds 16 keys of one query, and the outputs' products O^T = V^T . P^T take these registers as they are.  Probabilities of bf16 are rounded to bf16, their
// sums are not: outputs 2.3e-3 of their norm off, of which their own rounding is 1.7e-3.  A second number each would be half as many products again, which bound the tiles of many
// rows; of few rows, which the memory should bound, it takes 2 to 12 % more: a token of 32 requests, 8 heads of 4 queries over 4096 keys, 128 dimensions, 100.4 and 102.7 us, of 8
// heads over 2048, 64 dimensions, 34.8 and 39.5, of 64 requests over 1024, 128 dimensions, 23.3 and 26.2.
#pragma once
#include "chunk.hpp"
#include "profile.hpp"

namespace roco {
namespace chunk {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSub = 32;  // keys of a matrix tile

// Whether 16 bytes hold an infinite value or NaN.
template <int DT> __device__ __forceinline__ bool holds_special(const uint4& v) {
  // (the exponent's bits set: adding one to them carries)
  const auto one = [](uint32_t x) {
    if (DT == kBF16) return ((x & 0x7f800000u) + 0x00800000u) | (((x & 0x7f80u) + 0x80u) << 16);
    return (x & 0x7f800000u) + 0x00800000u;
  };
  return ((one(v.x) | one(v.y) | one(v.z) | one(v.w)) & 0x80000000u) != 0;
}

// ROWS rows of a request and a head, whose keys the workgroups of its splits share.
struct RowTile {
  Located at;
  int head, split, first_row, rows;
};
// (The later row tiles, which see more, first; a split's heads, or, where the splits differ, a head's splits side by side.)
template <int ROWS> __device__ __forceinline__ bool row_tile_of(const ChunkArgs& a, int id, RowTile& t, int splits) {
  if (!locate_tile<ROWS>(a, a.group, a.row_tiles - 1 - id % a.row_tiles, t.at)) return false;
  const int pair = id / a.row_tiles;
  const int by = a.equal_shares ? splits : a.heads, first = pair / by, second = pair - first * by;
  t.head = __builtin_amdgcn_readfirstlane(a.equal_shares ? first : second);
  t.split = __builtin_amdgcn_readfirstlane(a.equal_shares ? second : first);
  t.first_row = t.at.tile * ROWS;
  t.rows = min(t.at.count * a.group - t.first_row, ROWS);
  return t.rows > 0;
}
// What it sees, in stages of KEYS keys: the cache's and the chunk's, and the shares of them that its workgroups take.  With equal_shares a share of a tile of more
// than a quarter of its rows is as long as one of the request that sees the most: shorter ones have fewer, and no more of their outputs to be joined.
template <int DT, int ROWS, int KEYS> struct Plan {
  int n, cache_stages, stages, per, used;
  __device__ __forceinline__ Plan(const ChunkArgs& a, const RowTile& t) {
    n = __builtin_amdgcn_readfirstlane(min(max(a.n_used[t.at.request * a.heads + t.head], 0), budget_of(a.pages, a.B, t.at.request)));
    cache_stages = (n + KEYS - 1) / KEYS;
    stages = __builtin_amdgcn_readfirstlane(cache_stages + (t.first_row + t.rows - 1) / a.group / KEYS + 1);
    per = max((stages + a.splits - 1) / a.splits, chunk_least_keys(DT, ROWS) / KEYS);
    if (a.equal_shares && t.rows > ROWS / 4) {
      const int lane = threadIdx.x & (kWave - 1);
      int longest = 0;
#pragma unroll 1
      for (int r = lane; r < a.requests; r += kWave) {
        const int count = min(max(a.start[r + 1], 0), a.tokens) - min(max(a.start[r], 0), a.tokens);
        const int held = min(max(a.n_used[r * a.heads + t.head], 0), budget_of(a.pages, a.B, r));
        if (count > 0) longest = max(longest, held + count);
      }
#pragma unroll
      for (int s = 1; s < kWave; s *= 2) longest = max(longest, __shfl_xor(longest, s, kWave));
      per = max(per, (longest + KEYS * a.splits - 1) / (KEYS * a.splits));
    }
    per = __builtin_amdgcn_readfirstlane(per);
    used = __builtin_amdgcn_readfirstlane((stages + per - 1) / per);
  }
};
// A row's place among the packed ones, [tokens][heads][group]; a split's share of it lies there in the split's plane.
__device__ __forceinline__ size_t packed_row(const ChunkArgs& a, const RowTile& t, int row, int token) {
  return (static_cast<size_t>(t.at.first + token) * a.heads + t.head) * a.group + (row - token * a.group);
}

// This workgroup's row tile: those of a (split, head) pair, which read the same keys, side by side on a die, the eight dies taking a contiguous share each.
template <int ROWS> __device__ __forceinline__ bool my_tile(const ChunkArgs& a, RowTile& mine) {
  const int total = a.row_tiles * a.heads * a.splits, share = (total + 7) / 8;
  const int id = static_cast<int>(blockIdx.x % 8) * share + static_cast<int>(blockIdx.x / 8);
  return id < total && row_tile_of<ROWS>(a, id, mine, a.splits);
}

// A wave's results for NG groups of 32 rows: the values that were taken out (see below) added, and the rows written, or a split's share of them.
template <int DT, int HD, int NG, bool WINDOW> struct Finish {
  using R = Rows<DT, HD>;
  static __device__ __forceinline__ void add_back(const ChunkArgs& a, const RowTile& mine, const int (&token)[NG], const Frag (&own)[NG][R::kSteps], const float (&m)[NG],
                                                  f32x16 (&o)[NG][R::kBlocks], int zeroed, int last_token) {
    const int lane = late_thread_id() & (kWave - 1), half = lane >> 5;
    if (zeroed != 0x7fffffff) {
      const size_t at_head = static_cast<size_t>(mine.head) * R::kBytes;
#pragma unroll 1
      for (int j = zeroed; j <= last_token; ++j) {
        const int64_t byte = static_cast<int64_t>(mine.at.first + j) * a.kv_stride + at_head;
        const char *const kj = static_cast<const char*>(a.k_new) + byte, *const vj = static_cast<const char*>(a.v_new) + byte;
        if (!__any(holds_special<DT>(load16(vj + lane % R::kChunks * 16)))) continue;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          float x = 0.0f;
#pragma unroll
          for (int kk = 0; kk < R::kSteps; ++kk) {
            float q8[8], k8[8];
            unpack16<DT>(__builtin_bit_cast(uint4, own[g][kk]), q8);
            unpack16<DT>(load16(kj + (2 * kk + half) * 16), k8);
#pragma unroll
            for (int e = 0; e < Elem<DT>::per16; ++e) x = fmaf(q8[e], k8[e], x);
          }
          x = (x + __shfl_xor(x, 32, kWave)) * a.scale_log2;
          if (WINDOW && token[g] - j < a.recency_window) x += a.recency_bias_log2;
          const float pj = fast_exp2(x - (m[g] > -INFINITY ? m[g] : 0.0f));
          if (j > token[g]) continue;
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
              for (int e = 0; e < 4; ++e) o[g][db][4 * g4 + e] = fmaf(pj, v4[e], o[g][db][4 * g4 + e]);
            }
        }
      }
    }
  }
  static __device__ __forceinline__ void run(const ChunkArgs& a, const RowTile& mine, int used, const int (&row)[NG], const int (&token)[NG], const Frag (&own)[NG][R::kSteps],
                                             float (&m)[NG], float (&l)[NG], f32x16 (&o)[NG][R::kBlocks], int zeroed, int last_token) {
    const int lane = late_thread_id() & (kWave - 1), half = lane >> 5;
    add_back(a, mine, token, own, m, o, zeroed, last_token);
    const int first_row = mine.first_row, rows = first_row + mine.rows;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      l[g] += __shfl_xor(l[g], 32, kWave);  // each half has summed different keys of the same query
      if (row[g] >= rows) continue;
      const size_t out_row = packed_row(a, mine, row[g], token[g]);
      if (used > 1) {
        const size_t part = mine.split * static_cast<size_t>(a.tokens) * a.heads * a.group + out_row;
        if (half == 0) {
          a.part_m[part] = m[g];
          a.part_l[part] = l[g];
        }
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db)
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4)
            *reinterpret_cast<tree::f32x4*>(a.part_o + part * HD + 32 * db + 8 * g4 + 4 * half) =
                tree::f32x4{o[g][db][4 * g4], o[g][db][4 * g4 + 1], o[g][db][4 * g4 + 2], o[g][db][4 * g4 + 3]};
        continue;
      }
      if (half == 0 && a.lse != nullptr) a.lse[out_row] = kLn2 * (m[g] + __log2f(l[g]));
      const float inv = 1.0f / l[g];
#pragma unroll
      for (int db = 0; db < R::kBlocks; ++db)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
          tree::store4<DT>(a.out, out_row * HD + 32 * db + 8 * g4 + 4 * half,
                           tree::f32x4{o[g][db][4 * g4] * inv, o[g][db][4 * g4 + 1] * inv, o[g][db][4 * g4 + 2] * inv, o[g][db][4 * g4 + 3] * inv});
    }
  }
};

// The rows of the packed ones that this lane has, their tokens, and the queries of the wave's rows as B operands.
template <int DT, int HD, int NG>
__device__ __forceinline__ void take_rows(const ChunkArgs& a, const RowTile& mine, int wave_row, int (&row)[NG], int (&token)[NG], Frag (&own)[NG][Rows<DT, HD>::kSteps]) {
  using R = Rows<DT, HD>;
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5, rows = mine.first_row + mine.rows;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    row[g] = wave_row + 32 * g + (lane & 31);
    const int there = min(row[g], rows - 1);
    token[g] = there / a.group;
    const char* const q_row = static_cast<const char*>(a.q) + static_cast<int64_t>(mine.at.first + token[g]) * a.q_stride +
                              (static_cast<size_t>(mine.head) * a.group + (there - token[g] * a.group)) * R::kBytes;
#pragma unroll
    for (int kk = 0; kk < R::kSteps; ++kk) own[g][kk] = *reinterpret_cast<const Frag*>(q_row + (2 * kk + half) * 16);
  }
}

// The outputs lie in the accumulation registers.  Left to itself the compiler has the queries there, and copies a fragment of them before every
// instruction.  It does not know what the instruction in the assembly does: whoever looks at the outputs waits first (settled).
__device__ __forceinline__ void add_product(f32x16& o, const Frag& v, const Frag& p) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(o) : "v"(v), "v"(p));
}
template <int NG, int BLOCKS> __device__ __forceinline__ void settled(f32x16 (&o)[NG][BLOCKS]) {
  asm volatile("s_nop 15\n\ts_nop 3" ::);
#pragma unroll
  for (int g = 0; g < NG; ++g)
#pragma unroll
    for (int db = 0; db < BLOCKS; ++db) asm volatile("" : "+a"(o[g][db]));
}

// bf16, for many rows.  A wave has NG groups of 32 rows: with two of them a fragment that is read from LDS feeds two matrix instructions (with one, reads at the rate
// of the matrix instructions are all that LDS can give).  Stages of 64 keys, a group of 16 slots asked for by each wave, which then lie in one page.
// A half step takes 32 keys: their probabilities, from scores that the half step before has left, the scores of the next 32, and the products of the 32 before,
// a matrix instruction of either kind in turn, with vector work between them; a wave issues in order, and with the registers of two groups it is alone on its
// SIMD, so that what counts is the number of its instructions.
// Measured, 8 heads of 4 queries, 128 dimensions: 4 requests, 512 tokens over 4096 keys, 159 us (0.92 PFLOP/s), with chunk_attend 191; one, 1024 over 32768, 541 us
// (1.03 PFLOP/s) and 613.  The matrix cores are busy for 40 % of that; without the exponentials it would be 8 % less, without the one or the other product 25 %.
template <int HD> struct PairForm {
  static constexpr int NG = 2;                            // groups of 32 rows of a wave
  using R = Rows<kBF16, HD>;
  static constexpr int kOperand = 64 * R::kBytes;         // bytes of K, or of V, of a stage
  static constexpr int kRing = 4;
  static constexpr int kBytes = 2 * kRing * kOperand;
  static constexpr int kLoads = 16 * R::kBytes / 1024;    // of a wave, for its 16 rows of an operand
};

template <int HD, bool WINDOW>
__global__ __launch_bounds__(kThreads, 1) void chunk_attend_pair(ChunkArgs a) {
  constexpr int DT = kBF16;
  using R = Rows<DT, HD>;
  using F = PairForm<HD>;
  constexpr int NG = F::NG, NR = F::kRing, kSide = 2 * NR;                     // stages whose counts and positions are there
  constexpr int kStageLoads = 2 * F::kLoads + (WINDOW ? 1 : 0);    // the positions of a stage's slots come along
  extern __shared__ __attribute__((aligned(1024))) char ring[];    // stages of K, then of V
  __shared__ __attribute__((aligned(256))) int32_t pos_s[WINDOW ? kWaves : 1][WINDOW ? kSide : 1][kWave];
  __shared__ __attribute__((aligned(16))) int32_t there_s[kSide][kWaves];  // how many of a group's 16 slots, or tokens, are there
  RowTile mine;
  if (!my_tile<4 * 32 * NG>(a, mine)) return;
  const Located& at = mine.at;
  const int head = mine.head, first_row = mine.first_row, rows = first_row + mine.rows;
  const int u = at.request * a.heads + head;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int half = lane >> 5;
  const Plan<DT, 4 * 32 * NG, 64> plan(a, mine);
  const int n = plan.n, cache_stages = plan.cache_stages;
  const int t0 = mine.split * plan.per, t1 = min(plan.stages, t0 + plan.per);
  if (t0 >= t1) return;

  // ---- the wave's 16 rows of a stage
  const uint32_t ring_addr = lds_address(ring) + wave * 16 * R::kBytes;
  int koff[F::kLoads], voff[F::kLoads];
#pragma unroll
  for (int i = 0; i < F::kLoads; ++i) {
    const int r = R::kPerLoad * i + lane / R::kChunks;
    koff[i] = r * R::kBytes + (((lane % R::kChunks) ^ R::swizzle_k(r)) << 4);
    voff[i] = r * R::kBytes + (((lane % R::kChunks) ^ R::swizzle_v(r)) << 4);
  }
  const Groups groups(a.pages, a.B, a.heads, at.request, head);
  const v4i32 pbuf = make_buffer(a.pos + static_cast<size_t>(u) * a.B, WINDOW ? static_cast<uint32_t>(n) * 4u : 0u);
  const int64_t new_byte = static_cast<int64_t>(at.first) * a.kv_stride + static_cast<int64_t>(head) * R::kBytes;
  const int more_stride = static_cast<int>(a.kv_stride) - R::kBytes;  // of the chunk's rows
  int page_ahead = 0;
  const auto look_ahead = [&](int t) {
    if (t < min(t1, cache_stages)) page_ahead = __builtin_amdgcn_readfirstlane(groups.page_of(min(t * 64 + 16 * wave, n - 1)));
  };
  struct Place { int64_t byte; int count; };  // of the first of the rows, in the caches or the chunk's arrays; how many there are
  const auto request_k = [&](int t) {
    const int slot = t * 64 + 16 * wave;
    Place p;
    if (t < cache_stages) {
      uint32_t r;
      p.count = __builtin_amdgcn_readfirstlane(min(max((t < t1 ? n : 0) - slot, 0), 16));
      if (!groups.row_of(slot, page_ahead, r)) p.count = 0;
      p.byte = static_cast<int64_t>(p.count > 0 ? r : 0u) * R::kBytes;
      look_ahead(t + 1);
    } else {
      const int j = slot - cache_stages * 64;
      p.count = __builtin_amdgcn_readfirstlane(min(max((t < t1 ? at.count : 0) - j, 0), 16));
      p.byte = new_byte + static_cast<int64_t>(p.count > 0 ? j : 0) * a.kv_stride;
    }
    there_s[t & (kSide - 1)][wave] = p.count;
    return p;
  };
  struct Request { v4i32 buf; uint32_t dst; int more; };
  const int lane_row = lane / R::kChunks;
  const auto request_rows = [&](auto of_v, int t, const Place& p) {
    constexpr bool kOfV = decltype(of_v)::value;
    Request r;
    const bool of_new = t >= cache_stages;
    const char* const base = static_cast<const char*>(kOfV ? (of_new ? a.v_new : a.V) : (of_new ? a.k_new : a.K)) + p.byte;
    r.dst = ring_addr + ((kOfV ? NR : 0) + (t & (NR - 1))) * F::kOperand;
    r.more = of_new ? more_stride : 0;
    r.buf = make_buffer(base, p.count > 0 ? static_cast<uint32_t>(p.count - 1) * static_cast<uint32_t>(R::kBytes + r.more) + R::kBytes : 0u);
    return r;
  };
  const auto request_load = [&](auto of_v, const Request& r, int i) {
    load16_to_lds(r.buf, r.dst + i * 1024, (decltype(of_v)::value ? voff[i] : koff[i]) + (lane_row + R::kPerLoad * i) * r.more, 0);
  };
  // Step t takes K of the stages t and t + 1 and V of t - 1 and t; it asks for K of t + NR - 1 and V of t + NR - 2, the loads one by one between its matrix
  // instructions.  (Stages behind the last one have no rows: what is asked for then are zeros, and every step asks for as many loads.)
  Place newest = {0, 0}, before = {0, 0};
  Request pending;
  const auto side_k = [&](int t, int i) {  // K of stage t, in parts i = 0 .. kLoads
    if (i == 0) {
      before = newest;
      newest = request_k(t);
      pending = request_rows(std::false_type(), t, newest);
      // (a wave-wide load of the stage's 64 positions; behind the unit's last slot, and for the chunk's tokens, zeros)
      if (WINDOW)
        mfma::load4_to_lds(pbuf, lds_address(&pos_s[WINDOW ? wave : 0][WINDOW ? t & (kSide - 1) : 0][0]), t >= cache_stages ? 0x7ffffffc : (t * 64 + lane) * 4, 0);
    } else if (i <= F::kLoads) {
      request_load(std::false_type(), pending, i - 1);
    }
  };
  const auto side_v = [&](int t, int i) {  // V of stage t, whose K was the one before
    if (i == 0) pending = request_rows(std::true_type(), t, before);
    else if (i <= F::kLoads) request_load(std::true_type(), pending, i - 1);
  };
  look_ahead(t0);
#pragma unroll 1
  for (int t = t0; t < t0 + NR - 1; ++t) {
#pragma unroll
    for (int i = 0; i <= F::kLoads; ++i) side_k(t, i);
#pragma unroll
    for (int i = 0; i <= F::kLoads && t > t0; ++i) side_v(t - 1, i);
  }

  // ---- the wave's query rows
  const int wave_row = first_row + 32 * NG * wave;
  int row[NG], token[NG];
  Frag own[NG][R::kSteps];
  take_rows<DT, HD, NG>(a, mine, wave_row, row, token, own);
  const int wave_first = __builtin_amdgcn_readfirstlane(token[0]);                           // tokens of the wave's rows
  const int wave_last = __builtin_amdgcn_readfirstlane((min(rows, wave_row + 32 * NG) - 1) / a.group);
  const int tile_first = __builtin_amdgcn_readfirstlane(first_row / a.group);                // first of the row tile's
  const bool idle = wave_row >= rows;
  // half stages up to here hold something that the wave's rows see
  const int end = idle ? 0 : min(2 * t1, 2 * cache_stages + wave_last / kSub + 1);
  float m[NG], l[NG];
  f32x16 o[NG][R::kBlocks];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.0f;
#pragma unroll
    for (int db = 0; db < R::kBlocks; ++db) o[g][db] = f32x16{0};
  }
  const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f;
  const int w = WINDOW ? a.recency_window : 0, qp0 = WINDOW ? a.qpos0[at.request] : 0;
  // fragment reads: K row lane % 32, chunk 2 kk + half (stages lie at multiples of 1 KiB: the step is an exclusive or of the address); V transposed, rows
  // 4 half + lane % 16 / 4 (+ 8), 8 bytes of columns 32 db + 16 (lane / 16 % 2) + 4 (lane % 4)
  const uint32_t kfrag = lds_address(ring) + (lane & 31) * R::kBytes + ((half ^ R::swizzle_k(lane & 31)) << 4);
  const int vrow = 4 * half + ((lane & 15) >> 2);
  const uint32_t vfrag = lds_address(ring) + NR * F::kOperand + vrow * R::kBytes + (R::swizzle_v(vrow) << 4) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  int zeroed = 0x7fffffff;  // the first of the chunk's tokens whose value may have been taken out (see below)

  struct Probabilities { Frag b[2]; };  // rounded to bf16, two in a register
  const auto put2 = [&](Probabilities& p, int e, float v0, float v1) {  // (e is even)
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    p.b[e >> 3][(e >> 1) & 3] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(v0), static_cast<__bf16>(v1)});
  };
  const auto read_v = [&](uint32_t vt, int part) {  // of 16 keys and 32 dimensions
    const uint32_t v_at = (vt ^ (part % R::kBlocks << 6)) + part / R::kBlocks * 16 * R::kBytes;
    return read_frag_transposed(v_at, v_at + 8 * R::kBytes);
  };
  // A half step at half stage c: scores s of it, to probabilities p; scores s_next of half stage c + 1; products with p_before and V of c - 1.  (What a first or a
  // last one has not got it computes all the same, from whatever lies in LDS: other paths would have the outputs in other registers, and copies
  // where they meet.)
  // The first fragments have been read by the half step before (kf, vf); side(i) is the part of the requests that comes beside the i-th matrix instructions.
  constexpr int kSlots = R::kSteps, kEach = 16 / kSlots, kEarly = 2;
  static_assert(kSlots == 2 * R::kBlocks && kSlots >= F::kLoads + 1, "as many instructions of the one kind as of the other");
  Frag k_early[kEarly], v_early[kEarly];
  const auto k_addr = [&](int c) { return kfrag + ((c >> 1) & (NR - 1)) * F::kOperand + (c & 1) * (kSub * R::kBytes); };
  const auto v_addr = [&](int c) { return vfrag + ((c >> 1) & (NR - 1)) * F::kOperand + (c & 1) * (kSub * R::kBytes); };
  const auto read_early = [&](int c, int i) {  // for half step c
    k_early[i] = read_frag(k_addr(c + 1) ^ (i << 5));
    v_early[i] = read_v(v_addr(c - 1), i);
  };
  const auto half_step = [&](int c, bool full, f32x16 (&s)[NG], f32x16 (&s_next)[NG], Probabilities (&p)[NG], const Probabilities (&p_before)[NG], auto side) {
    const int t = c >> 1, h = c & 1;
    const bool of_new = t >= cache_stages;
    const int j0 = (c - 2 * cache_stages) * kSub;  // the first token
    const int32_t* const pos_c = &pos_s[WINDOW ? wave : 0][WINDOW ? t & (kSide - 1) : 0][kSub * h];
    bool interior = of_new ? w <= wave_first - (j0 + kSub - 1) : full;  // (in this order: w may be the largest number)
    if (WINDOW && !of_new) {  // outside the window of every row
      const int at_slot = pos_c[lane & 31];
      interior = interior && !__any(at_slot <= qp0 + wave_last && at_slot > qp0 + wave_first - w);
    }
    // The reference need not be the running maximum: the terms are taken against it as it stands, and only a tile whose sum leaves the safe
    // range -- the first one, whose reference is -inf, and scores that rise by more than 16 powers of two -- raises it below.
    float sum[NG], neg[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      sum[g] = 0.0f;
      neg[g] = -m[g];
      s_next[g] = f32x16{0};
    }
    const uint32_t k_at = k_addr(c + 1), vt = v_addr(c - 1);
    Frag kf[kSlots], vf[kSlots];
#pragma unroll
    for (int i = 0; i < kEarly; ++i) {
      kf[i] = k_early[i];
      vf[i] = v_early[i];
    }
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      if (i + kEarly < kSlots) {
        kf[i + kEarly] = read_frag(k_at ^ ((i + kEarly) << 5));
        vf[i + kEarly] = read_v(vt, i + kEarly);
      } else {
        read_early(c + 1, i + kEarly - kSlots);
      }
      side(i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        s_next[g] = score_step<DT>(kf[i], own[g][i], s_next[g]);
        __builtin_amdgcn_sched_barrier(0);
        float v[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          v[e] = fast_exp2(fmaf(s[g][kEach * i + e], sc, neg[g]));
          asm volatile("" : "+v"(v[e]));  // (without a use here the compiler forms them where they are first needed, behind the last product)
        }
        __builtin_amdgcn_sched_barrier(0);
        add_product(o[g][i % R::kBlocks], vf[i], p_before[g].b[i / R::kBlocks]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < kEach; e += 2) {
          put2(p[g], kEach * i + e, v[e], v[e + 1]);
          sum[g] += v[e];
          sum[g] += v[e + 1];
          asm volatile("" : "+v"(sum[g]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (c == 2 * t0) {
      settled(o);
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db) o[g][db] = f32x16{0};
    }
    bool again = !interior;
#pragma unroll
    for (int g = 0; g < NG; ++g) again = again || __builtin_amdgcn_ballot_w64(!(sum[g] <= 0x1p16f)) != 0;
    if (again && c < end) {
      settled(o);
      const int4 here = *reinterpret_cast<const int4*>(there_s[t & (kSide - 1)]);
      const int there[2] = {h == 0 ? here.x : here.z, h == 0 ? here.y : here.w};
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x = s[g][e] * sc;
          if (!interior) {
            const int k = 8 * (e >> 2) + 4 * half + (e & 3);  // of the 32 keys
            if (WINDOW) {
              const int away = qp0 + token[g] - (of_new ? qp0 + j0 + k : pos_c[k]);
              x += static_cast<unsigned>(away) < static_cast<unsigned>(w) ? bias : 0.0f;
            }
            const bool seen = of_new ? j0 + k <= token[g] : (k & 15) < there[e >> 3];
            x = seen ? x : -INFINITY;
          }
          s[g][e] = x;
          most = fmaxf(most, x);
        }
        most = fmaxf(most, __shfl_xor(most, 32, kWave));  // the two halves feed one product
        const float m_new = fmaxf(m[g], most);
        if (__any(m_new > m[g])) {
          const float alpha = m[g] > -INFINITY ? fast_exp2(m[g] - m_new) : 0.0f;
          l[g] *= alpha;
#pragma unroll
          for (int db = 0; db < R::kBlocks; ++db) o[g][db] *= alpha;
        }
        m[g] = m_new;
        const float ref = m_new > -INFINITY ? m_new : 0.0f;  // nothing seen yet: every term is 2^-inf = 0
        sum[g] = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float v0 = fast_exp2(s[g][e] - ref), v1 = fast_exp2(s[g][e + 1] - ref);
          put2(p[g], e, v0, v1);
          sum[g] += v0;
          sum[g] += v1;
        }
      }
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      if (c < end) l[g] += sum[g];
      else p[g].b[0] = p[g].b[1] = Frag{0, 0, 0, 0};  // behind the wave's last half stage
    }
  };
  // Some row of the tile does not see all of the chunk's tokens in a stage.  A value that is infinite or NaN must not reach the rows that do not see its
  // token, and 0 times it would: such rows of V are zero in the products, and added in the end to the rows that see them.
  const auto take_out = [&](int t) {
    const int j0 = (t - cache_stages) * 64;
    if (t >= t1 || j0 < 0 || j0 + 63 <= tile_first) return;
    char* const tileV = ring + (NR + (t & (NR - 1))) * F::kOperand;
    bool any = false;
#pragma unroll 2
    for (int i = 0; i < F::kOperand / 1024; ++i) any |= holds_special<DT>(*reinterpret_cast<const uint4*>(tileV + i * 1024 + lane * 16));
    if (!__any(any)) return;  // (all waves look at the same rows)
    zeroed = min(zeroed, j0);
    __syncthreads();
#pragma unroll 1
    for (int j = 16 * wave; j < 16 * wave + 16; ++j) {
      uint4* const chunk = reinterpret_cast<uint4*>(tileV + j * R::kBytes) + lane % R::kChunks;
      if (__any(holds_special<DT>(*chunk))) *chunk = make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
  };
  // The queries must have arrived before the loop: a wait for them inside it would also wait for the stages requested last.
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();                     // all waves' shares of the first stages are there
  const auto next_step = [&](int t) {
    // K of stage t + 1 and V of stage t are wanted; what was asked for in the step before may still be on its way
    wait_loads<kStageLoads>();
    __syncthreads();  // the other waves' shares are there too, and everybody has done with the step before
    take_out(t);
  };
  if (2 * t0 >= end) {  // nothing that this wave's rows see, but the other waves want its loads
#pragma unroll 1
    for (int t = t0; t <= t1; ++t) {
      next_step(t);
#pragma unroll
      for (int i = 0; i <= F::kLoads; ++i) side_k(t + NR - 1, i);
#pragma unroll
      for (int i = 0; i <= F::kLoads; ++i) side_v(t + NR - 2, i);
    }
  } else {
    f32x16 s0[NG], s1[NG];
    Probabilities p0[NG], p1[NG];
    const uint32_t k_at = kfrag + (t0 & (NR - 1)) * F::kOperand;
#pragma unroll
    for (int g = 0; g < NG; ++g) s0[g] = f32x16{0};
#pragma unroll
    for (int kk = 0; kk < R::kSteps; ++kk) {
      const Frag k = read_frag(k_at ^ (kk << 5));
#pragma unroll
      for (int g = 0; g < NG; ++g) s0[g] = score_step<DT>(k, own[g][kk], s0[g]);
    }
#pragma unroll
    for (int i = 0; i < kEarly; ++i) read_early(2 * t0, i);
#pragma unroll 1
    for (int t = t0; t <= t1; ++t) {
      next_step(t);
      const int4 here = *reinterpret_cast<const int4*>(there_s[t & (kSide - 1)]);
      const bool full = (__builtin_amdgcn_readfirstlane(here.x & here.y & here.z & here.w) & 16) != 0;
      half_step(2 * t, full, s0, s1, p0, p1, [&](int i) { side_k(t + NR - 1, i); });
      half_step(2 * t + 1, full, s1, s0, p1, p0, [&](int i) { side_v(t + NR - 2, i); });
    }
    settled(o);
  }
  wait_loads<0>();
  if (!idle) Finish<DT, HD, NG, WINDOW>::run(a, mine, plan.used, row, token, own, m, l, o, zeroed, min((t1 - cache_stages) * 64 - 1, wave_last));
}

// 32 rows of a wave, 32 keys of a stage, one after the other, and as many waves as there is room for.
// Measured: 24 requests, of which 18 decode a token and the others take 384 or fewer, 8 heads of 4 queries, over 4096 keys or fewer, 140 us (156 with as many
// shares for short requests as for long ones); 6 of up to 333 tokens over 2048, 12 heads, 64 dimensions, with a recency window, 40 us (45 with the
// window looked for in every score).
template <int DT, int HD> struct TileForm {
  using R = Rows<DT, HD>;
  static constexpr int kTileBytes = kSub * R::kBytes;             // of K, then as many of V
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kStages = kStageBytes > 16384 ? 2 : DT == kBF16 && HD == 128 ? 3 : 4;
  static constexpr int kBytes = kStages * kStageBytes;
  static constexpr int kAhead = kStages - 1;                      // stages that are asked for before their turn
  static constexpr int kLoads = 8 * R::kBytes / 1024;             // of a wave, for its eight rows of K or of V
  static constexpr int kWavesPerSimd = DT == kF32 ? 2 : HD == 128 ? 3 : 4;
};

template <int DT, int HD, bool WINDOW>
__global__ __launch_bounds__(kThreads, (TileForm<DT, HD>::kWavesPerSimd)) void chunk_attend(ChunkArgs a) {
  using R = Rows<DT, HD>;
  using F = TileForm<DT, HD>;
  constexpr int kSide = WINDOW ? 1 : 0;  // the positions of a tile's slots come along
  constexpr int kTileLoads = 2 * F::kLoads + kSide;
  extern __shared__ __attribute__((aligned(1024))) char ring[];
  __shared__ __attribute__((aligned(256))) int32_t pos_s[WINDOW ? kWaves : 1][WINDOW ? F::kStages : 1][kWave];
  RowTile mine;
  if (!my_tile<128>(a, mine)) return;
  const Located& at = mine.at;
  const int head = mine.head, first_row = mine.first_row, rows = first_row + mine.rows;
  const int u = at.request * a.heads + head;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int half = lane >> 5;
  const Plan<DT, 128, kSub> plan(a, mine);
  const int n = plan.n, cache_tiles = plan.cache_stages;
  const int t0 = mine.split * plan.per, t1 = min(plan.stages, t0 + plan.per);
  if (t0 >= t1) return;
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
  const int64_t new_byte = static_cast<int64_t>(at.first) * a.kv_stride + static_cast<int64_t>(head) * R::kBytes;
  const int more_stride = static_cast<int>(a.kv_stride) - R::kBytes;  // of the chunk's rows
  int ahead[2] = {0, 0};  // pages of the two groups of the tile that is asked for next
  const auto look_ahead = [&](int t) {
    if (t >= min(t1, cache_tiles)) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) ahead[i] = __builtin_amdgcn_readfirstlane(groups.page_of(min(t * kSub + 16 * i, n - 1)));
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
        const int slot = t * kSub + 16 * i;
        uint32_t r;
        int count = __builtin_amdgcn_readfirstlane(min(max(n - slot, 0), 16));
        if (!groups.row_of(slot, ahead[i], r)) count = 0;
        there |= static_cast<uint32_t>(count) << (8 * i);
        if (i == wave >> 1) row_at = count > 0 ? r : 0u;
      }
      const uint32_t here = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(min(max(static_cast<int>((there >> (8 * (wave >> 1))) & 0xffu) - sub, 0), 8)));
      const size_t byte = static_cast<size_t>(row_at + (here > 0 ? sub : 0)) * R::kBytes;
      const v4i32 kbuf = make_buffer(static_cast<const char*>(a.K) + byte, here * R::kBytes), vbuf = make_buffer(static_cast<const char*>(a.V) + byte, here * R::kBytes);
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) load16_to_lds(kbuf, dst + i * 1024, koff[i], 0);
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) load16_to_lds(vbuf, dst + F::kTileBytes + i * 1024, voff[i], 0);
      look_ahead(t + 1);
    } else {
      const int j = (t - cache_tiles) * kSub + 8 * wave, here = __builtin_amdgcn_readfirstlane(min(max(at.count - j, 0), 8));
      const int64_t byte = new_byte + static_cast<int64_t>(here > 0 ? j : 0) * a.kv_stride;
      const uint32_t size = here > 0 ? static_cast<uint32_t>(here - 1) * static_cast<uint32_t>(a.kv_stride) + R::kBytes : 0u;
      const v4i32 kbuf = make_buffer(static_cast<const char*>(a.k_new) + byte, size), vbuf = make_buffer(static_cast<const char*>(a.v_new) + byte, size);
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) {
        const int more = (R::kPerLoad * i + lane / R::kChunks) * more_stride;
        load16_to_lds(kbuf, dst + i * 1024, koff[i] + more, 0);
        load16_to_lds(vbuf, dst + F::kTileBytes + i * 1024, voff[i] + more, 0);
      }
    }
    // (a wave-wide load of 64 words; behind the unit's last slot, and for the chunk's tokens, zeros)
    if (WINDOW) mfma::load4_to_lds(pbuf, pos_addr + stage * (kWave * 4), t < cache_tiles ? (t * kSub + lane) * 4 : 0x7ffffffc, 0);
    return there;
  };
  uint32_t there[F::kStages];  // of the tile in use and those behind it
  look_ahead(t0);
#pragma unroll
  for (int i = 0; i < F::kAhead; ++i) there[i] = t0 + i < t1 ? request(t0 + i, i) : 0u;

  const int wave_row = first_row + 32 * wave;
  int row[1], token[1];
  Frag own[1][R::kSteps];
  take_rows<DT, HD, 1>(a, mine, wave_row, row, token, own);
  const int wave_first = __builtin_amdgcn_readfirstlane(token[0]);
  const int wave_last = __builtin_amdgcn_readfirstlane((min(rows, wave_row + 32) - 1) / a.group);
  const int tile_first = __builtin_amdgcn_readfirstlane(first_row / a.group);
  const bool idle = wave_row >= rows;
  float m[1] = {-INFINITY}, l[1] = {0.0f};
  f32x16 o[1][R::kBlocks];
#pragma unroll
  for (int db = 0; db < R::kBlocks; ++db) o[0][db] = f32x16{0};
  const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f;
  const int w = a.recency_window, qp0 = WINDOW ? a.qpos0[at.request] : 0;
  // fragment reads: K row lane % 32, chunk 2 kk + half; V of fp32 row 4 half (+ e + 8 i), column 32 db + lane % 32, of bf16 as in chunk_attend_pair
  const uint32_t kfrag = (lane & 31) * R::kBytes + ((half ^ R::swizzle_k(lane & 31)) << 4);
  const int vrow = 4 * half + (DT == kBF16 ? (lane & 15) >> 2 : 0);
  const uint32_t vfrag = F::kTileBytes + vrow * R::kBytes + (R::swizzle_v(vrow) << 4) + (DT == kBF16 ? ((lane >> 4) & 1) * 32 + (lane & 3) * 8 : (lane & 31) * 4);
  int zeroed = 0x7fffffff;  // (see chunk_attend_pair)
  // The queries must have arrived before the loop: a wait for them inside it would also wait for the tiles requested last.
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  int stage = 0;
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    if (t + F::kAhead - 1 < t1) wait_loads<(F::kAhead - 1) * kTileLoads>();  // the tiles behind it may still be on their way
    else wait_loads<0>();
    __syncthreads();  // tile t is in LDS, and everybody has issued its last read of tile t - 1
    const uint32_t here = there[0];
#pragma unroll
    for (int i = 0; i + 1 < F::kAhead; ++i) there[i] = there[i + 1];
    there[F::kAhead - 1] = t + F::kAhead < t1 ? request(t + F::kAhead, stage == 0 ? F::kAhead : stage - 1) : 0u;
    const uint32_t st = ring_addr + stage * F::kStageBytes;
    const int32_t* const pos_t = &pos_s[WINDOW ? wave : 0][WINDOW ? stage : 0][0];
    stage = stage + 1 == F::kStages ? 0 : stage + 1;
    const bool of_new = t >= cache_tiles;
    const int j0 = (t - cache_tiles) * kSub;  // the tile's first token
    if (of_new && j0 + kSub - 1 > tile_first) {  // (as take_out of chunk_attend_pair)
      char* const tileV = ring + (st - ring_addr) + F::kTileBytes;
      bool any = false;
#pragma unroll 2
      for (int i = 0; i < F::kTileBytes / 1024; ++i) any |= holds_special<DT>(*reinterpret_cast<const uint4*>(tileV + i * 1024 + lane * 16));
      if (__any(any)) {
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
    f32x16 s = {0};
#pragma unroll
    for (int kk = 0; kk < R::kSteps; ++kk) s = score_step<DT>(read_frag((st + kfrag) ^ (kk << 5)), own[0][kk], s);
    bool interior = of_new ? (WINDOW ? w : 0) <= wave_first - (j0 + kSub - 1) : here == 0x1010u;
    if (WINDOW && !of_new) {  // outside the window of every row
      const int at_slot = pos_t[lane & 31];
      interior = interior && !__any(at_slot <= qp0 + wave_last && at_slot > qp0 + wave_first - w);
    }
    float sum = 0.0f;
    bool done = false;
    float p[16];  // the probabilities, of bf16 rounded to bf16
    bf16x8 pf[2];
    const auto keep = [&](int e, float v) {
      if (DT == kBF16) pf[e >> 3][e & 7] = static_cast<__bf16>(v);
      else p[e] = v;
      sum += v;
    };
    if (interior) {
      // The reference need not be the running maximum: the terms are taken against it as it stands, and only a tile whose sum leaves the safe
      // range -- the first one, whose reference is -inf, and scores that rise by more than 16 powers of two -- raises it below.
      const float neg = -m[0];
#pragma unroll
      for (int e = 0; e < 16; ++e) keep(e, fast_exp2(fmaf(s[e], sc, neg)));
      done = __builtin_amdgcn_ballot_w64(!(sum <= 0x1p16f)) == 0;
    }
    if (!done) {
      float most = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x = s[e] * sc;
        if (!interior) {
          const int k = 8 * (e >> 2) + 4 * half + (e & 3);  // of the tile's keys
          if (WINDOW) {
            const int away = qp0 + token[0] - (of_new ? qp0 + j0 + k : pos_t[k]);
            x += static_cast<unsigned>(away) < static_cast<unsigned>(w) ? bias : 0.0f;
          }
          const bool seen = of_new ? j0 + k <= token[0] : (k & 15) < static_cast<int>((here >> (k & 16 ? 8 : 0)) & 0xffu);
          x = seen ? x : -INFINITY;
        }
        s[e] = x;
        most = fmaxf(most, x);
      }
      most = fmaxf(most, __shfl_xor(most, 32, kWave));  // the two halves feed one product
      const float m_new = fmaxf(m[0], most);
      if (__any(m_new > m[0])) {
        const float alpha = m[0] > -INFINITY ? fast_exp2(m[0] - m_new) : 0.0f;
        l[0] *= alpha;
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db) o[0][db] *= alpha;
      }
      m[0] = m_new;
      const float ref = m_new > -INFINITY ? m_new : 0.0f;  // nothing seen yet: every term is 2^-inf = 0
      sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; ++e) keep(e, fast_exp2(s[e] - ref));
    }
    l[0] += sum;
    const uint32_t vt = st + vfrag;
    if constexpr (DT == kBF16) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db) {
          const uint32_t v_at = (vt ^ (db << 6)) + ks * 16 * R::kBytes;
          o[0][db] = score_step<DT>(read_frag_transposed(v_at, v_at + 8 * R::kBytes), __builtin_bit_cast(Frag, pf[ks]), o[0][db]);
        }
    } else {
      typedef const __attribute__((address_space(3))) float* LdsFloats;
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db) {
          const float v = *(LdsFloats)(static_cast<uintptr_t>((vt ^ (db << 7)) + (8 * (e >> 2) + (e & 3)) * R::kBytes));
          o[0][db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[e], o[0][db], 0, 0, 0);
        }
    }
  }
  if (!idle) Finish<DT, HD, 1, WINDOW>::run(a, mine, plan.used, row, token, own, m, l, o, zeroed, min((t1 - cache_tiles) * kSub - 1, wave_last));
}

// One to 32 rows of a request: four waves that share them, each with a quarter of the workgroup's keys, tiles of its own and no barrier until their shares are joined
// in LDS.  A tile's K is asked for as soon as the scores of the one before are formed, its V after that one's products.
// Measured: a token of 32 requests, 8 heads of 4 queries, over 4096 keys each, bf16 / 128, 103 us (5.2 TB/s); of 8 heads of one over 2048, fp32 / 128, 104 us (5.2 TB/s; with
// tiles of 128 rows, three waves of four without any, 286); fp32, 5 of up to 101 tokens over 1501, 5 heads of 3 queries, 70 us; 4 that decode a token over 500, 4 heads, 64
// dimensions, 14 us.
template <int DT, int HD> struct FewForm {
  using R = Rows<DT, HD>;
  static constexpr int kOperand = kSub * R::kBytes, kWaveBytes = 2 * kOperand, kBytes = kWaves * kWaveBytes;
  static constexpr int kLoads = kOperand / 1024;                  // of a tile's K, or V
  static constexpr int kWavesPerSimd = kBytes > 65536 ? 1 : kBytes > 32768 ? 2 : 4;
};

template <int DT, int HD, bool WINDOW>
__global__ __launch_bounds__(kThreads, (FewForm<DT, HD>::kWavesPerSimd)) void chunk_attend_few(ChunkArgs a) {
  using R = Rows<DT, HD>;
  using F = FewForm<DT, HD>;
  constexpr int kSide = WINDOW ? 1 : 0;
  extern __shared__ __attribute__((aligned(1024))) char ring[];
  __shared__ __attribute__((aligned(256))) int32_t pos_s[WINDOW ? kWaves : 1][WINDOW ? 2 : 1][kWave];
  __shared__ float m_s[kWaves][kWave], l_s[kWaves][kWave];
  RowTile mine;
  if (!my_tile<32>(a, mine)) return;
  const Located& at = mine.at;
  const int head = mine.head, first_row = mine.first_row, rows = first_row + mine.rows;
  const int u = at.request * a.heads + head;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int half = lane >> 5;
  const Plan<DT, 32, kSub> plan(a, mine);
  const int n = plan.n, cache_tiles = plan.cache_stages;
  const int first_tile = mine.split * plan.per, last_tile = min(plan.stages, first_tile + plan.per);
  if (first_tile >= last_tile) return;
  const int each = (last_tile - first_tile + kWaves - 1) / kWaves;
  const int t0 = __builtin_amdgcn_readfirstlane(min(last_tile, first_tile + wave * each)), t1 = __builtin_amdgcn_readfirstlane(min(last_tile, t0 + each));
  const Groups groups(a.pages, a.B, a.heads, at.request, head);
  char* const my_lds = ring + wave * F::kWaveBytes;
  const uint32_t lds = lds_address(my_lds), pos_addr = lds_address(&pos_s[WINDOW ? wave : 0][0][0]);
  int koff[F::kLoads], voff[F::kLoads];
#pragma unroll
  for (int i = 0; i < F::kLoads; ++i) {
    const int r = R::kPerLoad * i + lane / R::kChunks;
    koff[i] = r * R::kBytes + (((lane % R::kChunks) ^ R::swizzle_k(r)) << 4);
    voff[i] = r * R::kBytes + (((lane % R::kChunks) ^ R::swizzle_v(r)) << 4);
  }
  const v4i32 pbuf = make_buffer(a.pos + static_cast<size_t>(u) * a.B, WINDOW ? static_cast<uint32_t>(n) * 4u : 0u);
  const int64_t new_byte = static_cast<int64_t>(at.first) * a.kv_stride + static_cast<int64_t>(head) * R::kBytes;
  const int more_stride = static_cast<int>(a.kv_stride) - R::kBytes;
  int ahead[2] = {0, 0};  // pages of the two groups of the tile that is asked for next
  const auto look_ahead = [&](int t) {
    if (t >= min(t1, cache_tiles)) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) ahead[i] = __builtin_amdgcn_readfirstlane(groups.page_of(min(t * kSub + 16 * i, n - 1)));
  };
  // A tile's place: rows of the cache, 16 of a page each, or of the chunk, side by side but for the stride.
  struct Place { uint32_t row[2]; int count[2]; };
  const auto place_of = [&](int t) {
    Place p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (t < cache_tiles) {
        const int slot = t * kSub + 16 * i;
        p.count[i] = __builtin_amdgcn_readfirstlane(min(max(n - slot, 0), 16));
        if (!groups.row_of(slot, ahead[i], p.row[i])) p.count[i] = 0;
        if (p.count[i] == 0) p.row[i] = 0;
      } else {
        const int j = (t - cache_tiles) * kSub + 16 * i;
        p.count[i] = __builtin_amdgcn_readfirstlane(min(max(at.count - j, 0), 16));
        p.row[i] = static_cast<uint32_t>(p.count[i] > 0 ? j : 0);
      }
    }
    return p;
  };
  const auto request = [&](auto of_v, int t, const Place& p) {
    constexpr bool kOfV = decltype(of_v)::value;
    const bool of_new = t >= cache_tiles;
    const char* const base = static_cast<const char*>(kOfV ? (of_new ? a.v_new : a.V) : (of_new ? a.k_new : a.K));
    const int more = of_new ? more_stride : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const char* const from = base + (of_new ? new_byte + static_cast<int64_t>(p.row[i]) * a.kv_stride : static_cast<int64_t>(p.row[i]) * R::kBytes);
      const v4i32 buf = make_buffer(from, p.count[i] > 0 ? static_cast<uint32_t>(p.count[i] - 1) * static_cast<uint32_t>(R::kBytes + more) + R::kBytes : 0u);
#pragma unroll
      for (int k = 0; k < F::kLoads / 2; ++k) {
        const int at_load = i * (F::kLoads / 2) + k;
        // (a group's offsets begin at its first row: 16 rows are whole loads, and the swizzles repeat)
        load16_to_lds(buf, lds + (kOfV ? F::kOperand : 0) + at_load * 1024, (kOfV ? voff[at_load] : koff[at_load]) - 16 * i * R::kBytes + (R::kPerLoad * k + lane / R::kChunks) * more, 0);
      }
    }
  };
  const auto request_k = [&](int t, const Place& p) {
    if (WINDOW) mfma::load4_to_lds(pbuf, pos_addr + (t & 1) * (kWave * 4), t < cache_tiles ? (t * kSub + lane) * 4 : 0x7ffffffc, 0);
    request(std::false_type(), t, p);
  };
  const auto reads_done = [&]() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };  // what is overwritten next has been read
  int row[1], token[1];
  Frag own[1][R::kSteps];
  look_ahead(t0);
  take_rows<DT, HD, 1>(a, mine, first_row, row, token, own);
  const int rows_first = __builtin_amdgcn_readfirstlane(first_row / a.group), rows_last = __builtin_amdgcn_readfirstlane((rows - 1) / a.group);
  float m[1] = {-INFINITY}, l[1] = {0.0f};
  f32x16 o[1][R::kBlocks];
#pragma unroll
  for (int db = 0; db < R::kBlocks; ++db) o[0][db] = f32x16{0};
  const float sc = a.scale_log2, bias = WINDOW ? a.recency_bias_log2 : 0.0f;
  const int w = WINDOW ? a.recency_window : 0, qp0 = WINDOW ? a.qpos0[at.request] : 0;
  const uint32_t kfrag = lds + (lane & 31) * R::kBytes + ((half ^ R::swizzle_k(lane & 31)) << 4);
  const int vrow = 4 * half + (DT == kBF16 ? (lane & 15) >> 2 : 0);
  const uint32_t vt = lds + F::kOperand + vrow * R::kBytes + (R::swizzle_v(vrow) << 4) + (DT == kBF16 ? ((lane >> 4) & 1) * 32 + (lane & 3) * 8 : (lane & 31) * 4);
  int zeroed = 0x7fffffff;
  // (the queries have arrived: a wait for them below would also wait for the tiles requested last)
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  Place here = {{0, 0}, {0, 0}};
  if (t0 < t1) {
    here = place_of(t0);
    request_k(t0, here);
    request(std::true_type(), t0, here);
    look_ahead(t0 + 1);
  }
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    const bool of_new = t >= cache_tiles, more_tiles = t + 1 < t1;
    const int j0 = (t - cache_tiles) * kSub;
    const int there[2] = {here.count[0], here.count[1]};
    wait_loads<F::kLoads>();  // K is there; V may still be on its way
    f32x16 s = {0};
#pragma unroll
    for (int kk = 0; kk < R::kSteps; ++kk) s = score_step<DT>(read_frag(kfrag ^ (kk << 5)), own[0][kk], s);
    reads_done();
    if (more_tiles) {
      here = place_of(t + 1);
      request_k(t + 1, here);
      look_ahead(t + 2);
    }
    const int32_t* const pos_t = &pos_s[WINDOW ? wave : 0][WINDOW ? t & 1 : 0][0];
    bool interior = of_new ? w <= rows_first - (j0 + kSub - 1) : there[0] + there[1] == kSub;
    if (WINDOW && !of_new) {  // outside the window of every row
      const int at_slot = pos_t[lane & 31];
      interior = interior && !__any(at_slot <= qp0 + rows_last && at_slot > qp0 + rows_first - w);
    }
    float most = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float x = s[e] * sc;
      if (!interior) {
        const int k = 8 * (e >> 2) + 4 * half + (e & 3);
        if (WINDOW) {
          const int away = qp0 + token[0] - (of_new ? qp0 + j0 + k : pos_t[k]);
          x += static_cast<unsigned>(away) < static_cast<unsigned>(w) ? bias : 0.0f;
        }
        const bool seen = of_new ? j0 + k <= token[0] : (k & 15) < there[e >> 3];
        x = seen ? x : -INFINITY;
      }
      s[e] = x;
      most = fmaxf(most, x);
    }
    most = fmaxf(most, __shfl_xor(most, 32, kWave));
    const float m_new = fmaxf(m[0], most);
    if (__any(m_new > m[0])) {
      const float alpha = m[0] > -INFINITY ? fast_exp2(m[0] - m_new) : 0.0f;
      l[0] *= alpha;
#pragma unroll
      for (int db = 0; db < R::kBlocks; ++db) o[0][db] *= alpha;
    }
    m[0] = m_new;
    const float ref = m_new > -INFINITY ? m_new : 0.0f;  // nothing seen yet: every term is 2^-inf = 0
    float p[16];
    bf16x8 pf[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float v = fast_exp2(s[e] - ref);
      if (DT == kBF16) pf[e >> 3][e & 7] = static_cast<__bf16>(v);
      else p[e] = v;
      l[0] += v;
    }
    if (more_tiles) wait_loads<F::kLoads + kSide>();  // V is there; K of the next tile may still be on its way
    else wait_loads<0>();
    if (of_new && j0 + kSub - 1 > rows_first) {  // (as take_out of chunk_attend_pair)
      char* const tileV = my_lds + F::kOperand;
      bool any = false;
#pragma unroll 2
      for (int i = 0; i < F::kLoads; ++i) any |= holds_special<DT>(*reinterpret_cast<const uint4*>(tileV + i * 1024 + lane * 16));
      if (__any(any)) {
        zeroed = min(zeroed, j0);
#pragma unroll 1
        for (int j = 0; j < kSub; ++j) {
          uint4* const chunk = reinterpret_cast<uint4*>(tileV + j * R::kBytes) + lane % R::kChunks;
          if (__any(holds_special<DT>(*chunk))) *chunk = make_uint4(0u, 0u, 0u, 0u);
        }
        reads_done();
      }
    }
    if constexpr (DT == kBF16) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db) {
          const uint32_t v_at = (vt ^ (db << 6)) + ks * 16 * R::kBytes;
          o[0][db] = score_step<DT>(read_frag_transposed(v_at, v_at + 8 * R::kBytes), __builtin_bit_cast(Frag, pf[ks]), o[0][db]);
        }
    } else {
      typedef const __attribute__((address_space(3))) float* LdsFloats;
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int db = 0; db < R::kBlocks; ++db) {
          const float v = *(LdsFloats)(static_cast<uintptr_t>((vt ^ (db << 7)) + (8 * (e >> 2) + (e & 3)) * R::kBytes));
          o[0][db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[e], o[0][db], 0, 0, 0);
        }
    }
    reads_done();
    if (more_tiles) request(std::true_type(), t + 1, here);
  }
  Finish<DT, HD, 1, WINDOW>::add_back(a, mine, token, own, m, o, zeroed, min((t1 - cache_tiles) * kSub - 1, rows_last));
  // ---- the waves' shares: 16 bytes of a row a lane, each wave then has a quarter of the dimensions
  constexpr int kParts = 4 * R::kBlocks, kMine = kParts / kWaves;
  l[0] += __shfl_xor(l[0], 32, kWave);
  m_s[wave][lane] = m[0];
  l_s[wave][lane] = l[0];
#pragma unroll
  for (int k = 0; k < kParts; ++k)
    *reinterpret_cast<tree::f32x4*>(my_lds + (k * kWave + lane) * 16) = tree::f32x4{o[0][k / 4][4 * (k % 4)], o[0][k / 4][4 * (k % 4) + 1], o[0][k / 4][4 * (k % 4) + 2], o[0][k / 4][4 * (k % 4) + 3]};
  __syncthreads();
  if (row[0] >= rows) return;
  float M = -INFINITY, sum = 0.0f, weight[kWaves];
#pragma unroll
  for (int v = 0; v < kWaves; ++v) M = fmaxf(M, m_s[v][lane]);
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    weight[v] = m_s[v][lane] > -INFINITY ? fast_exp2(m_s[v][lane] - M) : 1.0f;  // (no maximum: a sum of zero, or NaN)
    sum += l_s[v][lane] * weight[v];
  }
  const size_t out_row = packed_row(a, mine, row[0], token[0]);
  const size_t part = mine.split * static_cast<size_t>(a.tokens) * a.heads * a.group + out_row;
  if (wave == 0 && half == 0) {
    if (plan.used > 1) {
      a.part_m[part] = M;
      a.part_l[part] = sum;
    } else if (a.lse != nullptr) {
      a.lse[out_row] = kLn2 * (M + __log2f(sum));
    }
  }
  const float inv = 1.0f / sum;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = wave * kMine + i, d0 = 32 * (k / 4) + 8 * (k % 4) + 4 * half;
    tree::f32x4 all = tree::f32x4{0};
#pragma unroll
    for (int v = 0; v < kWaves; ++v) all += *reinterpret_cast<const tree::f32x4*>(ring + v * F::kWaveBytes + (k * kWave + lane) * 16) * weight[v];
    if (plan.used > 1) *reinterpret_cast<tree::f32x4*>(a.part_o + part * HD + d0) = all;
    else tree::store4<DT>(a.out, out_row * HD + d0, all * inv);
  }
}

// The splits' shares of a tile's rows, HD / 4 lanes with 16 bytes of a row each; four splits at a time, in their order.  `parts` workgroups a tile: with one for
// every few rows most of the time goes into finding out which (24 requests with 6 chunks of 384 tokens, 148 -> 140 us; 32 that decode a token, 112 -> 107).
template <int DT, int HD, int ROWS, int KEYS> __global__ __launch_bounds__(kThreads) void chunk_join(ChunkArgs a, int parts) {
  constexpr int LANES = HD / 4, PER = kThreads / LANES, kAtOnce = 4;
  RowTile t;
  if (!row_tile_of<ROWS>(a, blockIdx.x / parts, t, 1)) return;
  const Plan<DT, ROWS, KEYS> plan(a, t);
  if (plan.used == 1) return;  // (one split has written its rows)
  const int sub = threadIdx.x % LANES;
  const size_t plane = static_cast<size_t>(a.tokens) * a.heads * a.group;
#pragma unroll 1
  for (int i = blockIdx.x % parts * PER + threadIdx.x / LANES; i < t.rows; i += parts * PER) {
    const int row = t.first_row + i;
    const size_t at = packed_row(a, t, row, row / a.group);
    float M = -INFINITY, sum = 0.0f;
    tree::f32x4 o = tree::f32x4{0};
#pragma unroll 1
    for (int k0 = 0; k0 < plan.used; k0 += kAtOnce) {
      float m[kAtOnce], l[kAtOnce];
      tree::f32x4 part[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const size_t from = min(k0 + k, plan.used - 1) * plane + at;
        m[k] = a.part_m[from];
        l[k] = a.part_l[from];
        part[k] = *reinterpret_cast<const tree::f32x4*>(a.part_o + from * HD + 4 * sub);
      }
      float most = M;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) most = fmaxf(most, m[k]);
      const float before = M > -INFINITY ? fast_exp2(M - most) : 1.0f;
      o *= before;
      sum *= before;
      M = most;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (k0 + k >= plan.used) break;
        const float w = m[k] > -INFINITY ? fast_exp2(m[k] - M) : 1.0f;  // (no maximum: a sum of zero, or NaN)
        o += part[k] * w;
        sum += l[k] * w;
      }
    }
    tree::store4<DT>(a.out, at * HD + 4 * sub, o * (1.0f / sum));
    if (a.lse != nullptr && sub == 0) a.lse[at] = kLn2 * (M + __log2f(sum));
  }
}

#pragma clang diagnostic pop

template <int DT, int HD, int ROWS, int KEYS, class Kernel> hipError_t launch_tiles(Kernel kernel, int lds, const ChunkArgs& a, hipStream_t s) {
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return hipErrorInvalidValue;
  const int total = a.row_tiles * a.heads * a.splits;
  {
    ProfScope ps(kProfChunkAttend, s);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>((total + 7) / 8 * 8)), dim3(kThreads), lds, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  ProfScope ps(kProfChunkJoin, s);
  // (at most 4096 of them, and no more than four times an average tile's rows are for)
  const int per = kThreads / (HD / 4), tiles = a.row_tiles * a.heads;
  const long long rows = 4ll * a.tokens * a.group / a.requests;
  const int parts = static_cast<int>(std::max(1ll, std::min({static_cast<long long>(ROWS / per), 4096ll / tiles, (rows + per - 1) / per})));
  hipLaunchKernelGGL((chunk_join<DT, HD, ROWS, KEYS>), dim3(static_cast<unsigned>(tiles) * parts), dim3(kThreads), 0, s, a, parts);
  return hipGetLastError();
}
template <int DT, int HD, bool WINDOW> hipError_t launch_attend_form(const ChunkArgs& a, hipStream_t s) {
  if constexpr (DT == kBF16 && HD == 128)
    if (a.row_tile == 256) return launch_tiles<DT, HD, 256, 64>(chunk_attend_pair<HD, WINDOW>, PairForm<HD>::kBytes, a, s);
  if (a.row_tile == 32) return launch_tiles<DT, HD, 32, 32>(chunk_attend_few<DT, HD, WINDOW>, FewForm<DT, HD>::kBytes, a, s);
  return launch_tiles<DT, HD, 128, 32>(chunk_attend<DT, HD, WINDOW>, TileForm<DT, HD>::kBytes, a, s);
}
template <int DT, int HD> hipError_t launch_attend(const ChunkArgs& a, hipStream_t s) {
  return a.recency_window > 0 ? launch_attend_form<DT, HD, true>(a, s) : launch_attend_form<DT, HD, false>(a, s);
}

}  // namespace chunk
}  // namespace roco
