// What the rows of a chunk add to the statistics of the slots and of the chunk's own tokens:
//   pbar[i, j] = mean over the group's heads of exp(logit - lse),  Acc[j] += sum_i pbar[i, j],  Acc2[j] += sum_i pbar[i, j]^2.
//
// The probabilities are formed again from one pass over the queries: left behind by the attention they would be 4 bytes per slot, head and
// token.  A workgroup owns keys, 32 in the lanes of each group of a wave as B operands in registers, and walks the query rows, which come in tiles
// of 64 through a ring in LDS; the result tile has its key in the lane and 16 rows in the lane's registers, so that the sums run down the
// registers: no exchange between lanes, no atomics, a fixed order.  Which (token, head) a tile's row holds is the choice of the lane that
// fetches it: the heads of a token, filled up to a power of two, lie in consecutive registers of one lane, and their mean is a sum of registers.
#pragma once
#include "chunk.hpp"
#include "profile.hpp"

namespace roco {
namespace chunk {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

constexpr int kQueryTile = 64;  // rows of a stage

template <int DT, int HD> struct ColumnForm {
  using R = Rows<DT, HD>;
  static constexpr int kGroups = DT == kBF16 ? 2 : 1;              // of 32 keys of a wave
  static constexpr int kKeys = kWaves * 32 * kGroups;              // of a workgroup
  static constexpr int kTileBytes = kQueryTile * R::kBytes;
  static constexpr int kStages = kTileBytes <= 16384 ? 4 : 2;
  static constexpr int kAhead = kStages - 1;
  static constexpr int kLoads = kTileBytes / kWaves / 1024;        // of a wave and tile
};

// P: heads of a token, filled up to a power of two (32: 17 to 32 heads, 64: 33 to 64).
template <int DT, int HD, int P> __global__ __launch_bounds__(kThreads, 2) void chunk_columns(ChunkArgs a, int cache_blocks, int fresh_blocks) {
  using R = Rows<DT, HD>;
  using F = ColumnForm<DT, HD>;
  constexpr int NG = F::kGroups;
  constexpr int kTokens = kQueryTile / P;                          // of a tile
  constexpr int kTileLoads = F::kLoads + 1;
  extern __shared__ __attribute__((aligned(1024))) char ring[];
  __shared__ __attribute__((aligned(256))) float lse_s[F::kStages][kWaves][kQueryTile];  // (a copy for each wave, which waits for its own loads)
  // workgroups of the slots, and behind them of the chunk's tokens; a unit's side by side on a die
  const int total = cache_blocks * a.units + fresh_blocks * a.heads, share = (total + 7) / 8;
  const int id = static_cast<int>(blockIdx.x % 8) * share + static_cast<int>(blockIdx.x / 8);
  if (static_cast<int>(blockIdx.x / 8) >= share || id >= total) return;
  const bool of_fresh = id >= cache_blocks * a.units;
  Located at;
  int head, block;
  if (of_fresh) {
    const int i = id - cache_blocks * a.units;
    head = i / fresh_blocks;
    if (!locate_tile<F::kKeys>(a, 1, i % fresh_blocks, at)) return;
    block = at.tile;
  } else {
    const int u = id / cache_blocks;
    block = id % cache_blocks;
    at.request = u / a.heads;
    head = u % a.heads;
    at.first = __builtin_amdgcn_readfirstlane(min(max(a.start[at.request], 0), a.tokens));
    at.count = __builtin_amdgcn_readfirstlane(min(max(a.start[at.request + 1], 0), a.tokens)) - at.first;
  }
  const int u = at.request * a.heads + head;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int half = lane >> 5;
  const int budget = budget_of(a.pages, a.B, at.request);
  const int n = __builtin_amdgcn_readfirstlane(min(max(a.n_used[u], 0), budget));
  const int c = __builtin_amdgcn_readfirstlane(min(at.count, budget));  // tokens taken over
  const int keys = of_fresh ? c : n, j0 = block * F::kKeys;
  if (c <= 0 || j0 >= keys) return;

  // the keys
  const Groups groups(a.pages, a.B, a.heads, at.request, head);
  Frag own[NG][R::kSteps];
  int kj[NG], kpos[NG];
  bool there[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    kj[g] = j0 + (wave * NG + g) * 32 + (lane & 31);
    const int j = min(kj[g], keys - 1);
    const char* base;
    there[g] = true;
    if (of_fresh) {
      base = static_cast<const char*>(a.k_new) + static_cast<int64_t>(at.first + j) * a.kv_stride + static_cast<size_t>(head) * R::kBytes;
      kpos[g] = j;
    } else {
      uint32_t r;
      const int page = a.pages.table != nullptr ? a.pages.table[static_cast<size_t>(at.request) * a.pages.max_pages + (j >> a.pages.page_log2)] : 0;
      there[g] = groups.row_of(j, page, r);
      base = static_cast<const char*>(a.K) + static_cast<size_t>(there[g] ? r : 0u) * R::kBytes;
      kpos[g] = a.recency_window > 0 ? a.pos[static_cast<size_t>(u) * a.B + j] - a.qpos0[at.request] : 0;  // against the chunk's first token
    }
#pragma unroll
    for (int kk = 0; kk < R::kSteps; ++kk) own[g][kk] = *reinterpret_cast<const Frag*>(base + (2 * kk + half) * 16);
  }

  // the walk over the rows: of the chunk's own keys, only from the block's first token on
  const int t0 = of_fresh ? j0 / kTokens : 0, t1 = (c + kTokens - 1) / kTokens;
  const uint32_t ring_addr = lds_address(ring), lse_addr = lds_address(&lse_s[0][wave][0]);
  // row x of a half tile of 32 is register 4 (x / 8) + x % 4 of half x / 4 % 2
  const auto virtual_row = [](int x) { return (x & 32) + ((x >> 2) & 1) * 16 + ((x >> 3) & 3) * 4 + (x & 3); };
  int qoff[F::kLoads];
#pragma unroll
  for (int i = 0; i < F::kLoads; ++i) {
    const int x = (wave * F::kLoads + i) * R::kPerLoad + lane / R::kChunks, v = virtual_row(x);
    const int h = v % P;
    qoff[i] = h < a.group ? static_cast<int>(v / P * a.q_stride) + h * R::kBytes + (((lane % R::kChunks) ^ R::swizzle_k(x & 31)) << 4) : 0x7ffffff0;
  }
  const int loff = lane % P < a.group ? ((lane / P) * a.heads * a.group + lane % P) * 4 : 0x7ffffffc;
  const char* const q0 = static_cast<const char*>(a.q) + static_cast<int64_t>(at.first) * a.q_stride + static_cast<size_t>(head) * a.group * R::kBytes;
  const float* const l0 = a.lse + (static_cast<size_t>(at.first) * a.heads + head) * a.group;
  const auto request = [&](int t, int stage) {
    const int first = t * kTokens, mine = uniform_min(c - first, kTokens);
    const v4i32 qbuf = make_buffer(q0 + static_cast<int64_t>(first) * a.q_stride, static_cast<uint32_t>(mine - 1) * static_cast<uint32_t>(a.q_stride) + a.group * R::kBytes);
    const v4i32 lbuf = make_buffer(l0 + static_cast<size_t>(first) * a.heads * a.group, static_cast<uint32_t>((mine - 1) * a.heads * a.group + a.group) * 4u);
#pragma unroll
    for (int i = 0; i < F::kLoads; ++i) load16_to_lds(qbuf, ring_addr + stage * F::kTileBytes + (wave * F::kLoads + i) * 1024, qoff[i], 0);
    mfma::load4_to_lds(lbuf, lse_addr + stage * (kWaves * kQueryTile * 4), loff, 0);
  };
#pragma unroll
  for (int i = 0; i < F::kAhead; ++i)
    if (t0 + i < t1) request(t0 + i, i);
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): the keys are in before the loop

  const float sc = a.scale_log2, bias = a.recency_bias_log2, inv = 1.0f / static_cast<float>(a.group);
  const int w = a.recency_window;
  const bool squares = !a.pol.keeps_last_score() && !a.pol.counts_above_average(), filled_up = P != a.group;
  const uint32_t frag = (lane & 31) * R::kBytes + ((half ^ R::swizzle_k(lane & 31)) << 4);
  const int last_key = j0 + (wave * NG + NG) * 32 - 1;  // of the wave's
  const bool idle = j0 + wave * NG * 32 >= keys;
  float sum[NG], sum2[NG], heads_sum[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) sum[g] = sum2[g] = heads_sum[g] = 0.0f;
  int stage = 0;
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    if (t + F::kAhead - 1 < t1) wait_loads<(F::kAhead - 1) * kTileLoads>();
    else wait_loads<0>();
    __syncthreads();
    if (t + F::kAhead < t1) request(t + F::kAhead, stage == 0 ? F::kStages - 1 : stage - 1);
    const uint32_t st = ring_addr + stage * F::kTileBytes + frag;
    const float* const lse_t = &lse_s[stage][wave][16 * half];
    stage = stage == F::kStages - 1 ? 0 : stage + 1;
    const int first = t * kTokens;
    if (idle || (of_fresh && first + kTokens - 1 < last_key - 32 * NG + 1)) continue;
    // everything is seen by every key, and outside the recency windows
    bool interior = squares && first + kTokens <= c && !(of_fresh && first < last_key);
    if (w > 0) {
#pragma unroll
      for (int g = 0; g < NG; ++g) interior = interior && !__any(first - kpos[g] < w && first + kTokens - 1 - kpos[g] >= 0);
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      f32x16 s[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) s[g] = f32x16{0};
#pragma unroll
      for (int kk = 0; kk < R::kSteps; ++kk) {
        const Frag qf = read_frag((st ^ (kk << 5)) + sub * 32 * R::kBytes);
#pragma unroll
        for (int g = 0; g < NG; ++g) s[g] = score_step<DT>(qf, own[g][kk], s[g]);
      }
      float lse[16];
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const tree::f32x4 v = *reinterpret_cast<const tree::f32x4*>(lse_t + 32 * sub + 4 * e4);
#pragma unroll
        for (int e = 0; e < 4; ++e) lse[4 * e4 + e] = v[e] * kLog2e;
      }
      const auto add = [&](auto inside) {
        constexpr bool kInside = decltype(inside)::value;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x = fmaf(s[g][e], sc, -lse[e]);
            const int local = (32 * sub + 16 * half + e) / P;  // the row's token
            if (!kInside && w > 0) x += static_cast<unsigned>(first + local - kpos[g]) < static_cast<unsigned>(w) ? bias : 0.0f;
            float p = fast_exp2(x);
            if (filled_up && e % P >= a.group && P <= 16) p = 0.0f;
            if (P > 16 && filled_up) p = (32 * sub + 16 * half + e) % P >= a.group ? 0.0f : p;
            heads_sum[g] = (P <= 16 ? e % P == 0 : e == 0 && (P == 32 || sub == 0)) ? p : heads_sum[g] + p;
            if ((P <= 16 && (e + 1) % P == 0) || (e == 15 && (P == 32 || (P == 64 && sub == 1)))) {
              float mean = heads_sum[g];
              if (P > 16) mean += __shfl_xor(mean, 32, kWave);
              mean *= inv;
              const int token = first + local;
              if (kInside) {
                sum[g] += mean;
                sum2[g] = fmaf(mean, mean, sum2[g]);
              } else {
                const bool counts = token < c && !(of_fresh && token < kj[g]);
                const float second = squares ? mean * mean : a.pol.keeps_last_score() ? (token == c - 1 ? mean : 0.0f)
                                                           : a.pol.second_statistic(0.0f, mean, static_cast<float>(n + token + 1));
                sum[g] += counts ? mean : 0.0f;
                sum2[g] += counts ? second : 0.0f;
              }
            }
          }
        }
      };
      if (interior) add(std::true_type());
      else add(std::false_type());
    }
  }
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    if (P <= 16) {  // (with more heads both halves have the same sums)
      sum[g] += __shfl_xor(sum[g], 32, kWave);
      sum2[g] += __shfl_xor(sum2[g], 32, kWave);
    }
    if (half != 0 || kj[g] >= keys) continue;
    if (of_fresh) {
      const size_t i = static_cast<size_t>(at.first + kj[g]) * a.heads + head;
      a.fresh[i] = sum[g];
      a.fresh[static_cast<size_t>(a.tokens) * a.heads + i] = sum2[g];
    } else {
      float* const to = a.sums + static_cast<size_t>(u) * 2 * a.B + kj[g];
      to[0] = there[g] ? sum[g] : -1.0f;  // (not seen)
      to[a.B] = sum2[g];
    }
  }
}

#pragma clang diagnostic pop

template <int DT, int HD, int P> hipError_t launch_columns_form(const ChunkArgs& a, hipStream_t s) {
  using F = ColumnForm<DT, HD>;
  constexpr int kLds = F::kStages * F::kTileBytes;
  const void* const fn = reinterpret_cast<const void*>(chunk_columns<DT, HD, P>);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) return hipErrorInvalidValue;
  const int cache_blocks = (a.B + F::kKeys - 1) / F::kKeys, fresh_blocks = tiles_of(a.requests, a.tokens, 1, F::kKeys);
  const int total = cache_blocks * a.units + fresh_blocks * a.heads;
  hipLaunchKernelGGL((chunk_columns<DT, HD, P>), dim3(static_cast<unsigned>((total + 7) / 8 * 8)), dim3(kThreads), kLds, s, a, cache_blocks, fresh_blocks);
  return hipGetLastError();
}
template <int DT, int HD> hipError_t launch_columns(const ChunkArgs& a, hipStream_t s) {
  ProfScope ps(kProfChunkColumns, s);
  if (a.group <= 1) return launch_columns_form<DT, HD, 1>(a, s);
  if (a.group <= 2) return launch_columns_form<DT, HD, 2>(a, s);
  if (a.group <= 4) return launch_columns_form<DT, HD, 4>(a, s);
  if (a.group <= 8) return launch_columns_form<DT, HD, 8>(a, s);
  if (a.group <= 16) return launch_columns_form<DT, HD, 16>(a, s);
  return a.group <= 32 ? launch_columns_form<DT, HD, 32>(a, s) : launch_columns_form<DT, HD, 64>(a, s);
}

}  // namespace chunk
}  // namespace roco
