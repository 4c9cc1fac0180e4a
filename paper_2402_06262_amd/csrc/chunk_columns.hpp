// What the rows of a chunk add to the statistics of the slots and of the chunk's own tokens:
//   pbar[i, j] = mean over the group's heads of exp(logit - lse),  Acc[j] += sum_i pbar[i, j],  Acc2[j] += sum_i pbar[i, j]^2.
//
// The probabilities are formed again from one pass over the queries: left behind by the attention they would be 4 bytes per slot, head and
// token.  A workgroup owns keys, 32 in the lanes of each group of a wave as B operands in registers, and walks the query rows, which come in tiles
// of 64 through a ring in LDS; the result tile has its key in the lane and 16 rows in the lane's registers, so that the sums run down the
// registers: no exchange between lanes, no atomics, a fixed order.  Which (token, head) a tile's row holds is the choice of the lane that
// fetches it: the heads of a token, filled up to a power of two, lie in consecutive registers of one lane, and their mean is a sum of registers.
// The scores of the next 32 rows are formed between the exponentials of these.  A chunk's rows are shared by up to 16 workgroups of a block of keys,
// whose sums chunk_apply adds in their order.
// Measured, all of roco_chunk_commit and the copy that restores the state, passes on one state: 4 requests of 512 tokens, 8 heads of 4 queries, 4096 slots, bf16, 128
// dimensions, 108 us (102 with states in turn; the products would take 60 at the 1.2 PFLOP/s of a large library product, the vector instructions 50), with one workgroup along
// the rows 122; 12 of up to 200, groups of 8, 2048 slots, 64 dimensions, 60 us and 66.  With one path for all rows, of selects and of branches within, 154 and 102 us of the
// kernel alone, and the requests side by side on a die, so that one had the longest.  A token of 32 requests, 8 heads, 2048 slots, fp32 / 128, 97 to 102 us (213 with the
// rows that a tile has not, 134 with room for three tiles), of 8 heads of 4 queries over 4096 slots, bf16 / 128, 90 to 97 us and 105 (K alone, 268 MB of either, would take
// 38 at the 7.0 TB/s that reads alone reach).
#pragma once
#include "chunk_choose.hpp"
#include "profile.hpp"

namespace roco {
namespace chunk {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

template <int DT, int HD> struct ColumnForm {
  using R = Rows<DT, HD>;
  static constexpr int kGroups = column_keys(DT) / kWaves / 32;    // of 32 keys of a wave
  static constexpr int kKeys = column_keys(DT);                    // of a workgroup
  static constexpr int kTileBytes = kQueryTile * R::kBytes;
  static constexpr int kStages = kTileBytes > 16384 ? 3 : 4;       // the tile in use, the next one, and others on their way
  static constexpr int kLoads = kTileBytes / kWaves / 1024;        // of a wave and tile
};

// P: heads of a token, filled up to a power of two (32: 17 to 32 heads, 64: 33 to 64).
template <int DT, int HD, int P> __global__ __launch_bounds__(kThreads, 2) void chunk_columns(ChunkArgs a, int choosers, int cache_blocks, int fresh_blocks, int stages) {
  using R = Rows<DT, HD>;
  using F = ColumnForm<DT, HD>;
  constexpr int NG = F::kGroups;
  constexpr int kTokens = kQueryTile / P;                          // of a tile
  constexpr int kTileLoads = F::kLoads + 1;
  extern __shared__ __attribute__((aligned(1024))) char ring[];
  __shared__ __attribute__((aligned(256))) float lse_s[F::kStages][kWaves][kQueryTile];  // (a copy for each wave, which waits for its own loads)
  // a workgroup for each unit that chooses its slots, if it has not been done; whole eights of them
  if (static_cast<int>(blockIdx.x) < choosers) {
    uint32_t* const words = reinterpret_cast<uint32_t*>(ring);
    if (static_cast<int>(blockIdx.x) < a.units) choose_slots<kThreads>(a, blockIdx.x, words, words + kChoiceWords<kThreads>);
    return;
  }
  // workgroups of the chunk's tokens, then of the slots; either in contiguous shares of the eight dies, with a unit's, which read the same queries, side by side
  // (and a head's units: a share of requests would have longer chunks than another)
  const int cache_each = cache_blocks * a.row_splits, fresh_each = fresh_blocks * a.row_splits;  // of a unit, and of a head
  const int cache_total = cache_each * a.units, fresh_total = fresh_each * a.heads, cache_share = (cache_total + 7) / 8, fresh_share = (fresh_total + 7) / 8;
  const int die = static_cast<int>(blockIdx.x % 8), i_die = (static_cast<int>(blockIdx.x) - choosers) / 8;
  const bool of_fresh = i_die < fresh_share;
  const int id = of_fresh ? die * fresh_share + i_die : die * cache_share + i_die - fresh_share;
  if (id >= (of_fresh ? fresh_total : cache_total)) return;
  Located at;
  int head, block, split;
  if (of_fresh) {
    head = id / fresh_each;
    split = id % fresh_each / fresh_blocks;
    if (!locate_tile<F::kKeys>(a, 1, id % fresh_blocks, at)) return;
    block = at.tile;
  } else {
    const int pair = id / cache_each;
    split = id % cache_each / cache_blocks;
    block = id % cache_blocks;
    head = pair / a.requests;
    at.request = __builtin_amdgcn_readfirstlane(pair % a.requests);
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
  // the walk over the rows: of the chunk's own keys, only from the block's first token on
  const int first_tile = of_fresh ? j0 / kTokens : 0;
  const RowShares shares((c + kTokens - 1) / kTokens - first_tile, a.row_splits);
  const int t0 = first_tile + split * shares.per, t1 = min(first_tile + shares.tiles, t0 + shares.per);
  if (t0 >= t1) return;

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
  for (int i = 0; i < F::kStages - 1; ++i)
    if (t0 + i < t1) request(t0 + i, i);
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): the keys are in before the loop
  __syncthreads();                     // the other waves' shares of the first tiles, too

  const float sc = a.scale_log2, bias = a.recency_bias_log2, log2_group = __log2f(static_cast<float>(a.group));
  const int w = a.recency_window;
  const bool squares = !a.pol.keeps_last_score() && !a.pol.counts_above_average(), filled_up = P != a.group;
  const uint32_t frag = (lane & 31) * R::kBytes + ((half ^ R::swizzle_k(lane & 31)) << 4);
  const int last_key = j0 + (wave * NG + NG) * 32 - 1;  // of the wave's
  float sum[NG], sum2[NG], mean[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) sum[g] = sum2[g] = mean[g] = 0.0f;
  int from[NG];  // the first token that sees the key
#pragma unroll
  for (int g = 0; g < NG; ++g) from[g] = of_fresh ? kj[g] : 0;
  int stage = 0;
  const auto next_tile = [&](int t) {  // the one behind t is wanted
    if (t + F::kStages - 2 < t1) wait_loads<(F::kStages - 3) * kTileLoads>();
    else wait_loads<0>();
    __syncthreads();
    if (t + F::kStages - 1 < t1) request(t + F::kStages - 1, stage == 0 ? F::kStages - 1 : stage - 1);
  };
  // Rows 32 h .. of tile t, in stage `at_stage`, from scores s; the scores of the 32 rows behind them, which begin at `next` in LDS, into s_next.
  // A matrix instruction, then vector work on the scores before: a wave keeps both busy, and two of them fill the gaps.
  constexpr int kEach = 16 / R::kSteps, kEarly = R::kSteps >= 4 ? 2 : 1;
  // The kinds of tiles: every key sees every row, and the heads of a token are a power of two; they are filled up; some keys do not see some rows; of
  // the rest, with recency windows or other statistics than the squares' sum.
  constexpr int kInside = 0, kFilled = 1, kPartly = 2, kAny = 3;
  const bool last_only = a.pol.keeps_last_score();
  const auto half_tile = [&](auto h_, auto kind_, auto ahead_, int t, int at_stage, uint32_t next, f32x16 (&s)[NG], f32x16 (&s_next)[NG]) {
    constexpr int h = decltype(h_)::value, kKind = decltype(kind_)::value;
    constexpr bool kAhead = decltype(ahead_)::value;  // there are rows behind them
    const int first = t * kTokens;
    const float* const lse_t = &lse_s[at_stage][wave][16 * half + 32 * h];
    Frag qf[R::kSteps];
#pragma unroll
    for (int i = 0; i < kEarly && kAhead; ++i) qf[i] = read_frag(next ^ (i << 5));
    float less[16];
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const tree::f32x4 v = *reinterpret_cast<const tree::f32x4*>(lse_t + 4 * e4);
#pragma unroll
      for (int e = 0; e < 4; ++e) less[4 * e4 + e] = fmaf(v[e], -kLog2e, -log2_group);
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) s_next[g] = f32x16{0};
#pragma unroll
    for (int kk = 0; kk < R::kSteps; ++kk) {
      if (kAhead && kk + kEarly < R::kSteps) qf[kk + kEarly] = read_frag(next ^ ((kk + kEarly) << 5));
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        if (kAhead) s_next[g] = score_step<DT>(qf[kk], own[g][kk], s_next[g]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = kEach * kk; e < kEach * kk + kEach; ++e) {
          float x = fmaf(s[g][e], sc, less[e]);
          const int local = (32 * h + 16 * half + e) / P;  // the row's token
          if (kKind == kAny) x += static_cast<unsigned>(first + local) - static_cast<unsigned>(kpos[g]) < static_cast<unsigned>(w) ? bias : 0.0f;
          float p = fast_exp2(x);
          if (kKind != kInside) p = (P <= 16 ? e : 32 * h + 16 * half + e) % P >= a.group ? 0.0f : p;
          mean[g] = (P <= 16 ? e % P == 0 : e == 0 && (P == 32 || h == 0)) ? p : mean[g] + p;
          if ((P <= 16 && (e + 1) % P == 0) || (e == 15 && (P == 32 || (P == 64 && h == 1)))) {
            if (P > 16) mean[g] += __shfl_xor(mean[g], 32, kWave);
            const int token = first + local;
            if (kKind >= kPartly) mean[g] = token >= from[g] && token < c ? mean[g] : 0.0f;
            sum[g] += mean[g];
            if (kKind != kAny) {
              sum2[g] = fmaf(mean[g], mean[g], sum2[g]);
            } else {
              const float last = token == c - 1 ? mean[g] : 0.0f, above = mean[g] * static_cast<float>(n + token + 1) > 1.0f ? 1.0f : 0.0f;
              sum2[g] += squares ? mean[g] * mean[g] : last_only ? last : above;
            }
          }
        }
        asm volatile("" : "+v"(mean[g]), "+v"(sum[g]), "+v"(sum2[g]));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const auto first_scores = [&](f32x16 (&s0)[NG]) {
#pragma unroll
    for (int g = 0; g < NG; ++g) s0[g] = f32x16{0};
#pragma unroll
    for (int kk = 0; kk < R::kSteps; ++kk) {
      const Frag qf = read_frag((ring_addr + frag) ^ (kk << 5));
#pragma unroll
      for (int g = 0; g < NG; ++g) s0[g] = score_step<DT>(qf, own[g][kk], s0[g]);
    }
  };
  const auto in_reach = [&](int first) {  // some row and key of one another (a row that there is not may be farther from its key than any number)
    bool window = false;
    if (w > 0) {
#pragma unroll
      for (int g = 0; g < NG; ++g) window = window || __any(first - kpos[g] < w && first + kTokens - 1 >= kpos[g]);
    }
    return window;
  };
  const bool no_keys = j0 + wave * NG * 32 >= keys;
  if (t1 - t0 == 1 && c - t0 * kTokens <= kTokens / 2) {  // half a tile has all the rows, a decoding token's for one
    if (!no_keys) {
      f32x16 s0[NG], s1[NG];
      first_scores(s0);
      if (in_reach(t0 * kTokens) || !squares) half_tile(std::integral_constant<int, 0>(), std::integral_constant<int, kAny>(), std::false_type(), t0, 0, 0u, s0, s1);
      else half_tile(std::integral_constant<int, 0>(), std::integral_constant<int, kPartly>(), std::false_type(), t0, 0, 0u, s0, s1);
    }
  } else if (no_keys) {  // no keys of this wave, but the other waves want its loads
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
      next_tile(t);
      stage = stage + 1 == stages ? 0 : stage + 1;
    }
  } else {
    f32x16 s0[NG], s1[NG];
    first_scores(s0);
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
      next_tile(t);
      const int first = t * kTokens, now = stage;
      stage = stage + 1 == stages ? 0 : stage + 1;
      const bool window = in_reach(first);
      const uint32_t second = ring_addr + now * F::kTileBytes + 32 * R::kBytes + frag, next = ring_addr + stage * F::kTileBytes + frag;
      const auto tile = [&](auto kind) {
        half_tile(std::integral_constant<int, 0>(), kind, std::true_type(), t, now, second, s0, s1);
        half_tile(std::integral_constant<int, 1>(), kind, std::true_type(), t, now, next, s1, s0);
      };
      if (window || !squares) tile(std::integral_constant<int, kAny>());
      else if (first + kTokens > c || (of_fresh && first < last_key)) tile(std::integral_constant<int, kPartly>());
      else if (filled_up) tile(std::integral_constant<int, kFilled>());
      else tile(std::integral_constant<int, kInside>());
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
      float* const to = a.fresh + split * 2 * a.fresh_plane() + i;
      to[0] = sum[g];
      to[a.fresh_plane()] = sum2[g];
    } else {
      float* const to = a.sums + (static_cast<size_t>(split) * a.units + u) * 2 * a.B + kj[g];
      to[0] = there[g] ? sum[g] : -1.0f;  // (not seen)
      to[a.B] = sum2[g];
    }
  }
}

#pragma clang diagnostic pop

template <int DT, int HD, int P> hipError_t launch_columns_form(const ChunkArgs& a, hipStream_t s) {
  using F = ColumnForm<DT, HD>;
  const int choosers = chosen_beside(a.B) ? (a.units + 7) / 8 * 8 : 0;
  // (no more stages than a request can have tiles: fewer of them let more workgroups onto a compute unit)
  const int tokens = column_tokens(a.group), stages = std::min(F::kStages, (a.tokens + tokens - 1) / tokens);
  const int lds = std::max(stages * F::kTileBytes, choosers > 0 ? (kChoiceWords<kThreads> + 2 * a.B) * 4 : 0);
  const void* const fn = reinterpret_cast<const void*>(chunk_columns<DT, HD, P>);
  // (the most that any call asks for: another thread's smaller call could lower a limit of this one's own before the launch)
  constexpr int kMostLds = std::max(F::kStages * F::kTileBytes, (kChoiceWords<kThreads> + 2 * kMostChosenBeside) * 4);
  if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, kMostLds) != hipSuccess) return hipErrorInvalidValue;
  const int cache_blocks = (a.B + F::kKeys - 1) / F::kKeys, fresh_blocks = tiles_of(a.requests, a.tokens, 1, F::kKeys);
  const int total = (cache_blocks * a.row_splits * a.units + 7) / 8 + (fresh_blocks * a.row_splits * a.heads + 7) / 8;
  hipLaunchKernelGGL((chunk_columns<DT, HD, P>), dim3(static_cast<unsigned>(total) * 8 + choosers), dim3(kThreads), lds, s, a, choosers, cache_blocks, fresh_blocks, stages);
  return hipGetLastError();
}
template <int DT, int HD> hipError_t launch_columns(const ChunkArgs& a, hipStream_t s) {
  ProfScope ps(kProfChunkColumns, s);
  switch (kQueryTile / column_tokens(a.group)) {
    case 1: return launch_columns_form<DT, HD, 1>(a, s);
    case 2: return launch_columns_form<DT, HD, 2>(a, s);
    case 4: return launch_columns_form<DT, HD, 4>(a, s);
    case 8: return launch_columns_form<DT, HD, 8>(a, s);
    case 16: return launch_columns_form<DT, HD, 16>(a, s);
    case 32: return launch_columns_form<DT, HD, 32>(a, s);
    default: return launch_columns_form<DT, HD, 64>(a, s);
  }
}

}  // namespace chunk
}  // namespace roco
