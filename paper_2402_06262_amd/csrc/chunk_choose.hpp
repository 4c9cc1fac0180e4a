// The victims of a chunk, and the slots that its tokens take.
#pragma once
#include "chunk.hpp"

namespace roco {
namespace chunk {

// words: kChoiceWords<NT> of LDS; var_key: room for [2][B] ranking keys
template <int NT> constexpr int kChoiceWords = SelectLds<1>::kWords + (NT / kWave + 1 + 3) / 4 * 4;
template <int NT> __device__ __forceinline__ void choose_slots(const ChunkArgs& a, int u, uint32_t* words, uint32_t* var_key) {
  uint32_t *const sel_sh = words, *const scan_sh = words + SelectLds<1>::kWords;
  const int tid = threadIdx.x, B = a.B;
  const int request = u / a.heads, head = u - request * a.heads;
  const int first = min(max(a.start[request], 0), a.tokens), count = max(min(max(a.start[request + 1], 0), a.tokens) - first, 0);
  const int budget = budget_of(a.pages, B, request);
  const int n = min(max(a.n_used[u], 0), budget), c = min(count, budget);
  const int n_new = min(budget, n + c), E = n + c - n_new;
  int32_t* const info = a.info + static_cast<size_t>(u) * 4;
  if (tid == 0) {
    info[0] = c;
    info[1] = n;
    info[2] = n_new;
  }
  // tokens that took the place of none
  const auto record = [&](int k, int slot, int position) {
    const size_t at = static_cast<size_t>(first + k) * a.heads + head;
    if (a.evicted_slot != nullptr) a.evicted_slot[at] = slot;
    if (a.evicted_pos != nullptr) a.evicted_pos[at] = position;
  };
  for (int k = E + tid; k < count; k += NT) record(k, -1, -1);  // (the freed slots come before the empty ones)
  if (c == 0) return;
  int32_t* const mark = a.mark + static_cast<size_t>(u) * B;
  for (int j = n + tid; j < n_new; j += NT) mark[j] = E + j - n;
  if (E == 0) {
    for (int j = tid; j < n; j += NT) mark[j] = -1;
    return;
  }
  const float* const acc = a.stats + static_cast<size_t>(u) * 3 * B;
  const float* const acc2 = acc + B;
  const float* const cnt = acc2 + B;
  const int32_t* const pos = a.pos + static_cast<size_t>(u) * B;
  uint32_t* const mas_key = var_key + B;
  constexpr int kEach = 4;  // slots of a thread at a time: their loads are in flight together
#pragma unroll 1
  for (int i0 = tid; i0 < n; i0 += kEach * NT) {
    float f[kEach], f2[kEach], fc[kEach];
    int fp[kEach];
    uint32_t mas[kEach], var[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = min(i0 + e * NT, n - 1);
      f[e] = acc[i];
      f2[e] = acc2[i];
      fc[e] = cnt[i];
      fp[e] = pos[i];
    }
    ranking_keys<kEach>(f, f2, fc, fp, a.pol, mas, var);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = min(i0 + e * NT, n - 1);
      mas_key[i] = mas[e];
      var_key[i] = var[e];
    }
  }
  __syncthreads();
  const uint32_t m = min(static_cast<uint32_t>(n), static_cast<uint32_t>(a.pol.scope_size(min(a.scope, budget), n)) + static_cast<uint32_t>(E) - 1u);
  KSmallest r = {0u, 0u};
#pragma unroll 1
  for (int phase = 0; phase < 2; ++phase) {
    const uint32_t* const key = phase == 0 ? var_key : mas_key;
    r = select_k_smallest<NT, 1, 1>([&](int i) -> uint32_t { return key[i]; }, n, phase == 0 ? m : static_cast<uint32_t>(E),
                                                phase == 0 && a.pol.scope_is_window(), sel_sh, phase == 0 || a.pol.spreads_importance());
    if (phase == 0) {
      for (int i = tid; i < n; i += NT)
        if (!r.has(var_key[i], i)) mas_key[i] = 0xffffffffu;  // outside the scope
      __syncthreads();
    }
  }
  // the i-th victim's slot gets token i: thread t has the contiguous slots from t * per on
  const int per = (n + NT - 1) / NT, lo = min(n, tid * per), hi = min(n, lo + per);
  uint32_t mine = 0, all;
#pragma unroll 1
  for (int j = lo; j < hi; ++j) mine += r.has(mas_key[j], j) ? 1u : 0u;
  uint32_t rank = block_exclusive_scan<NT>(mine, scan_sh, all);
#pragma unroll 1
  for (int j = lo; j < hi; ++j) {
    const bool out = r.has(mas_key[j], j);
    const int k = out ? static_cast<int>(rank++) : -1;
    mark[j] = k;
    if (out) record(k, j, pos[j]);
  }
}

}  // namespace chunk
}  // namespace roco
