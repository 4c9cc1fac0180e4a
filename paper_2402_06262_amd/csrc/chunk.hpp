// What the kernels of chunks share: which request a tile of packed rows belongs to, and the matrix products of 32 x 32 tiles.
#pragma once
#include <algorithm>

#include "tree.hpp"

namespace roco {
namespace chunk {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

using mfma::bf16x8;
using mfma::f32x16;
using mfma::lds_address;
using mfma::load16_to_lds;
using mfma::make_buffer;
using mfma::v4i32;
using mfma::wait_loads;
using tree::budget_of;
using tree::uniform_max;
using tree::uniform_min;

constexpr int kThreads = 256, kWaves = kThreads / kWave;
typedef const __attribute__((address_space(4))) int32_t* ConstWords;  // (read by scalar loads, which the tiles' loads do not wait for)

// A tile of the rows of one request: `tile` counts them, the request's tokens are first .. first + count - 1 of the packed ones.
struct Located { int request, tile, first, count; };

// Tiles of ROWS rows, `group` of them for a token.  A request's tiles begin at number floor(start group / ROWS) + request: room enough for
// all of its tiles, whatever the others have, so that no launch has to count them; a number that is nobody's is left out.  64 requests are
// looked at per step, a lane each.
template <int ROWS> __device__ __forceinline__ bool locate_tile(const ChunkArgs& a, int group, int t, Located& at) {
  const int lane = threadIdx.x & (kWave - 1);
  const auto start_of = [&](int r) { return min(max(a.start[r], 0), a.tokens); };
  int lo = 0, hi = a.requests, base = 0;
  bool known = false;
#pragma unroll 1
  do {
    const int step = (hi - lo + kWave - 1) / kWave, r = lo + lane * step;
    const int s = start_of(min(r, a.requests));
    const int b = static_cast<int>(static_cast<uint32_t>(s) * static_cast<uint32_t>(group) / ROWS) + r;
    const int count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(r < hi && b <= t));
    if (count == 0) return false;
    lo += (count - 1) * step;
    hi = min(hi, lo + step);
    if (step == 1) {
      at.first = __shfl(s, count - 1, kWave);
      base = __shfl(b, count - 1, kWave);
      known = count < kWave;
      at.count = __shfl(s, min(count, kWave - 1), kWave) - at.first;
    }
  } while (hi - lo > 1);
  if (!known) {
    at.first = start_of(lo);
    at.count = start_of(lo + 1) - at.first;
    base = static_cast<int>(static_cast<uint32_t>(at.first) * static_cast<uint32_t>(group) / ROWS) + lo;
  }
  at.request = __builtin_amdgcn_readfirstlane(lo);
  at.tile = __builtin_amdgcn_readfirstlane(t - base);
  at.first = __builtin_amdgcn_readfirstlane(at.first);
  at.count = __builtin_amdgcn_readfirstlane(at.count);
  return at.tile >= 0 && at.count > 0;
}
// Tiles that a launch needs for all requests.
inline int tiles_of(int requests, int tokens, int group, int rows) {
  return static_cast<int>(static_cast<long long>(tokens) * group / rows) + requests;
}

// Rows of BYTES bytes in LDS: chunk c (16 bytes) of row r lies in slot c ^ swizzle.  K: 32 rows of one chunk are read together; V: of bf16
// eight rows of 64 bytes (transposed), of fp32 two rows, four apart, of 128 bytes.
template <int DT, int HD> struct Rows {
  static constexpr int kBytes = HD * (DT == kBF16 ? 2 : 4);
  static constexpr int kChunks = kBytes / 16;
  static constexpr int kSteps = kChunks / 2;        // of a score: two lane halves with a chunk each
  static constexpr int kBlocks = HD / 32;           // of 32 output dimensions
  static constexpr int kPerLoad = 1024 / kBytes;    // rows of a wave-wide load
  static __device__ __forceinline__ int swizzle_k(int r) { return kBytes == 128 ? (r >> 1) & 7 : r & 15; }
  static __device__ __forceinline__ int swizzle_v(int r) {
    if (DT == kF32) return ((r >> 2) & 1) << 3;
    return HD == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
  }
};

// Scores of 32 rows `a` against 32 rows `b`, the chunk that the lane holds of either (lane l: row l % 32, half l / 32 of a step's two chunks);
// register e of the result belongs to row 8 (e / 4) + 4 (l / 32) + e % 4 of `a` and row l % 32 of `b`.
typedef uint4_vec Frag;  // (a vector of the language: of a structure of four words the compiler makes four values, and copies to put them together again)
template <int DT> __device__ __forceinline__ f32x16 score_step(const Frag& a, const Frag& b, f32x16 c) {
  if constexpr (DT == kBF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
}
__device__ __forceinline__ Frag read_frag(uint32_t lds_addr) {
  typedef const __attribute__((address_space(3))) Frag* LdsFrag;
  return *(LdsFrag)(static_cast<uintptr_t>(lds_addr));
}
// Two transposed reads of 16-bit elements.
__device__ __forceinline__ Frag read_frag_transposed(uint32_t lo_addr, uint32_t hi_addr) {
  const mfma::v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mfma::lds_v4i16*)(static_cast<uintptr_t>(lo_addr)));
  const mfma::v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mfma::lds_v4i16*)(static_cast<uintptr_t>(hi_addr)));
  return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A unit's slots in groups of 16: a page holds whole groups.
struct Groups {
  ConstWords table;  // the request's, or null
  int page_log2, n_pages, head, heads;
  uint32_t first_row;  // without a table: row of the unit's slot 0
  __device__ __forceinline__ Groups(const CachePages& pages, int B, int heads_, int request, int head_)
      : table(pages.table != nullptr ? (ConstWords)(pages.table + static_cast<size_t>(request) * pages.max_pages) : nullptr),
        page_log2(pages.page_log2), n_pages(pages.n_pages), head(head_), heads(heads_),
        first_row(static_cast<uint32_t>(request * heads_ + head_) * static_cast<uint32_t>(B)) {}
  __device__ __forceinline__ int page_of(int slot) const { return table != nullptr ? table[slot >> page_log2] : 0; }
  // Row of `slot`, whose page is known, in the caches; false: there is no such page.
  __device__ __forceinline__ bool row_of(int slot, int page, uint32_t& row) const {
    row = first_row + static_cast<uint32_t>(slot);
    if (table == nullptr) return true;
    if (page < 0 || page >= n_pages) return false;
    row = (static_cast<uint32_t>(page * heads + head) << page_log2) + static_cast<uint32_t>(slot & ((1 << page_log2) - 1));
    return true;
  }
};

// The sums of a chunk's probabilities: tiles of 64 rows of queries, of as many tokens as there are powers of two of heads in them; keys of a workgroup.
constexpr int kQueryTile = 64;
constexpr int column_keys(int dtype) { return dtype == kBF16 ? 256 : 128; }
inline int column_tokens(int group) {
  int tokens = kQueryTile;
  while (kQueryTile / tokens < group) tokens /= 2;
  return tokens;
}
// Up to this budget a unit's slots are chosen by a workgroup of 256 threads beside those of the sums, not by one of 1024 before them (8 heads of 4 queries, 128
// dimensions, chunks of 16: 64 units of 1024 slots 26 -> 19 us, of 4096 43 -> 35; 8 units of 2048 25 -> 21, of 4096 25 -> 26).
constexpr int kMostChosenBeside = 4096;
inline bool chosen_beside(int B) { return B <= kMostChosenBeside; }
// Tiles of rows, shared by the workgroups of a block of keys.
struct RowShares {
  int tiles, per, used;
  __device__ __forceinline__ RowShares(int tiles_, int splits) : tiles(tiles_), per(max((tiles + splits - 1) / splits, kLeastTiles)), used((tiles + per - 1) / per) {}
  static constexpr int kLeastTiles = 4;
};

#pragma clang diagnostic pop

}  // namespace chunk
}  // namespace roco
