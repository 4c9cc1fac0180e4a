// What the kernels of drafted trees share: where a cache's rows lie, tiles of them on their way to LDS, matrix products of both
// storage types, and which nodes of a tree a node sees.
#pragma once
#include "block_fused.hpp"

namespace roco {
namespace tree {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"

using fused::f32x4;
using mfma::lds_address;
using mfma::lds_read_transposed;
using mfma::load16_to_lds;
using mfma::make_buffer;
using mfma::reads_done;
using mfma::v4i32;
using mfma::wait_loads;

// Tiles of BYTES, one wave's, in groups of 16 slots: a page holds whole groups, and what a group's load finds behind its last row
// comes back as zeros (the group has a buffer descriptor of its own, of as many rows as are there).
// Chunk c (16 bytes) of a row r of K lies in slot c ^ swizzle_k(r), of V in slot c ^ swizzle_v(r), so that what the lanes read together
// falls on distinct banks: 16 rows of one chunk of K; of V 32 bytes of 8 rows (bf16, transposed) or 64 bytes of every fourth row (fp32).
template <int DT, int HD, int BYTES = 8192> struct Tile {
  static constexpr int kBytes = HD * (DT == kBF16 ? 2 : 4);   // of a row
  static constexpr int kChunks = kBytes / 16;
  static constexpr int kPerLoad = kWave / kChunks;            // rows of a wave-wide load
  static constexpr int kSlots = BYTES / kBytes;
  static constexpr int kGroups = kSlots / 16;
  static constexpr int kLoads = BYTES / 1024, kGroupLoads = kLoads / kGroups;
  static constexpr int kSteps = kChunks / 4;                  // of a score: four lane groups with a chunk each
  static constexpr int kBlocks = HD / 16;                     // of 16 output dimensions
  static __device__ __forceinline__ int swizzle_k(int r) { return kBytes == 128 ? (r >> 1) & 7 : r & 15; }
  static __device__ __forceinline__ int swizzle_v(int r) {
    if (DT == kF32) return ((r >> 2) & 3) << 2;
    return HD == 128 ? ((r & 3) << 2) ^ (((r >> 2) & 1) << 1) : ((r >> 1) & 3) << 1;
  }
};

// Scores of 16 rows `a` against 16 rows `b`, the chunk that the lane holds of either (lane l: row l % 16, lane group l / 16);
// register e of the result belongs to row 4 (l / 16) + e of `a` and row l % 16 of `b`.
template <int DT> __device__ __forceinline__ f32x4 score_step(const uint4& a, const uint4& b, f32x4 c) {
  if constexpr (DT == kBF16) {
    return fused::mfma16(a, b, c);
  } else {
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
  }
}

// Four consecutive elements, rounded to the storage type.
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

// The nodes that node `lane` of a tree sees, a bit each: itself and those above it, from its parent.  Twice as far up with every step.  A
// parent that is not an earlier node is none.
__device__ __forceinline__ uint64_t seen_nodes(int parent, int nodes, int lane) {
  int up = parent;
  if (up >= lane || up < 0 || lane >= nodes) up = -1;
  uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const int at = max(up, 0);
    const uint32_t lo2 = __shfl(lo, at, kWave), hi2 = __shfl(hi, at, kWave);
    const int up2 = __shfl(up, at, kWave);
    if (up >= 0) {
      lo |= lo2;
      hi |= hi2;
      up = up2;
    }
  }
  return lo | static_cast<uint64_t>(hi) << 32;
}
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int lane) {
  const uint32_t lo = __shfl(static_cast<uint32_t>(v), lane, kWave), hi = __shfl(static_cast<uint32_t>(v >> 32), lane, kWave);
  return lo | static_cast<uint64_t>(hi) << 32;
}

// Minimum and maximum of values that are the same for all lanes: the compiler forms a clamp on the vector ALU.
__device__ __forceinline__ int uniform_min(int a, int b) {
  int r;
  asm("s_min_i32 %0, %1, %2" : "=s"(r) : "s"(a), "s"(b) : "scc");
  return r;
}
__device__ __forceinline__ int uniform_max(int a, int b) {
  int r;
  asm("s_max_i32 %0, %1, %2" : "=s"(r) : "s"(a), "s"(b) : "scc");
  return r;
}

// Slots of a request's units, and how many of them a unit uses.
__device__ __forceinline__ int budget_of(const CachePages& pages, int B, int request) {
  return pages.budget != nullptr ? min(max(pages.budget[request], 0), B) : B;
}

// Workgroups that a unit of n slots needs along its slots.
__device__ __forceinline__ int splits_used(int n, int chunk) { return max((n + chunk - 1) / chunk, 1); }

// A wave's tiles of the slots [row0, row1) of a unit: every W-th one, from a start that differs between workgroups so that they do not
// walk the memory channels in lock step; behind the cache's tiles come `node_tiles` of a tree's nodes.  The tile numbers `t` are the
// wave's own; they are asked for in order, every STEP-th one.
template <int DT, int HD, int W, int BYTES = 8192, int STEP = 1> struct Walk {
  using T = Tile<DT, HD, BYTES>;
  static constexpr int G = T::kGroups;
  typedef const __attribute__((address_space(4))) int32_t* Table;  // (constant: read by scalar loads, which the tiles' loads do not wait for)
  int row0, row1, cache_tiles, mine, rot, wave, nodes;
  uint32_t first_row;     // without a table: row of the unit's slot 0
  int head, heads, page_log2, n_pages;
  bool paged;
  Table table;            // the request's
  int ahead[G];           // pages of the groups of the tile that is asked for next

  __device__ __forceinline__ void init(const CachePages& pages, int B, int heads_, int unit, int request, int row0_, int row1_, int nodes_, int wave_, unsigned start) {
    row0 = row0_; row1 = row1_; nodes = nodes_; wave = wave_;
    cache_tiles = (max(row1 - row0, 0) + T::kSlots - 1) / T::kSlots;
    const int node_tiles = (nodes + T::kSlots - 1) / T::kSlots;
    mine = (cache_tiles + node_tiles - wave + W - 1) / W;
    rot = mine > 0 ? static_cast<int>(start % static_cast<unsigned>(mine)) : 0;
    first_row = static_cast<uint32_t>(unit) * static_cast<uint32_t>(B);
    heads = heads_;
    head = unit - request * heads;
    page_log2 = pages.page_log2;
    n_pages = pages.n_pages;
    paged = pages.table != nullptr;
    table = (Table)(pages.table + static_cast<size_t>(request) * pages.max_pages);
    look_ahead(0);
  }
  __device__ __forceinline__ int index(int t) const {  // among the workgroup's tiles
    int i = t + rot;
    if (i >= mine) i -= mine;
    return i * W + wave;
  }
  __device__ __forceinline__ bool is_nodes(int t) const { return index(t) >= cache_tiles; }
  __device__ __forceinline__ int first_slot(int t) const { return row0 + index(t) * T::kSlots; }
  __device__ __forceinline__ int first_node(int t) const { return (index(t) - cache_tiles) * T::kSlots; }
  __device__ __forceinline__ void look_ahead(int t) {
    if (!paged || cache_tiles == 0) return;
#pragma unroll
    for (int i = 0; i < G; ++i) ahead[i] = table[uniform_min(first_slot(t) + 16 * i, row1 - 1) >> page_log2];
  }

  // Rows of the groups of tile t in their array, and how many of each are there (a byte each).
  struct Place { uint32_t row[G]; uint32_t there; };
  __device__ __forceinline__ Place place(int t) {
    Place p;
    p.there = 0;
    const bool of_nodes = is_nodes(t);
    const int first = of_nodes ? first_node(t) : first_slot(t), end = of_nodes ? nodes : row1;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int slot = first + 16 * i;
      int there = uniform_min(uniform_max(end - slot, 0), 16);
      uint32_t row = (of_nodes ? 0u : first_row) + static_cast<uint32_t>(slot);
      if (paged && !of_nodes) {
        const int page = ahead[i];
        if (page < 0 || page >= n_pages) there = 0;  // such a page is not touched, and what it would hold is not seen
        row = (static_cast<uint32_t>(page * heads + head) << page_log2) + static_cast<uint32_t>(slot & ((1 << page_log2) - 1));
      }
      p.row[i] = there > 0 ? row : 0u;
      p.there |= static_cast<uint32_t>(there) << (8 * i);
    }
    if (t + STEP < mine) look_ahead(t + STEP);
    return p;
  }
};

// 16 bytes at an LDS address.
__device__ __forceinline__ uint4 lds_read16(uint32_t addr) {
  typedef const __attribute__((address_space(3))) mfma::v4i32 lds_v4i32;
  return __builtin_bit_cast(uint4, *(lds_v4i32*)(static_cast<uintptr_t>(addr)));
}
__device__ __forceinline__ uint2 lds_read_transposed_at(uint32_t addr) {
  const mfma::v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mfma::lds_v4i16*)(static_cast<uintptr_t>(addr)));
  return __builtin_bit_cast(uint2, v);
}

// Byte offsets inside a group's rows of the chunks that this lane fetches with the group's loads.
template <int DT, int HD, bool VALUES> __device__ __forceinline__ void load_offsets(int* off) {
  using T = Tile<DT, HD>;
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int i = 0; i < T::kGroupLoads; ++i) {
    const int r = T::kPerLoad * i + lane / T::kChunks;
    off[i] = r * T::kBytes + (((lane % T::kChunks) ^ (VALUES ? T::swizzle_v(r) : T::swizzle_k(r))) << 4);
  }
}

// Requests a tile.  STREAMING: of a cache that is far larger than the chip's last-level cache, with the non-temporal hint.
template <int DT, int HD, bool STREAMING, int G>
__device__ __forceinline__ void request_tile(const void* rows, const uint32_t (&row)[G], uint32_t there, uint32_t lds, const int* off) {
  using T = Tile<DT, HD>;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const v4i32 buf = make_buffer(static_cast<const char*>(rows) + static_cast<size_t>(row[i]) * T::kBytes, ((there >> (8 * i)) & 0xffu) * T::kBytes);
#pragma unroll
    for (int j = 0; j < T::kGroupLoads; ++j) mfma::load16_to_lds_hint<STREAMING>(buf, lds + (i * T::kGroupLoads + j) * 1024, off[j], 0);
  }
}

#pragma clang diagnostic pop

}  // namespace tree
}  // namespace roco
