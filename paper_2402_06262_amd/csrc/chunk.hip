// Chunks of new tokens: which form of the attention a call takes, and the taking over into the budgeted cache, in two launches or three.
//
//   chunk_columns : the sums of the chunk's probabilities (chunk_columns.hpp), for slots that are evicted too.  Beside them, or before them in
//   chunk_choose    a launch of its own for large budgets, one workgroup per unit chooses E = max(0, n + c - budget) victims by the statistics
//                   as they stand (two exact searches, as in block_prepare), and the slots that the chunk's tokens take, in ascending
//                   order: ChunkArgs::mark (chunk_choose.hpp).
//   chunk_apply   : the sums added to the statistics; the tokens' rows, positions and statistics to their slots.
#include <stdlib.h>

#include <algorithm>

#include "chunk_choose.hpp"
#include "profile.hpp"

namespace roco {

hipError_t launch_chunk_attend_bf16_128(const ChunkArgs& a, hipStream_t s);  // a file each
hipError_t launch_chunk_attend_bf16_64(const ChunkArgs& a, hipStream_t s);
hipError_t launch_chunk_attend_f32_128(const ChunkArgs& a, hipStream_t s);
hipError_t launch_chunk_attend_f32_64(const ChunkArgs& a, hipStream_t s);
hipError_t launch_chunk_columns_bf16_128(const ChunkArgs& a, hipStream_t s);
hipError_t launch_chunk_columns_bf16_64(const ChunkArgs& a, hipStream_t s);
hipError_t launch_chunk_columns_f32_128(const ChunkArgs& a, hipStream_t s);
hipError_t launch_chunk_columns_f32_64(const ChunkArgs& a, hipStream_t s);

namespace {

using namespace chunk;

constexpr int kChooseThreads = 1024;

// LDS: the ranking keys are in LDS (B <= kMaxDecodeBudgetLds).
template <bool LDS> __global__ __launch_bounds__(kChooseThreads, 8) void chunk_choose(ChunkArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds_keys[];  // [2][B]
  __shared__ __attribute__((aligned(16))) uint32_t words[kChoiceWords<kChooseThreads>];
  choose_slots<kChooseThreads>(a, blockIdx.x, words, LDS ? lds_keys : a.keys + static_cast<size_t>(blockIdx.x) * 2 * a.B);
}

// A workgroup's slots of one unit.
constexpr int kApplySlots = 256;
__global__ __launch_bounds__(kThreads) void chunk_apply(ChunkArgs a, int row_bytes, int blocks, int tile_tokens, int keys) {
  __shared__ int32_t list_s[kApplySlots], listed_s;  // slots that tokens take
  const int u = blockIdx.x / blocks, row0 = blockIdx.x % blocks * kApplySlots, tid = threadIdx.x;
  const int request = u / a.heads, head = u - request * a.heads;
  const int32_t* const info = a.info + static_cast<size_t>(u) * 4;
  const int c = info[0], n_new = info[2];
  if (c == 0 || row0 >= n_new) return;
  const int first = min(max(a.start[request], 0), a.tokens);
  if (tid == 0) {
    listed_s = 0;
    if (row0 == 0) a.n_used[u] = n_new;
  }
  __syncthreads();
  const int j = row0 + tid;
  const size_t at = static_cast<size_t>(u) * a.B;
  if (j < n_new) {
    const int k = a.mark[at + j];
    float* const acc = a.stats + 3 * at + j;
    if (k >= 0) {
      const size_t i = static_cast<size_t>(first + k) * a.heads + head;
      const RowShares shares((c + tile_tokens - 1) / tile_tokens - k / keys * keys / tile_tokens, a.row_splits);
      float own = 0.0f, own2 = 0.0f;
#pragma unroll 4
      for (int s = 0; s < shares.used; ++s) {
        const float* const from = a.fresh + s * 2 * a.fresh_plane() + i;
        own += from[0];
        own2 += from[a.fresh_plane()];
      }
      acc[0] = own;
      acc[a.B] = own2;
      acc[2 * static_cast<size_t>(a.B)] = static_cast<float>(c - k);
      a.pos[at + j] = a.qpos0[request] + k;
      list_s[atomicAdd(&listed_s, 1)] = tid;
    } else {
      const RowShares shares((c + tile_tokens - 1) / tile_tokens, a.row_splits);
      float more = 0.0f, more2 = 0.0f;
#pragma unroll 4
      for (int s = 0; s < shares.used; ++s) {
        const float* const from = a.sums + 2 * (static_cast<size_t>(s) * a.units * a.B + at) + j;
        more += from[0];
        more2 += from[a.B];
      }
      if (!(more < 0.0f)) {  // (below zero: not seen)
        acc[0] += more;
        acc[a.B] = (a.pol.keeps_last_score() ? 0.0f : acc[a.B]) + more2;
        acc[2 * static_cast<size_t>(a.B)] += static_cast<float>(c);
      }
    }
  }
  __syncthreads();
  const int lanes = row_bytes / 16, listed = listed_s, col = tid % lanes * 16;
#pragma unroll 1
  for (int i = tid / lanes; i < listed; i += kThreads / lanes) {
    const int slot = row0 + list_s[i], k = a.mark[at + slot];
    const Groups groups(a.pages, a.B, a.heads, request, head);
    uint32_t row;
    const int page = a.pages.table != nullptr ? a.pages.table[static_cast<size_t>(request) * a.pages.max_pages + (slot >> a.pages.page_log2)] : 0;
    if (!groups.row_of(slot, page, row)) continue;
    const int64_t src = static_cast<int64_t>(first + k) * a.kv_stride + static_cast<int64_t>(head) * row_bytes + col;
    const uint4 key = load16(static_cast<const char*>(a.k_new) + src), value = load16(static_cast<const char*>(a.v_new) + src);
    const size_t dst = static_cast<size_t>(row) * row_bytes + col;
    *reinterpret_cast<uint4*>(static_cast<char*>(a.K) + dst) = key;
    *reinterpret_cast<uint4*>(static_cast<char*>(a.V) + dst) = value;
  }
}

}  // namespace

// Row tiles of all heads, times the splits: of a grid with more of them many may have nothing to do.
constexpr long long kMostTiles = 4096;

// The form of the attention that a call takes.  Row tiles of 256, where requests of bf16 rows of 128 dimensions have 1024 of them or more on average: 4096 cached keys,
// group 4, 8 heads, 8 requests of 256 tokens: 160 us against 216 with 128; 1 request of as many: 61 against 59; 8 requests of 100: 148 against 127; with 64
// dimensions, 8 requests of 512: 244 against 237.  Of 32, where they have few: one token of 32 requests, 8 heads, over 2048 keys, fp32 / 128 104 us against 286, fp32 / 64 62 and 165,
// bf16 / 64 35 and 36; of 4 heads over 4096, bf16 / 128, 103 and 106.  12 tokens of 8 requests, 4 heads each, over 2048: bf16 / 128 25 and 32, bf16 / 64 26 and 25, fp32 / 128 77 and
// 152; 64 tokens bf16 / 128 61 and 45, fp32 / 128 207 and 221; 512, groups of 2, fp32 / 128 386 and 359.  And where there is little work in all, which they share out more finely: 100
// tokens of 4 requests, 16 heads, over 300 keys 13 and 26; 64 of 16, 8 heads, over 1000 36 and 32.
// Splits: those with the shortest time, of a compute unit's workgroups one after the other, or of one that has four waves alone half as long again for each
// further one; a workgroup being as long as its waves' tiles of 32 keys and, for its start, its share of the outputs and the joining, eight more (at 128 dimensions).
static int chunk_row_tile(int dtype, int head_dim, int requests, int heads, int group, int tokens, long long keys) {
  const char* const rows_asked = getenv("ROCO_CHUNK_ROWS");
  const int asked_tile = rows_asked != nullptr ? atoi(rows_asked) : 0;
  const bool can_pair = dtype == kBF16 && head_dim == 128;
  const bool can_few = static_cast<long long>(tiles_of(requests, tokens, group, 32)) * heads <= kMostWorkgroups - 8;  // (as workgroups of a launch, whole eights)
  if ((asked_tile == 32 && can_few) || asked_tile == 128 || (asked_tile == 256 && can_pair)) return asked_tile;
  const long long rows = static_cast<long long>(tokens) * group;
  return rows <= (dtype == kF32 ? 256ll : head_dim == 128 ? 32ll : 8ll) * requests || rows * heads * keys <= 160000 ? 32 : can_pair && rows >= 1024ll * requests ? 256 : 128;
}
static int chunk_splits_asked() {
  const char* const asked = getenv("ROCO_CHUNK_SPLITS");
  return asked != nullptr ? std::min(atoi(asked), kMostChunkSplits) : 0;
}
static long long chunk_key_tiles(int tokens, int B) { return (static_cast<long long>(B) + tokens + 31) / 32; }
// Splits that `keys` tiles of them have work for.
static long long chunk_most_splits(int dtype, int row_tile, long long keys) {
  const int least_keys = chunk_least_keys(dtype, row_tile);
  return std::min<long long>(kMostChunkSplits, (keys * 32 + (row_tile == 32 ? least_keys - 1 : 0)) / least_keys);
}
ChunkSplits chunk_attend_splits(int dtype, int head_dim, int requests, int heads, int group, int tokens, int B) {
  const int splits = chunk_splits_asked();
  ChunkSplits c;
  const long long rows = static_cast<long long>(tokens) * group, keys = chunk_key_tiles(tokens, B);
  c.row_tile = chunk_row_tile(dtype, head_dim, requests, heads, group, tokens, keys);
  const bool pair = c.row_tile == 256, few = c.row_tile == 32;
  c.row_tiles = tiles_of(requests, tokens, group, c.row_tile);
  const long long tiles = static_cast<long long>(c.row_tiles) * heads, full = pair ? rows / 256 * heads : tiles;
  const int most = static_cast<int>(std::max(1ll, std::min(chunk_most_splits(dtype, c.row_tile, keys), kMostTiles / tiles)));
  const bool alone = pair || (few ? dtype == kF32 && head_dim == 128 : dtype == kF32);  // on its compute unit
  c.splits = 1;
  long long least = -1;
  for (int i = 1; i <= most; ++i) {
    const long long each = (full * i + 255) / 256, waves = few ? 4 * i : i;
    const long long cost = 4 * (alone ? 2 * each : 1 + each) * ((keys + waves - 1) / waves + head_dim / 16) + (few ? i : 0);
    if (least < 0 || cost < least) {
      least = cost;
      c.splits = i;
    }
  }
  if (splits >= 1 && tiles * 32 < kMostWorkgroups) c.splits = static_cast<int>(std::max(1ll, std::min<long long>(splits, (kMostWorkgroups - 8) / tiles)));
  // Shares of equal length, where there is work for it to matter and every die can have heads of its own: 24 requests, of which 6 have chunks of 384 tokens over 30 to
  // 4096 keys, 8 heads of 4 queries, 164 -> 147 us; 16 of 128 or one over 8192 or fewer, 114 -> 106; 4 of 600 or fewer over 4096, 183 -> 158; 23 of 175 over
  // 7782, 64 dimensions, 391 -> 243.  With two heads, 24 of 384 or one 78 -> 86; without enough work, 2 to 10 % more (a look at all requests costs a microsecond).
  c.equal_shares = c.splits > 1 && requests > 1 && heads % 8 == 0 && rows > 32ll * requests && tiles * keys >= 20000;
  return c;
}

// A call with more tokens has more row tiles and so, often, fewer splits, and a smaller share of a workspace.  What it asks for is what every call with fewer may
// want: no more splits than there are keys for; and where tiles of R rows have more than one split, tiles times splits are kMostTiles at most, R kMostTiles rows.
long long chunk_most_shares(int dtype, int head_dim, int requests, int heads, int group, int tokens, int B) {
  const long long rows = static_cast<long long>(tokens) * group, keys = chunk_key_tiles(tokens, B);
  const int asked = chunk_splits_asked(), largest = chunk_row_tile(dtype, head_dim, requests, heads, group, tokens, keys);
  if (asked >= 1) return asked > 1 ? rows * heads * asked : 0;
  long long most = 0;
  for (int row_tile : {32, 128, 256}) {
    const long long splits = chunk_most_splits(dtype, row_tile, keys);
    if (row_tile <= largest && splits > 1) most = std::max(most, std::min(rows * heads * splits, row_tile * kMostTiles));
  }
  return most;
}

// Until there are 2048 workgroups, four rounds of them, while a chunk has four tiles of rows for each.
int chunk_row_splits(int dtype, int requests, int heads, int group, int tokens, int B, bool or_fewer) {
  const char* const asked = getenv("ROCO_CHUNK_ROW_SPLITS");
  const int splits = asked != nullptr ? std::min(atoi(asked), kMostRowSplits) : 0;
  const int keys = column_keys(dtype);
  const long long blocks = (static_cast<long long>(requests) * ((B + keys - 1) / keys) + tiles_of(requests, or_fewer ? 0 : tokens, 1, keys)) * heads;
  if (splits >= 1) return static_cast<int>(std::max(1ll, std::min<long long>(splits, (kMostWorkgroups - 16ll - static_cast<long long>(requests) * heads) / blocks)));
  const long long most = tokens / column_tokens(group) / RowShares::kLeastTiles;
  return static_cast<int>(std::max(1ll, std::min({2048 / blocks, most, static_cast<long long>(kMostRowSplits)})));
}

hipError_t launch_chunk_attend(int dtype, int head_dim, const ChunkArgs& a, hipStream_t s) {
  if (dtype == kBF16) return head_dim == 128 ? launch_chunk_attend_bf16_128(a, s) : launch_chunk_attend_bf16_64(a, s);
  return head_dim == 128 ? launch_chunk_attend_f32_128(a, s) : launch_chunk_attend_f32_64(a, s);
}

hipError_t launch_chunk_commit(int dtype, int head_dim, const ChunkArgs& a, hipStream_t s) {
  hipError_t e;
  if (!chosen_beside(a.B)) {
    ProfScope ps(kProfChunkChoose, s);
    const size_t key_lds = key_lds_bytes(a.B);
    if (!allow_key_lds(reinterpret_cast<const void*>(chunk_choose<true>), key_lds)) return hipErrorInvalidValue;
    if (key_lds == 0) hipLaunchKernelGGL((chunk_choose<false>), dim3(a.units), dim3(kChooseThreads), 0, s, a);
    else hipLaunchKernelGGL((chunk_choose<true>), dim3(a.units), dim3(kChooseThreads), key_lds, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (dtype == kBF16) e = head_dim == 128 ? launch_chunk_columns_bf16_128(a, s) : launch_chunk_columns_bf16_64(a, s);
  else e = head_dim == 128 ? launch_chunk_columns_f32_128(a, s) : launch_chunk_columns_f32_64(a, s);
  if (e != hipSuccess) return e;
  ProfScope ps(kProfChunkApply, s);
  const int blocks = (a.B + kApplySlots - 1) / kApplySlots;
  hipLaunchKernelGGL(chunk_apply, dim3(static_cast<unsigned>(a.units) * blocks), dim3(kThreads), 0, s, a, head_dim * (dtype == kBF16 ? 2 : 4), blocks,
                     column_tokens(a.group), column_keys(dtype));
  return hipGetLastError();
}

}  // namespace roco
