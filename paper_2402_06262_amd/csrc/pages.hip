// Pages of caches of different budgets: block tables and slot maps from the requests' lengths, and rows stored by slot map.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "profile.hpp"

namespace roco {
namespace {

constexpr int kSumThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kFillEntries = 4;      // of the map, side by side, per thread and step
constexpr int kSelfSummed = 2048;    // most requests whose sums every workgroup of the fill forms itself

// Pages and slots.  Their sums stay at 2^31 - 1 where they would pass it: a prefix is then behind every entry of a list or map.
struct Sums { uint32_t pages, rows; };
__device__ __forceinline__ Sums add_up(const Sums& x, const Sums& y) {
  return {min(x.pages + y.pages, 0x7fffffffu), min(x.rows + y.rows, 0x7fffffffu)};
}

// Exclusive prefix of such sums over the workgroup's threads, in their order, and their total.  sh: an entry per wave.
template <int NT> __device__ __forceinline__ Sums prefix_of(Sums v, Sums* sh, Sums& total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const auto other = [](uint32_t x, auto ctrl, auto row_mask) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, decltype(row_mask)::value, 0xF, false));
  };
  const auto step = [&](auto ctrl, auto row_mask) { v = add_up(v, {other(v.pages, ctrl, row_mask), other(v.rows, ctrl, row_mask)}); };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});
  Sums before = {__shfl_up(v.pages, 1, kWave), __shfl_up(v.rows, 1, kWave)};
  if (lane == 0) before = {0u, 0u};
  __syncthreads();  // nobody reads `sh` of a sum before
  if (lane == kWave - 1) sh[wave] = v;
  __syncthreads();
  Sums off = {0u, 0u};
  total = off;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) {
    if (w == wave) off = total;
    total = add_up(total, sh[w]);
  }
  return add_up(off, before);
}

struct Need { int first, last, held, want; };  // pages [first, last) are to be taken, slots [held, want) are new
__device__ __forceinline__ Need need_of(const PageTableArgs& a, int r) {
  Need x;
  const int most = a.max_pages << a.page_log2;
  x.held = a.held != nullptr ? min(max(a.held[r], 0), most) : 0;
  x.want = min(max(a.want[r], x.held), most);
  const int up = (1 << a.page_log2) - 1;
  x.first = (x.held + up) >> a.page_log2;
  x.last = (x.want + up) >> a.page_log2;
  return x;
}

// One workgroup: the prefix sums of pages and of new slots over the requests.
__global__ __launch_bounds__(kSumThreads) void page_sums(PageTableArgs a) {
  __shared__ Sums sh[kSumThreads / kWave];
  Sums sum = {0u, 0u};
#pragma unroll 1
  for (int r0 = 0; r0 < a.requests; r0 += kSumThreads) {
    const int r = r0 + threadIdx.x;
    Need x = {0, 0, 0, 0};
    if (r < a.requests) x = need_of(a, r);
    Sums more;
    const Sums before = add_up(sum, prefix_of<kSumThreads>({static_cast<uint32_t>(x.last - x.first), static_cast<uint32_t>(x.want - x.held)}, sh, more));
    if (r < a.requests) {
      a.page_start[r] = static_cast<int32_t>(before.pages);
      a.row_start[r] = static_cast<int32_t>(before.rows);
    }
    sum = add_up(sum, more);
  }
  if (threadIdx.x == 0) {
    a.page_start[a.requests] = static_cast<int32_t>(sum.pages);
    a.row_start[a.requests] = static_cast<int32_t>(sum.rows);
  }
}

// The map, kFillEntries entries per thread at a time, and the table, a wave per request.  SELF: every workgroup forms the requests' sums in its
// LDS, from lengths that the L2 has, instead of waiting for a launch that does: a step of 64 requests 7.7 -> 5.4 us.  A page number is asked
// for once for entries of the same page; a division and a search per entry took 19.6 us for 1024 requests of up to 8192 slots.
template <bool SELF> __global__ __launch_bounds__(kFillThreads) void page_fill(PageTableArgs a) {
  __shared__ Sums sh[kFillThreads / kWave];
  extern __shared__ int32_t sums_s[];  // SELF: pages before a request, new slots before it, slots that it holds and is to have
  int32_t *const page_s = sums_s, *const row_s = page_s + a.requests + 1, *const held_s = row_s + a.requests + 1, *const want_s = held_s + a.requests;
  const int tid = threadIdx.x;
  if (SELF) {
    constexpr int kEach = kSelfSummed / kFillThreads;
    const int each = (a.requests + kFillThreads - 1) / kFillThreads, r0 = tid * each;
    Sums mine[kEach], all = {0u, 0u};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      mine[i] = {0u, 0u};
      if (i < each && r0 + i < a.requests) {
        const Need x = need_of(a, r0 + i);
        mine[i] = {static_cast<uint32_t>(x.last - x.first), static_cast<uint32_t>(x.want - x.held)};
        held_s[r0 + i] = x.held;
        want_s[r0 + i] = x.want;
      }
      all = add_up(all, mine[i]);
    }
    Sums total, before = prefix_of<kFillThreads>(all, sh, total);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (i < each && r0 + i < a.requests) {
        page_s[r0 + i] = static_cast<int32_t>(before.pages);
        row_s[r0 + i] = static_cast<int32_t>(before.rows);
      }
      before = add_up(before, mine[i]);
    }
    if (tid == 0) {
      page_s[a.requests] = static_cast<int32_t>(total.pages);
      row_s[a.requests] = static_cast<int32_t>(total.rows);
    }
    __syncthreads();
    if (blockIdx.x == 0) {
      for (int r = tid; r <= a.requests; r += kFillThreads) {
        a.page_start[r] = page_s[r];
        a.row_start[r] = row_s[r];
      }
    }
  }
  const int32_t* const page_start = SELF ? page_s : a.page_start;
  const int32_t* const row_start = SELF ? row_s : a.row_start;
  auto lengths_of = [&](int r) {
    if (!SELF) return need_of(a, r);
    Need x;
    x.held = held_s[r];
    x.want = want_s[r];
    x.first = (x.held + (1 << a.page_log2) - 1) >> a.page_log2;
    x.last = (x.want + (1 << a.page_log2) - 1) >> a.page_log2;
    return x;
  };
  // Page number i of request r: one of those it takes now, or one that its table holds.
  auto page_of = [&](int r, const Need& x, int i) {
    if (i < x.first) return a.table[static_cast<size_t>(r) * a.max_pages + i];
    const uint32_t at = static_cast<uint32_t>(page_start[r]) + static_cast<uint32_t>(i - x.first);
    return at < static_cast<uint32_t>(a.n_free) ? a.free_pages[at] : -1;
  };
  const int waves = kFillThreads / kWave * gridDim.x;
  for (int r = blockIdx.x * (kFillThreads / kWave) + tid / kWave; r < a.requests; r += waves) {
    const Need x = lengths_of(r);
    for (int i = x.first + tid % kWave; i < x.last; i += kWave) a.table[static_cast<size_t>(r) * a.max_pages + i] = page_of(r, x, i);
  }
  const long long total = a.padded ? static_cast<long long>(a.requests) * a.rows : a.rows;
  const long long step = static_cast<long long>(gridDim.x) * kFillThreads * kFillEntries;
  const uint32_t low = (1u << a.page_log2) - 1, most_page = 0x7fffffffu >> a.page_log2, rows = static_cast<uint32_t>(a.rows);
  for (long long i0 = (static_cast<long long>(blockIdx.x) * kFillThreads + tid) * kFillEntries; i0 < total; i0 += step) {
    int r;       // request and new slot of the entry.  (New slots are compared with how many there are, not slots with lengths: a map
    uint32_t k;  // may go on far behind a request's last slot, and held + k pass 2^31)
    if (a.padded) {
      if (total <= 0x7fffffff) {
        r = static_cast<int>(static_cast<uint32_t>(i0) / rows);
        k = static_cast<uint32_t>(i0) - static_cast<uint32_t>(r) * rows;
      } else {
        r = static_cast<int>(i0 / a.rows);
        k = static_cast<uint32_t>(i0 % a.rows);
      }
    } else {
      int lo = 0, hi = a.requests;  // the last request that starts at i0 or before it
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (row_start[mid] <= i0) lo = mid;
        else hi = mid;
      }
      r = lo;
      k = static_cast<uint32_t>(i0) - static_cast<uint32_t>(row_start[r]);
    }
    Need x = lengths_of(r);
    uint32_t fresh = static_cast<uint32_t>(x.want - x.held);
    int at = -1, page = -1;  // page `at` of the request
    int4 entries;
    int* const e = &entries.x;
    const uint32_t last = static_cast<uint32_t>(x.held) + k + kFillEntries - 1;  // slot of the last entry, if they are all of this request
    if (a.padded && k + kFillEntries <= rows && k >= fresh) {
      entries = make_int4(-1, -1, -1, -1);
    } else if (k + kFillEntries <= fresh && (!a.padded || k + kFillEntries <= rows) && (last & low) >= kFillEntries - 1) {  // of one page
      page = page_of(r, x, static_cast<int>(last >> a.page_log2));
      const int entry = static_cast<int>((static_cast<uint32_t>(page) << a.page_log2) + (last & low) - (kFillEntries - 1));
      entries = static_cast<uint32_t>(page) > most_page ? make_int4(-1, -1, -1, -1) : make_int4(entry, entry + 1, entry + 2, entry + 3);
    } else {
#pragma unroll
      for (int j = 0; j < kFillEntries; ++j) {
        // the next request: behind the end of its row of a padded map, or of its new slots in a packed one
        while (r + 1 < a.requests && k >= (a.padded ? rows : fresh)) {
          k = a.padded ? 0 : k - fresh;
          x = lengths_of(++r);
          fresh = static_cast<uint32_t>(x.want - x.held);
          at = -1;
        }
        e[j] = -1;
        if (k < fresh) {
          const int slot = x.held + static_cast<int>(k);
          if (slot >> a.page_log2 != at) {
            at = slot >> a.page_log2;
            page = page_of(r, x, at);
          }
          // (a page so far on that its slots are no 31-bit numbers is none)
          if (static_cast<uint32_t>(page) <= most_page) e[j] = (page << a.page_log2) + (slot & static_cast<int>(low));
        }
        ++k;
      }
    }
    if (i0 + kFillEntries <= total) {
      *reinterpret_cast<int4*>(a.map + i0) = entries;
    } else {
#pragma unroll
      for (int j = 0; j < kFillEntries; ++j)
        if (i0 + j < total) a.map[i0 + j] = e[j];
    }
  }
}

// 16 bytes of a row of K and of V per lane; a row's lanes lie side by side.  Bound by the bytes.  STREAMING: rows that are more than the chip's
// last-level cache takes, with the non-temporal hint both ways (16 caches x 32 heads x 2048 rows of 256 bytes, twice: 151 -> 143 us, 5.6 TB/s).
template <bool STREAMING> __global__ __launch_bounds__(256) void page_store(PageStoreArgs a, int lanes_log2) {
  const int lanes = 1 << lanes_log2;
  const long long id = (static_cast<long long>(blockIdx.y) * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const long long row = id >> lanes_log2;  // (group, head, row), rows side by side
  const int col = static_cast<int>(id & (lanes - 1)) * 16;
  const long long i = row % a.rows, gh = row / a.rows;
  const int h = static_cast<int>(gh % a.heads);
  const long long group = gh / a.heads;
  if (group >= a.groups) return;
  const int slot = a.map[group * a.rows + i];
  const int page = slot >> a.page_log2;
  if (slot < 0 || page >= a.n_pages) return;
  const size_t src = static_cast<size_t>(group * a.group_stride + i * a.row_stride + h * a.head_stride) + col;
  const size_t dst = (((static_cast<size_t>(page) * a.heads + h) << a.page_log2) + (slot & ((1 << a.page_log2) - 1))) * a.row_bytes + col;
  const char *const k_row = static_cast<const char*>(a.K_rows) + src, *const v_row = static_cast<const char*>(a.V_rows) + src;
  const uint4 k = STREAMING ? load16_streaming(k_row) : load16(k_row), v = STREAMING ? load16_streaming(v_row) : load16(v_row);
  uint4_vec *const k_at = reinterpret_cast<uint4_vec*>(static_cast<char*>(a.K) + dst), *const v_at = reinterpret_cast<uint4_vec*>(static_cast<char*>(a.V) + dst);
  if (STREAMING) {
    __builtin_nontemporal_store(__builtin_bit_cast(uint4_vec, k), k_at);
    __builtin_nontemporal_store(__builtin_bit_cast(uint4_vec, v), v_at);
  } else {
    *k_at = __builtin_bit_cast(uint4_vec, k);
    *v_at = __builtin_bit_cast(uint4_vec, v);
  }
}

}  // namespace

hipError_t launch_page_tables(const PageTableArgs& a, hipStream_t s) {
  ProfScope ps(kProfPageTables, s);
  const long long total = a.padded ? static_cast<long long>(a.requests) * a.rows : a.rows;
  // a step of every thread, as far as that gives no more than six workgroups per compute unit (1024 prompts of up to 8192 slots: 512 of them
  // 15.9 us, 1024 13.0, 1536 13.2, 2048 14.1)
  const long long want = std::max<long long>((total + kFillThreads * kFillEntries - 1) / (kFillThreads * kFillEntries), (a.requests + 3) / 4);
  const dim3 grid(static_cast<unsigned>(std::min<long long>(want, 1536)));
  if (a.requests <= kSelfSummed) {
    hipLaunchKernelGGL((page_fill<true>), grid, dim3(kFillThreads), (4 * a.requests + 2) * sizeof(int32_t), s, a);
  } else {
    hipLaunchKernelGGL(page_sums, dim3(1), dim3(kSumThreads), 0, s, a);
    hipLaunchKernelGGL((page_fill<false>), grid, dim3(kFillThreads), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_page_store(const PageStoreArgs& a, hipStream_t s) {
  ProfScope ps(kProfPageStore, s);
  const int lanes_log2 = __builtin_ctz(a.row_bytes) - 4;
  const long long lanes = (static_cast<long long>(a.groups) * a.heads * a.rows) << lanes_log2;
  const long long groups = (lanes + 255) / 256, side = std::min<long long>(groups, kStoreSide);
  const dim3 grid(static_cast<unsigned>(side), static_cast<unsigned>((groups + side - 1) / side));
  if (a.streaming) hipLaunchKernelGGL((page_store<true>), grid, dim3(256), 0, s, a, lanes_log2);
  else hipLaunchKernelGGL((page_store<false>), grid, dim3(256), 0, s, a, lanes_log2);
  return hipGetLastError();
}

}  // namespace roco
