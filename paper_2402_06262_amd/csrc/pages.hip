// Pages of caches of different budgets: block tables and slot maps from the requests' lengths, and rows stored by slot map.
#include <algorithm>

#include "common.hpp"
#include "profile.hpp"

namespace roco {
namespace {

constexpr int kTableThreads = 1024;
constexpr int kMapPerBlock = 4096;   // entries of the map that a workgroup of the fill writes

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

// One workgroup: the prefix sums of pages and of new slots over the requests, and the new pages into the table.
__global__ __launch_bounds__(kTableThreads) void page_sums(PageTableArgs a) {
  __shared__ uint32_t sh[kTableThreads / kWave + 1];
  uint32_t pages = 0, rows = 0;
#pragma unroll 1
  for (int r0 = 0; r0 < a.requests; r0 += kTableThreads) {
    const int r = r0 + threadIdx.x;
    Need x = {0, 0, 0, 0};
    if (r < a.requests) x = need_of(a, r);
    uint32_t more_pages, more_rows;
    const uint32_t p = pages + block_exclusive_scan<kTableThreads>(static_cast<uint32_t>(x.last - x.first), sh, more_pages);
    const uint32_t s = rows + block_exclusive_scan<kTableThreads>(static_cast<uint32_t>(x.want - x.held), sh, more_rows);
    if (r < a.requests) {
      a.page_start[r] = static_cast<int32_t>(p);
      a.row_start[r] = static_cast<int32_t>(s);
    }
    pages += more_pages;
    rows += more_rows;
  }
  if (threadIdx.x == 0) {
    a.page_start[a.requests] = static_cast<int32_t>(pages);
    a.row_start[a.requests] = static_cast<int32_t>(rows);
  }
}

// Page number `i` of request r: one of those it takes now, or one that its table holds.
__device__ __forceinline__ int page_of(const PageTableArgs& a, int r, const Need& x, int start, int i) {
  if (i < x.first) return a.table[static_cast<size_t>(r) * a.max_pages + i];
  const int at = start + i - x.first;
  return at < a.n_free ? a.free_pages[at] : -1;
}

// The map, kMapPerBlock entries a workgroup, then (blocks from map_blocks on) the table, a workgroup per request.
__global__ __launch_bounds__(256) void page_fill(PageTableArgs a, int map_blocks) {
  if (static_cast<int>(blockIdx.x) >= map_blocks) {
    const int r = blockIdx.x - map_blocks;
    const Need x = need_of(a, r);
    const int start = a.page_start[r];
    for (int i = x.first + threadIdx.x; i < x.last; i += 256) a.table[static_cast<size_t>(r) * a.max_pages + i] = page_of(a, r, x, start, i);
    return;
  }
  const long long total = a.padded ? static_cast<long long>(a.requests) * a.rows : a.rows;
  const long long first = static_cast<long long>(blockIdx.x) * kMapPerBlock;
  const long long end = min(total, first + kMapPerBlock);
  const int low = (1 << a.page_log2) - 1;
  for (long long i = first + threadIdx.x; i < end; i += 256) {
    int r, k;
    if (a.padded) {
      r = static_cast<int>(i / a.rows);
      k = static_cast<int>(i % a.rows);
    } else {
      int lo = 0, hi = a.requests;  // the last request that starts at i or before it
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.row_start[mid] <= i) lo = mid;
        else hi = mid;
      }
      r = lo;
      k = static_cast<int>(i - a.row_start[r]);
    }
    const Need x = need_of(a, r);
    const int slot = x.held + k;
    int entry = -1;
    if (slot < x.want) {
      const int page = page_of(a, r, x, a.page_start[r], slot >> a.page_log2);
      if (page >= 0) entry = (page << a.page_log2) + (slot & low);
    }
    a.map[i] = entry;
  }
}

// 16 bytes of a row of K and of V per lane; a row's lanes lie side by side.
__global__ __launch_bounds__(256) void page_store(PageStoreArgs a, int lanes_log2) {
  const int lanes = 1 << lanes_log2;
  const long long id = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
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
  const uint4 k = load16(static_cast<const char*>(a.K_rows) + src), v = load16(static_cast<const char*>(a.V_rows) + src);
  *reinterpret_cast<uint4*>(static_cast<char*>(a.K) + dst) = k;
  *reinterpret_cast<uint4*>(static_cast<char*>(a.V) + dst) = v;
}

}  // namespace

hipError_t launch_page_tables(const PageTableArgs& a, hipStream_t s) {
  ProfScope ps(kProfPageTables, s);
  hipLaunchKernelGGL(page_sums, dim3(1), dim3(kTableThreads), 0, s, a);
  const long long total = a.padded ? static_cast<long long>(a.requests) * a.rows : a.rows;
  const int map_blocks = static_cast<int>((total + kMapPerBlock - 1) / kMapPerBlock);
  hipLaunchKernelGGL(page_fill, dim3(map_blocks + a.requests), dim3(256), 0, s, a, map_blocks);
  return hipGetLastError();
}

hipError_t launch_page_store(const PageStoreArgs& a, hipStream_t s) {
  ProfScope ps(kProfPageStore, s);
  const int lanes_log2 = __builtin_ctz(a.row_bytes) - 4;
  const long long lanes = (static_cast<long long>(a.groups) * a.heads * a.rows) << lanes_log2;
  hipLaunchKernelGGL(page_store, dim3(static_cast<unsigned>((lanes + 255) / 256)), dim3(256), 0, s, a, lanes_log2);
  return hipGetLastError();
}

}  // namespace roco
