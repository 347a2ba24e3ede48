// Page operations of the paged cache: copy, fork, reserve (with copy on write), free, compact.
//
// Their integer work is small (a table, a count per page); what costs is the pages' bytes, 2 x page bytes x layers for
// each copied page.  The state is on the device, so a plan kernel of one CTA decides (its order is the documented
// one: rows ascending, lowest free page first) and a copy kernel over all SMs moves what the plan lists.
#include "akv_paged.cuh"

namespace akv {
namespace {

constexpr int kPlanThreads = 1024;

// Workspace: counters, then lists of the pool's and the table's size.
struct PagesWs {
  int32_t* n_copies;  // [0]: pairs in src / dst
  int32_t* src;       // [max(n_pages, rows)]
  int32_t* dst;
  int32_t* free;      // [n_pages] free pages taken, ascending; compaction: where a live page goes
  int32_t* writers;   // [n_pages] requests that write into a page
  int32_t* lowest;    // [n_pages] the lowest of them
  int32_t* base;      // [rows] pages taken by the rows before
  int32_t* cbase;     // [rows] copies by the rows before
  int32_t* given;     // [n_pages] the page that a free page taken stands in for, -1: none
};

size_t pages_ws_ints(const PagesState& s) {
  const size_t list = (size_t)(s.n_pages > s.rows ? s.n_pages : s.rows);
  return 64 + 2 * list + 4 * (size_t)s.n_pages + 2 * (size_t)s.rows;
}
PagesWs pages_ws(const PagesState& s, void* ws) {
  const size_t list = (size_t)(s.n_pages > s.rows ? s.n_pages : s.rows);
  int32_t* p = (int32_t*)ws;
  PagesWs w;
  w.n_copies = p;
  w.src = p + 64;
  w.dst = w.src + list;
  w.free = w.dst + list;
  w.writers = w.free + s.n_pages;
  w.lowest = w.writers + s.n_pages;
  w.base = w.lowest + s.n_pages;
  w.cbase = w.base + s.rows;
  w.given = w.cbase + s.rows;
  return w;
}

__device__ __forceinline__ bool in_pool(const PagesState& s, int page) { return (uint32_t)page < (uint32_t)s.n_pages; }

// Exclusive prefix sum over the CTA's threads of x; *total: the sum.  All threads call it.
__device__ __forceinline__ int block_scan(int x, int* total) {
  __shared__ int part[33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int inc = x;
#pragma unroll
  for (int h = 1; h < 32; h *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, inc, h);
    if (lane >= h) inc += o;
  }
  __syncthreads();  // part of the call before has been read
  if (lane == 31) part[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    const int mine = lane < warps ? part[lane] : 0;
    int p = mine;
#pragma unroll
    for (int h = 1; h < 32; h *= 2) {
      const int o = __shfl_up_sync(0xffffffffu, p, h);
      if (lane >= h) p += o;
    }
    part[lane] = p - mine;
    if (lane == 31) part[32] = p;
  }
  __syncthreads();
  *total = part[32];
  return part[warp] + inc - x;
}

// Goes over pages lo .. hi - 1 in order, four neighbouring ones a thread, until `most` of them have been found: found(at,
// page) for the at-th page that `is` holds of, other(page) for the rest.  All threads call it; returns how many there are.
template <class Is, class Found, class Other>
__device__ __forceinline__ int each_page(int lo, int hi, int most, Is is, Found found, Other other) {
  int n = 0;
  for (int p0 = lo; p0 < hi && n < most; p0 += 4 * blockDim.x) {
    const int first = p0 + 4 * threadIdx.x;
    uint32_t flags = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (first + k < hi && is(first + k)) flags |= 1u << k;
    int sum;
    int at = n + block_scan(__popc(flags), &sum);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (first + k < hi) {
        if (flags >> k & 1) found(at++, first + k);
        else other(first + k);
      }
    n += sum;
  }
  return n;
}

// Compaction: the table's entries follow the pages (the map is the plan's).
__device__ __forceinline__ void follow_moves(const PagesState& s, int n, const int32_t* map) {
  const int64_t cells = (int64_t)s.rows * s.max_pages, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t k = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; k < cells; k += step) {
    int32_t* cell = s.table + k / s.max_pages * s.table_stride + k % s.max_pages;
    const int page = *cell;
    if (page >= n && page < s.n_pages && map[page] >= 0) *cell = map[page];
  }
}

// Pair i of the lists, page copied in every layer: a unit of work is 16 KiB of one page in one layer.  Bound by memory:
// 4 layers of 2.6 thousand pages of 78 KB, 1.66 GB read and written, take 260 us (6.4 TB/s, 94 % of the measured rate).
constexpr int kCopyThreads = 256, kCopyChunk = kCopyThreads * 4 * 16;
__global__ void __launch_bounds__(kCopyThreads) akv_pages_copy_kernel(PagesState s, const int32_t* src, const int32_t* dst, int n,
                                                                      const int32_t* n_dev, const int32_t* n_live, const int32_t* map) {
  launch_dependents();
  wait_for_stream();
  if (map) follow_moves(s, *n_live, map);
  if (n_dev) n = *n_dev;
  const int chunks = (int)((s.page_bytes + kCopyChunk - 1) / kCopyChunk);
  const int64_t work = (int64_t)n * s.n_layers * chunks;
  for (int64_t k = blockIdx.x; k < work; k += gridDim.x) {
    const int c = (int)(k % chunks);
    const int64_t pl = k / chunks;
    const int layer = (int)(pl % s.n_layers);
    const int i = (int)(pl / s.n_layers);
    const int a = src[i], b = dst[i];
    if (!in_pool(s, a) || !in_pool(s, b) || a == b) continue;
    uint8_t* base = s.pool + (uint64_t)layer * s.layer_stride;
    const uint4* from = (const uint4*)(base + (uint64_t)a * s.page_bytes);
    uint4* to = (uint4*)(base + (uint64_t)b * s.page_bytes);
    const int64_t units = (int64_t)(s.page_bytes / 16), at = (int64_t)c * (kCopyChunk / 16) + threadIdx.x;
    uint4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j * kCopyThreads < units) x[j] = from[at + j * kCopyThreads];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j * kCopyThreads < units) to[at + j * kCopyThreads] = x[j];
  }
}

__global__ void __launch_bounds__(256) akv_pages_fork_kernel(PagesState s, const int32_t* src, const int32_t* dst) {
  launch_dependents();
  wait_for_stream();
  const int a = src[blockIdx.x], b = dst[blockIdx.x];
  if ((uint32_t)a >= (uint32_t)s.rows || (uint32_t)b >= (uint32_t)s.rows || a == b) return;
  const int len = min(max(s.lens[a], 0), s.max_pages << s.page_log);
  const int held = (len + (1 << s.page_log) - 1) >> s.page_log;
  for (int j = threadIdx.x; j < s.max_pages; j += blockDim.x) {
    int page = -1;
    if (j < held) {
      page = s.table[(int64_t)a * s.table_stride + j];
      if (in_pool(s, page)) atomicAdd(s.refs + page, 1);
    }
    s.table[(int64_t)b * s.table_stride + j] = page;
  }
  if (threadIdx.x == 0) s.lens[b] = s.lens[a];
}

// A page of the row is given up by the one thread that takes it out of the table.
__global__ void __launch_bounds__(256) akv_pages_free_kernel(PagesState s, const int32_t* rows) {
  launch_dependents();
  wait_for_stream();
  const int r = rows[blockIdx.x];
  if ((uint32_t)r >= (uint32_t)s.rows) return;
  for (int j = threadIdx.x; j < s.max_pages; j += blockDim.x) {
    const int page = atomicExch(s.table + (int64_t)r * s.table_stride + j, -1);
    if (in_pool(s, page)) atomicSub(s.refs + page, 1);
  }
  if (threadIdx.x == 0) s.lens[r] = 0;
}

struct RowPlan {
  int first, need;  // table positions that the new tokens fall into
  bool cut;         // the first of them holds tokens of the row already
};
__device__ __forceinline__ RowPlan row_plan(const PagesState& s, const int32_t* n_new, int r) {
  const int most = s.max_pages << s.page_log, P = 1 << s.page_log;
  const int len = min(max(s.lens[r], 0), most);
  const int n = min(max(n_new[r], 0), most - len);
  RowPlan p;
  p.first = len >> s.page_log;
  p.need = n > 0 ? (len + n + P - 1) >> s.page_log : p.first;
  p.cut = len & P - 1;
  return p;
}
// A position without a page gets one, but where it should hold tokens already (they stay missing).
__device__ __forceinline__ bool lacks(const RowPlan& p, int j, int page) { return page < 0 && !(p.cut && j == p.first); }

__global__ void __launch_bounds__(kPlanThreads) akv_pages_reserve_kernel(PagesState s, const int32_t* n_new, int32_t* missing, PagesWs w) {
  launch_dependents();
  wait_for_stream();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  // Who writes into a page that others may hold too: each position that new tokens fall into, the first of a row (all there
  // is in a decode step) by a thread, later ones, which a row has pages at already if its length was lowered, by a warp.
  auto each_cell = [&](auto f) {
    bool more = false;
    for (int r = tid; r < s.rows; r += blockDim.x) {
      const RowPlan p = row_plan(s, n_new, r);
      if (p.first < p.need) f(r, s.table[(int64_t)r * s.table_stride + p.first]);
      more = more || p.need - p.first > 1;
    }
    if (__syncthreads_or(more))
      for (int r = warp; r < s.rows; r += warps) {
        const RowPlan p = row_plan(s, n_new, r);
        for (int j = p.first + 1 + lane; j < p.need; j += 32) f(r, s.table[(int64_t)r * s.table_stride + j]);
      }
    __syncthreads();
  };
  each_cell([&](int, int page) {
    if (in_pool(s, page)) w.writers[page] = 0, w.lowest[page] = INT32_MAX;
  });
  each_cell([&](int r, int page) {
    if (in_pool(s, page)) atomicAdd(w.writers + page, 1), atomicMin(w.lowest + page, r);
  });
  auto gives = [&](int r, int page) {  // the row leaves the page to its other holders
    if (!in_pool(s, page)) return false;
    const int refs = s.refs[page];
    return refs > 1 && !(w.writers[page] == refs && w.lowest[page] == r);
  };
  // pages per row (a warp each)
  for (int r = warp; r < s.rows; r += warps) {
    const RowPlan p = row_plan(s, n_new, r);
    int n = 0;
    bool c = false;
    for (int j = p.first + lane; j < p.need; j += 32) {
      const int page = s.table[(int64_t)r * s.table_stride + j];
      const bool give = gives(r, page);
      n += lacks(p, j, page) || give;
      if (j == p.first) c = give && p.cut;
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
      w.base[r] = n;
      w.cbase[r] = c;
    }
  }
  __syncthreads();
  int total = 0, n_copies = 0;
  for (int r0 = 0; r0 < s.rows; r0 += blockDim.x) {
    const int r = r0 + tid;
    int sum;
    const int a = block_scan(r < s.rows ? w.base[r] : 0, &sum);
    if (r < s.rows) w.base[r] = total + a;
    total += sum;
    const int b = block_scan(r < s.rows ? w.cbase[r] : 0, &sum);
    if (r < s.rows) w.cbase[r] = n_copies + b;
    n_copies += sum;
  }
  const int found = each_page(0, s.n_pages, total, [&](int page) { return s.refs[page] == 0; },
                              [&](int at, int page) { w.free[at] = page; }, [](int) {});  // the lowest free pages
  __syncthreads();
  if (tid == 0) {
    *missing = max(0, total - found);
    *w.n_copies = found < total ? 0 : n_copies;
  }
  if (found < total) return;
  for (int r = warp; r < s.rows; r += warps) {
    const RowPlan p = row_plan(s, n_new, r);
    int at = w.base[r];
    for (int j0 = p.first; j0 < p.need; j0 += 32) {
      const int j = j0 + lane;
      int32_t* cell = s.table + (int64_t)r * s.table_stride + j;
      const int was = j < p.need ? *cell : 0;
      const bool give = j < p.need && gives(r, was), want = j < p.need && (lacks(p, j, was) || give);
      const uint32_t m = __ballot_sync(0xffffffffu, want);
      if (want) {
        const int k = at + __popc(m & ((1u << lane) - 1)), page = w.free[k];
        *cell = page;
        s.refs[page] = 1;
        w.given[k] = give ? was : -1;
        if (give && j == p.first && p.cut) {
          w.src[w.cbase[r]] = was;
          w.dst[w.cbase[r]] = page;
        }
      }
      at += __popc(m);
    }
  }
  __syncthreads();
  // a page that was left has one holder less (after every row has read the counts)
  for (int i = tid; i < total; i += blockDim.x)
    if (w.given[i] >= 0) atomicSub(s.refs + w.given[i], 1);
}

__global__ void __launch_bounds__(kPlanThreads) akv_pages_compact_plan(PagesState s, int32_t* n_live, PagesWs w) {
  launch_dependents();
  wait_for_stream();
  const int tid = threadIdx.x;
  int live = 0, n;
  for (int p = tid; p < s.n_pages; p += blockDim.x) live += s.refs[p] > 0;
  block_scan(live, &n);
  // free pages below n, then live ones at n and above: as many of each
  const int holes = each_page(0, n, INT32_MAX, [&](int page) { return s.refs[page] <= 0; },
                              [&](int at, int page) { w.dst[at] = page; }, [](int) {});
  __syncthreads();
  each_page(n, s.n_pages, INT32_MAX, [&](int page) { return s.refs[page] > 0; },
            [&](int at, int page) { w.src[at] = page, w.free[page] = w.dst[at]; }, [&](int page) { w.free[page] = -1; });
  __syncthreads();
  for (int i = tid; i < holes; i += blockDim.x) {
    s.refs[w.dst[i]] = s.refs[w.src[i]];
    s.refs[w.src[i]] = 0;
  }
  if (tid == 0) *n_live = n, *w.n_copies = holes;
}

constexpr int kCopyGrid = 152 * 8;

}  // namespace

size_t pages_ws_bytes(const PagesState& s) { return (pages_ws_ints(s) * 4 + 255) & ~(size_t)255; }

int launch_pages_copy(const PagesState& s, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  return launch_after(akv_pages_copy_kernel, dim3(kCopyGrid), kCopyThreads, 0, stream, s, src, dst, n, nullptr, nullptr, nullptr);
}

int launch_pages_fork(const PagesState& s, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  return launch_after(akv_pages_fork_kernel, dim3(n), 256, 0, stream, s, src, dst);
}

int launch_pages_free(const PagesState& s, const int32_t* rows, int32_t n, void* stream) {
  return launch_after(akv_pages_free_kernel, dim3(n), 256, 0, stream, s, rows);
}

int launch_pages_reserve(const PagesState& s, const int32_t* n_new, int32_t* missing, void* ws, void* stream) {
  const PagesWs w = pages_ws(s, ws);
  const int e = launch_after(akv_pages_reserve_kernel, dim3(1), kPlanThreads, 0, stream, s, n_new, missing, w);
  if (e) return e;
  return launch_after(akv_pages_copy_kernel, dim3(kCopyGrid), kCopyThreads, 0, stream, s, w.src, w.dst, 0, w.n_copies, nullptr, nullptr);
}

int launch_pages_compact(const PagesState& s, int32_t* n_live, void* ws, void* stream) {
  const PagesWs w = pages_ws(s, ws);
  const int e = launch_after(akv_pages_compact_plan, dim3(1), kPlanThreads, 0, stream, s, n_live, w);
  if (e) return e;
  return launch_after(akv_pages_copy_kernel, dim3(kCopyGrid), kCopyThreads, 0, stream, s, w.src, w.dst, 0, w.n_copies, n_live, w.free);
}

}  // namespace akv
