// Host side of the paged cache's entry points: validation, and the views the kernels get.
#include <algorithm>
#include <cmath>
#include <utility>

#include "akv_internal.h"

namespace akv {
namespace {

struct PagedCall {
  PagedView v{};
  uint64_t page_bytes = 0;
};

akv_status check_params(const akv_paged_params* p, PagedCall* c) {
  if (!p) return fail(AKV_ERR_INVALID, "null params");
  if (p->head_dim != kD) return fail(AKV_ERR_UNSUPPORTED, "head_dim must be 128");
  if (p->n_kv_heads < 1 || p->n_q_heads < 1) return fail(AKV_ERR_INVALID, "n_kv_heads and n_q_heads must be >= 1");
  if (p->n_q_heads % p->n_kv_heads != 0) return fail(AKV_ERR_INVALID, "n_q_heads must be a multiple of n_kv_heads");
  if (p->n_kv_heads > 256 || p->n_q_heads / p->n_kv_heads > 64)
    return fail(AKV_ERR_UNSUPPORTED, "at most 256 KV heads and 64 query heads per KV head");
  int lg = 4;
  while (lg < 7 && (1 << lg) != p->page_tokens) ++lg;
  if ((1 << lg) != p->page_tokens) return fail(AKV_ERR_UNSUPPORTED, "page_tokens must be 16, 32, 64 or 128");
  if (p->group != 64 && p->group != 128) return fail(AKV_ERR_UNSUPPORTED, "group must be 64 or 128");
  if (p->dtype != AKV_DTYPE_BF16 && p->dtype != AKV_DTYPE_FP16) return fail(AKV_ERR_UNSUPPORTED, "dtype must be bf16 or fp16");
  if (p->flags & ~(AKV_FLAG_ROTATE | AKV_FLAG_BOUNDS)) return fail(AKV_ERR_INVALID, "unknown flags");
  if (p->reserved != 0) return fail(AKV_ERR_INVALID, "reserved must be 0");
  PagedView& v = c->v;
  v.H = p->n_kv_heads;
  v.G = p->n_q_heads / p->n_kv_heads;
  v.page_log = lg;
  v.ng = kD / p->group;
  v.half = p->dtype == AKV_DTYPE_FP16;
  v.rotate = (p->flags & AKV_FLAG_ROTATE) != 0;
  v.bounds = (p->flags & AKV_FLAG_BOUNDS) != 0;
  v.block_bytes = (uint32_t)(p->page_tokens / kSubTokens) * sub_bytes(v.ng) + (v.bounds ? 512u : 0u);
  v.page_bytes = c->page_bytes = (uint64_t)v.block_bytes * (uint64_t)v.H;
  rotation_signs(p->rot_seed, v.sign_bits);
  return AKV_OK;
}

akv_status check_pages(const akv_paged_params* p, const akv_pages* g, PagedCall* c) {
  akv_status st = check_params(p, c);
  if (st != AKV_OK) return st;
  if (!g) return fail(AKV_ERR_INVALID, "null pages");
  if (!g->pool || !g->table || !g->lens) return fail(AKV_ERR_INVALID, "null pool, table or lens");
  if (((uintptr_t)g->pool % 16) || ((uintptr_t)g->table % 4) || ((uintptr_t)g->lens % 4) || ((uintptr_t)g->refs % 4))
    return fail(AKV_ERR_INVALID, "pool must be 16-byte aligned; table, lens and refs 4-byte aligned");
  if (g->n_layers < 1 || g->n_pages < 1 || g->rows < 1 || g->max_pages < 1)
    return fail(AKV_ERR_INVALID, "n_layers, n_pages, rows and max_pages must be >= 1");
  if (g->table_stride < g->max_pages) return fail(AKV_ERR_INVALID, "table_stride must be >= max_pages");
  // token positions are 32-bit, and a round up to the next tile stays inside them
  if ((int64_t)g->max_pages * p->page_tokens > (1 << 30)) return fail(AKV_ERR_UNSUPPORTED, "more than 2^30 tokens per request");
  if ((int64_t)g->rows * p->n_kv_heads > (1 << 22)) return fail(AKV_ERR_UNSUPPORTED, "too many requests and heads");
  if ((int64_t)g->rows * g->max_pages > INT32_MAX) return fail(AKV_ERR_UNSUPPORTED, "table of more than 2^31 - 1 pages");
  const uint64_t layer = (uint64_t)g->n_pages * c->page_bytes;
  if (g->n_layers > 1 && ((g->layer_stride % 16) || g->layer_stride < layer))
    return fail(AKV_ERR_INVALID, "layer_stride must be a multiple of 16 and hold n_pages pages");
  if (g->n_layers > 1 && (uint64_t)(g->n_layers - 1) > (~0ull - layer) / g->layer_stride)
    return fail(AKV_ERR_INVALID, "layer_stride out of range");
  if (g->pool_bytes < layer + (g->n_layers > 1 ? (uint64_t)(g->n_layers - 1) * g->layer_stride : 0))
    return fail(AKV_ERR_TOO_SMALL, "pool shorter than its layers and pages");
  PagedView& v = c->v;
  v.base = (uint8_t*)g->pool;
  v.table = g->table;
  v.lens = g->lens;
  v.refs = g->refs;
  v.table_stride = g->table_stride;
  v.n_pages = g->n_pages;
  v.rows = g->rows;
  v.max_pages = g->max_pages;
  return AKV_OK;
}

akv_status check_layer(const akv_paged_params* p, const akv_pages* g, int32_t layer, PagedCall* c) {
  akv_status st = check_pages(p, g, c);
  if (st != AKV_OK) return st;
  if (layer < 0 || layer >= g->n_layers) return fail(AKV_ERR_INVALID, "layer out of range");
  if (layer) c->v.base += (uint64_t)layer * g->layer_stride;
  return AKV_OK;
}

akv_status check_rows(const akv_rows* r, const char* what) {
  if (!r || !r->ptr) return fail(AKV_ERR_INVALID, "null ", what);
  if ((uintptr_t)r->ptr % 2) return fail(AKV_ERR_INVALID, what, " must be 2-byte aligned");
  if (r->stride_b < 0 || r->stride_t < 0 || r->stride_h < 0) return fail(AKV_ERR_INVALID, what, ": negative stride");
  return AKV_OK;
}

akv_status check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || ((uintptr_t)ws % 256)) return fail(AKV_ERR_INVALID, "workspace must be non-null and 256-byte aligned");
  if (have < need) return fail(AKV_ERR_TOO_SMALL, "workspace shorter than its size call says");
  return AKV_OK;
}

akv_status check_query(int32_t T) {
  if (T < 1 || T > AKV_PAGED_MAX_QUERY) return fail(AKV_ERR_UNSUPPORTED, "1 to 64 query tokens per request");
  return AKV_OK;
}

akv_status check_selection(const akv_selection* s) {
  if (!s->pages || !s->count) return fail(AKV_ERR_INVALID, "selection: null pages or count");
  if (((uintptr_t)s->pages % 4) || ((uintptr_t)s->count % 4)) return fail(AKV_ERR_INVALID, "selection must be 4-byte aligned");
  if (s->top < 1 || s->top > (1 << 20)) return fail(AKV_ERR_INVALID, "selection: top must be in 1 .. 2^20");
  return AKV_OK;
}

// Rows to write T tokens of: rows on top of one another are refused.  Axes are taken from the smallest stride up, each
// has to step over all that lies within the ones before.
akv_status check_written(const akv_rows* r, const char* what, int32_t rows, int32_t T, int32_t heads) {
  akv_status st = check_rows(r, what);
  if (st != AKV_OK) return st;
  struct Axis {
    int64_t stride, n;
  } axes[3] = {{r->stride_b, rows}, {r->stride_t, T}, {r->stride_h, heads}};
  if (axes[1].stride < axes[0].stride) std::swap(axes[0], axes[1]);
  if (axes[2].stride < axes[1].stride) std::swap(axes[1], axes[2]);
  if (axes[1].stride < axes[0].stride) std::swap(axes[0], axes[1]);
  int64_t extent = kD;  // values from the first row's start to the last one's end
  for (const Axis& a : axes) {
    if (a.n <= 1) continue;
    if (a.stride < extent) return fail(AKV_ERR_INVALID, what, ": rows overlap");
    if (a.stride > (INT64_MAX / 2 - extent) / (a.n - 1)) return fail(AKV_ERR_INVALID, what, ": strides out of range");
    extent += a.stride * (a.n - 1);
  }
  return AKV_OK;
}

akv_status check_state(const akv_paged_params* p, const akv_pages* g, bool refs, PagesState* s) {
  PagedCall c;
  akv_status st = check_pages(p, g, &c);
  if (st != AKV_OK) return st;
  if (refs && !g->refs) return fail(AKV_ERR_INVALID, "null refs");
  s->table = g->table;
  s->lens = g->lens;
  s->refs = g->refs;
  s->table_stride = g->table_stride;
  s->pool = (uint8_t*)g->pool;
  s->layer_stride = g->n_layers > 1 ? g->layer_stride : 0;
  s->page_bytes = c.page_bytes;
  s->n_layers = g->n_layers;
  s->n_pages = g->n_pages;
  s->rows = g->rows;
  s->max_pages = g->max_pages;
  s->page_log = c.v.page_log;
  return AKV_OK;
}

akv_status check_list(const int32_t* a, const int32_t* b, int32_t n) {
  if (n < 0) return fail(AKV_ERR_INVALID, "negative count");
  if (n && (!a || !b)) return fail(AKV_ERR_INVALID, "null list");
  if (((uintptr_t)a % 4) || ((uintptr_t)b % 4)) return fail(AKV_ERR_INVALID, "lists must be 4-byte aligned");
  return AKV_OK;
}

akv_status check_share(const akv_share* s, const akv_pages* g) {
  // (every row's place among the others is counted)
  if (g->rows > (1 << 16)) return fail(AKV_ERR_UNSUPPORTED, "share: more than 2^16 rows");
  if (!s || !s->leader || !s->pages || !s->size || !s->order) return fail(AKV_ERR_INVALID, "null share or array of it");
  if (((uintptr_t)s->leader | (uintptr_t)s->pages | (uintptr_t)s->size | (uintptr_t)s->order) % 4)
    return fail(AKV_ERR_INVALID, "share must be 4-byte aligned");
  if (s->flags & ~AKV_SHARE_ALWAYS) return fail(AKV_ERR_INVALID, "share: unknown flags");
  return AKV_OK;
}

akv_status check_scores(const akv_scores* s, const char* what, const akv_pages* g, const akv_paged_params* p, bool written) {
  if (!s || !s->ptr) return fail(AKV_ERR_INVALID, "null ", what);
  if ((uintptr_t)s->ptr % 4) return fail(AKV_ERR_INVALID, what, " must be 4-byte aligned");
  if (s->cap < g->max_pages * p->page_tokens) return fail(AKV_ERR_TOO_SMALL, what, ": room for max_pages * page_tokens numbers a head");
  if (s->stride_b < 0 || s->stride_h < 0) return fail(AKV_ERR_INVALID, what, ": negative stride");
  if (!written) {
    const int64_t most = INT64_MAX / 16;
    if ((g->rows > 1 && s->stride_b > most / (g->rows - 1)) || (p->n_kv_heads > 1 && s->stride_h > most / (p->n_kv_heads - 1)))
      return fail(AKV_ERR_INVALID, what, ": strides out of range");
    return AKV_OK;
  }
  // numbers on top of one another: the smaller stride steps over a head's, the larger over all of the smaller's axis
  int64_t near = s->stride_h, far = s->stride_b, n = p->n_kv_heads, m = g->rows;
  if (far < near) std::swap(near, far), std::swap(n, m);
  int64_t extent = s->cap;
  for (int i = 0; i < 2; ++i) {
    const int64_t stride = i ? far : near, count = i ? m : n;
    if (count <= 1) continue;
    if (stride < extent) return fail(AKV_ERR_INVALID, what, ": heads' numbers overlap");
    if (stride > (INT64_MAX / 8 - extent) / (count - 1)) return fail(AKV_ERR_INVALID, what, ": strides out of range");
    extent += stride * (count - 1);
  }
  return AKV_OK;
}

// Numbers of `was` are read while those of `now` are written: each head's n of them have to be that head's of `now`, or on none of
// its.  Both have been checked, so that heads of `now` do not overlap, those of the smaller stride within a step of the larger.
bool apart(const akv_scores& was, const akv_scores& now, int64_t rows, int64_t heads, int64_t n) {
  const int64_t d = (int64_t)((uintptr_t)was.ptr - (uintptr_t)now.ptr) / 4;
  if (d == 0 && (rows == 1 || was.stride_b == now.stride_b) && (heads == 1 || was.stride_h == now.stride_h)) return true;
  auto extent = [&](const akv_scores& s) { return (rows - 1) * s.stride_b + (heads - 1) * s.stride_h + n; };
  if (d >= extent(now) || -d >= extent(was)) return true;
  struct Axis {
    int64_t stride, count;
    // the steps in which places x .. x + n - 1 may lie (n is no longer than one)
    int64_t step(int64_t x) const { return count == 1 ? 0 : x < 0 ? -1 : x / stride; }
  } b_axis{now.stride_b, rows}, h_axis{now.stride_h, heads};
  const bool b_far = heads == 1 || (rows > 1 && b_axis.stride >= h_axis.stride);
  const Axis &far = b_far ? b_axis : h_axis, &near = b_far ? h_axis : b_axis;
  for (int64_t b = 0; b < rows; ++b)
    for (int64_t h = 0; h < heads; ++h) {
      const int64_t x = d + b * was.stride_b + h * was.stride_h;
      for (int64_t f = std::max<int64_t>(0, far.step(x)); f <= std::min(far.count - 1, far.step(x + n - 1)); ++f) {
        const int64_t y = far.count == 1 ? x : x - f * far.stride;
        for (int64_t k = std::max<int64_t>(0, near.step(y)); k <= std::min(near.count - 1, near.step(y + n - 1)); ++k) {
          const int64_t off = near.count == 1 ? y : y - k * near.stride;
          if (off > -n && off < n && (off != 0 || (b_far ? f : k) != b || (b_far ? k : f) != h)) return false;
        }
      }
    }
  return true;
}

akv_status launched(int err, const char* what) {
  if (err) return fail(AKV_ERR_CUDA, what, " launch failed: ", cuda_error_string(err));
  return AKV_OK;
}

#define AKV_TRY(x)                     \
  do {                                 \
    const akv_status st_ = (x);        \
    if (st_ != AKV_OK) return st_;     \
  } while (0)

}  // namespace
}  // namespace akv

using namespace akv;

extern "C" {

akv_status akv_paged_page_bytes(const akv_paged_params* p, size_t* bytes) {
  PagedCall c;
  AKV_TRY(check_params(p, &c));
  if (!bytes) return fail(AKV_ERR_INVALID, "null bytes");
  *bytes = (size_t)c.page_bytes;
  return AKV_OK;
}

akv_status akv_paged_append(const akv_paged_params* p, const akv_pages* pages, int32_t layer, const akv_rows* K,
                            const akv_rows* V, int32_t T, const int32_t* n_new, akv_stream_t stream) {
  PagedCall c;
  AKV_TRY(check_layer(p, pages, layer, &c));
  if (T < 0) return fail(AKV_ERR_INVALID, "negative T");
  if (T == 0) return AKV_OK;  // (empty tensors have no address)
  AKV_TRY(check_rows(K, "K"));
  AKV_TRY(check_rows(V, "V"));
  if ((uintptr_t)n_new % 4) return fail(AKV_ERR_INVALID, "n_new must be 4-byte aligned");
  return launched(launch_paged_append(c.v, *K, *V, T, n_new, (void*)stream), "append");
}

akv_status akv_paged_read(const akv_paged_params* p, const akv_pages* pages, int32_t layer, const int32_t* start,
                          const akv_rows* K, const akv_rows* V, int32_t T, akv_stream_t stream) {
  PagedCall c;
  AKV_TRY(check_layer(p, pages, layer, &c));
  if (T < 0) return fail(AKV_ERR_INVALID, "negative T");
  if (T == 0) return AKV_OK;
  if (T > (1 << 30)) return fail(AKV_ERR_UNSUPPORTED, "more than 2^30 tokens per request");  // (32-bit token numbers)
  AKV_TRY(check_written(K, "K", pages->rows, T, p->n_kv_heads));
  AKV_TRY(check_written(V, "V", pages->rows, T, p->n_kv_heads));
  if ((uintptr_t)start % 4) return fail(AKV_ERR_INVALID, "start must be 4-byte aligned");
  return launched(launch_paged_read(c.v, start, *K, *V, T, (void*)stream), "read");
}

akv_status akv_paged_attn_workspace_size(const akv_paged_params* p, const akv_pages* pages, int32_t T, int32_t top,
                                         size_t* ws_bytes) {
  PagedCall c;
  AKV_TRY(check_pages(p, pages, &c));
  AKV_TRY(check_query(T));
  if (!ws_bytes) return fail(AKV_ERR_INVALID, "null ws_bytes");
  if (top < 0) return fail(AKV_ERR_INVALID, "negative top");
  *ws_bytes = paged_attn_ws_bytes(c.v, T, top);
  return AKV_OK;
}

akv_status akv_paged_attn(const akv_paged_params* p, const akv_pages* pages, int32_t layer, const akv_rows* q,
                          const akv_rows* out, float* lse, int32_t T, float sm_scale, const akv_selection* sel,
                          void* ws, size_t ws_bytes, akv_stream_t stream) {
  PagedCall c;
  AKV_TRY(check_layer(p, pages, layer, &c));
  AKV_TRY(check_query(T));
  AKV_TRY(check_rows(q, "q"));
  AKV_TRY(check_written(out, "out", pages->rows, T, p->n_q_heads));
  if ((uintptr_t)lse % 4) return fail(AKV_ERR_INVALID, "lse must be 4-byte aligned");
  if (!std::isfinite(sm_scale)) return fail(AKV_ERR_INVALID, "sm_scale must be finite");
  if (sel) AKV_TRY(check_selection(sel));
  AKV_TRY(check_ws(ws, ws_bytes, paged_attn_ws_bytes(c.v, T, sel ? sel->top : 0)));
  return launched(launch_paged_attn(c.v, *q, *out, lse, T, sm_scale, sel, ws, (void*)stream), "attention");
}

akv_status akv_paged_select_workspace_size(const akv_paged_params* p, const akv_pages* pages, int32_t T,
                                           size_t* ws_bytes) {
  PagedCall c;
  AKV_TRY(check_pages(p, pages, &c));
  AKV_TRY(check_query(T));
  if (!ws_bytes) return fail(AKV_ERR_INVALID, "null ws_bytes");
  *ws_bytes = paged_select_ws_bytes(c.v, T);
  return AKV_OK;
}

akv_status akv_paged_select(const akv_paged_params* p, const akv_pages* pages, int32_t layer, const akv_rows* q,
                            int32_t T, int32_t sink, int32_t recent, const akv_selection* sel, void* ws,
                            size_t ws_bytes, akv_stream_t stream) {
  PagedCall c;
  AKV_TRY(check_layer(p, pages, layer, &c));
  AKV_TRY(check_query(T));
  if (!c.v.bounds) return fail(AKV_ERR_INVALID, "the cache has no bounds (AKV_FLAG_BOUNDS)");
  AKV_TRY(check_rows(q, "q"));
  if (!sel) return fail(AKV_ERR_INVALID, "null selection");
  AKV_TRY(check_selection(sel));
  if (sink < 0 || recent < 0 || (int64_t)sink + recent > sel->top)
    return fail(AKV_ERR_INVALID, "sink and recent must be >= 0 and together at most top");
  AKV_TRY(check_ws(ws, ws_bytes, paged_select_ws_bytes(c.v, T)));
  return launched(launch_paged_select(c.v, *q, T, sink, recent, *sel, ws, (void*)stream), "selection");
}

akv_status akv_pages_share(const akv_paged_params* p, const akv_pages* pages, const akv_share* share, void* ws,
                           size_t ws_bytes, akv_stream_t stream) {
  PagesState s;
  AKV_TRY(check_state(p, pages, false, &s));
  AKV_TRY(check_share(share, pages));
  AKV_TRY(check_ws(ws, ws_bytes, pages_ws_bytes(s)));
  return launched(launch_pages_share(s, *share, ws, (void*)stream), "share");
}

akv_status akv_paged_attn_shared_workspace_size(const akv_paged_params* p, const akv_pages* pages, int32_t T,
                                                size_t* ws_bytes) {
  PagedCall c;
  AKV_TRY(check_pages(p, pages, &c));
  AKV_TRY(check_query(T));
  if (!ws_bytes) return fail(AKV_ERR_INVALID, "null ws_bytes");
  *ws_bytes = paged_shared_ws_bytes(c.v, T);
  return AKV_OK;
}

akv_status akv_paged_attn_shared(const akv_paged_params* p, const akv_pages* pages, int32_t layer, const akv_rows* q,
                                 const akv_rows* out, float* lse, int32_t T, float sm_scale, const akv_share* share,
                                 void* ws, size_t ws_bytes, akv_stream_t stream) {
  PagedCall c;
  AKV_TRY(check_layer(p, pages, layer, &c));
  AKV_TRY(check_query(T));
  AKV_TRY(check_rows(q, "q"));
  AKV_TRY(check_written(out, "out", pages->rows, T, p->n_q_heads));
  if ((uintptr_t)lse % 4) return fail(AKV_ERR_INVALID, "lse must be 4-byte aligned");
  if (!std::isfinite(sm_scale)) return fail(AKV_ERR_INVALID, "sm_scale must be finite");
  AKV_TRY(check_share(share, pages));
  AKV_TRY(check_ws(ws, ws_bytes, paged_shared_ws_bytes(c.v, T)));
  return launched(launch_paged_shared(c.v, *q, *out, lse, T, sm_scale, *share, ws, (void*)stream), "shared attention");
}

akv_status akv_paged_weights_workspace_size(const akv_paged_params* p, const akv_pages* pages, int32_t T, size_t* ws_bytes) {
  PagedCall c;
  AKV_TRY(check_pages(p, pages, &c));
  AKV_TRY(check_query(T));
  if (!ws_bytes) return fail(AKV_ERR_INVALID, "null ws_bytes");
  *ws_bytes = paged_weights_ws_bytes(c.v, T);
  return AKV_OK;
}

akv_status akv_paged_weights(const akv_paged_params* p, const akv_pages* pages, int32_t layer, const akv_rows* q,
                             const float* lse, int32_t T, float sm_scale, float decay, const akv_scores* was,
                             const akv_scores* now, void* ws, size_t ws_bytes, akv_stream_t stream) {
  PagedCall c;
  AKV_TRY(check_layer(p, pages, layer, &c));
  AKV_TRY(check_query(T));
  AKV_TRY(check_rows(q, "q"));
  if (!lse) return fail(AKV_ERR_INVALID, "null lse");
  if ((uintptr_t)lse % 4) return fail(AKV_ERR_INVALID, "lse must be 4-byte aligned");
  if (!std::isfinite(sm_scale)) return fail(AKV_ERR_INVALID, "sm_scale must be finite");
  if (!std::isfinite(decay)) return fail(AKV_ERR_INVALID, "decay must be finite");
  if (was) AKV_TRY(check_scores(was, "was", pages, p, false));
  AKV_TRY(check_scores(now, "now", pages, p, true));
  if (was && decay != 0.f && !apart(*was, *now, pages->rows, p->n_kv_heads, (int64_t)pages->max_pages * p->page_tokens))
    return fail(AKV_ERR_INVALID, "was lies on other numbers of now");
  AKV_TRY(check_ws(ws, ws_bytes, paged_weights_ws_bytes(c.v, T)));
  return launched(launch_paged_weights(c.v, *q, lse, T, sm_scale, decay, decay != 0.f ? was : nullptr, *now, ws, (void*)stream), "weights");
}

akv_status akv_paged_evict(const akv_paged_params* p, const akv_pages* pages, int32_t layer, const int32_t* src,
                           const int32_t* dst, int32_t n, const akv_scores* scores, const int32_t* keep, int32_t sink,
                           int32_t recent, const akv_kept* kept, akv_stream_t stream) {
  PagedCall c;
  AKV_TRY(check_layer(p, pages, layer, &c));
  if (c.v.bounds) return fail(AKV_ERR_UNSUPPORTED, "a cache with bounds (AKV_FLAG_BOUNDS) cannot evict");
  AKV_TRY(check_list(src, dst, n));
  if ((int64_t)n * p->n_kv_heads > (1 << 22)) return fail(AKV_ERR_UNSUPPORTED, "too many rows and heads");
  AKV_TRY(check_scores(scores, "scores", pages, p, true));
  if ((uintptr_t)keep % 4) return fail(AKV_ERR_INVALID, "keep must be 4-byte aligned");
  if (sink < 0 || recent < 0) return fail(AKV_ERR_INVALID, "sink and recent must be >= 0");
  if (!kept || (n && (!kept->tokens || !kept->count))) return fail(AKV_ERR_INVALID, "null kept or array of it");
  if (((uintptr_t)kept->tokens | (uintptr_t)kept->count) % 4) return fail(AKV_ERR_INVALID, "kept must be 4-byte aligned");
  if (kept->top < 1 || kept->top > (1 << 30)) return fail(AKV_ERR_INVALID, "kept: top must be in 1 .. 2^30");
  if (n == 0) return AKV_OK;
  return launched(launch_paged_evict(c.v, src, dst, n, *scores, keep, sink, recent, *kept, (void*)stream), "eviction");
}

akv_status akv_pages_trim(const akv_paged_params* p, const akv_pages* pages, const int32_t* rows, int32_t n,
                          akv_stream_t stream) {
  PagesState s;
  AKV_TRY(check_state(p, pages, true, &s));
  AKV_TRY(check_list(rows, rows, n));
  if (n == 0) return AKV_OK;
  return launched(launch_pages_trim(s, rows, n, (void*)stream), "trim");
}

akv_status akv_pages_workspace_size(const akv_paged_params* p, const akv_pages* pages, size_t* ws_bytes) {
  PagesState s;
  AKV_TRY(check_state(p, pages, false, &s));
  if (!ws_bytes) return fail(AKV_ERR_INVALID, "null ws_bytes");
  *ws_bytes = pages_ws_bytes(s);
  return AKV_OK;
}

akv_status akv_pages_copy(const akv_paged_params* p, const akv_pages* pages, const int32_t* src, const int32_t* dst,
                          int32_t n, akv_stream_t stream) {
  PagesState s;
  AKV_TRY(check_state(p, pages, false, &s));
  AKV_TRY(check_list(src, dst, n));
  if (n == 0) return AKV_OK;
  return launched(launch_pages_copy(s, src, dst, n, (void*)stream), "page copy");
}

akv_status akv_pages_fork(const akv_paged_params* p, const akv_pages* pages, const int32_t* src, const int32_t* dst,
                          int32_t n, akv_stream_t stream) {
  PagesState s;
  AKV_TRY(check_state(p, pages, true, &s));
  AKV_TRY(check_list(src, dst, n));
  if (n == 0) return AKV_OK;
  return launched(launch_pages_fork(s, src, dst, n, (void*)stream), "fork");
}

akv_status akv_pages_reserve(const akv_paged_params* p, const akv_pages* pages, const int32_t* n_new,
                             int32_t* missing, void* ws, size_t ws_bytes, akv_stream_t stream) {
  PagesState s;
  AKV_TRY(check_state(p, pages, true, &s));
  if (!n_new || !missing) return fail(AKV_ERR_INVALID, "null n_new or missing");
  if (((uintptr_t)n_new % 4) || ((uintptr_t)missing % 4)) return fail(AKV_ERR_INVALID, "n_new and missing must be 4-byte aligned");
  AKV_TRY(check_ws(ws, ws_bytes, pages_ws_bytes(s)));
  return launched(launch_pages_reserve(s, n_new, missing, ws, (void*)stream), "reserve");
}

akv_status akv_pages_free(const akv_paged_params* p, const akv_pages* pages, const int32_t* rows, int32_t n,
                          akv_stream_t stream) {
  PagesState s;
  AKV_TRY(check_state(p, pages, true, &s));
  AKV_TRY(check_list(rows, rows, n));
  if (n == 0) return AKV_OK;
  return launched(launch_pages_free(s, rows, n, (void*)stream), "free");
}

akv_status akv_pages_compact(const akv_paged_params* p, const akv_pages* pages, int32_t* n_live, void* ws,
                             size_t ws_bytes, akv_stream_t stream) {
  PagesState s;
  AKV_TRY(check_state(p, pages, true, &s));
  if (!n_live) return fail(AKV_ERR_INVALID, "null n_live");
  if ((uintptr_t)n_live % 4) return fail(AKV_ERR_INVALID, "n_live must be 4-byte aligned");
  AKV_TRY(check_ws(ws, ws_bytes, pages_ws_bytes(s)));
  return launched(launch_pages_compact(s, n_live, ws, (void*)stream), "compaction");
}

}  // extern "C"
