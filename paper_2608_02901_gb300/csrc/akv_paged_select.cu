// Choice of the pages that a query attends: a score per page in whole numbers, then the best of them.
#include "akv_paged.cuh"

namespace akv {
namespace {

// Exponent e of a finite a > 0 with a = f 2^e, f in [0.5, 1) (0 for a = 0), clamped to +-100.
__device__ __forceinline__ int exponent_of(float a) {
  int e = 0;
  frexpf(a, &e);
  return min(max(e, -100), 100);
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 .. 127
__device__ __forceinline__ int whole(float x, float unit) { return min(max(__float2int_rn(x * unit), -127), 127); }

// Float order as unsigned order (no NaN).
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // one zero
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kScoreWarps = 8;

// One warp: one page of one (request, query token, head).  A lane holds four dimensions.
__global__ void __launch_bounds__(32 * kScoreWarps) akv_paged_score_kernel(PagedView v, const uint16_t* q, int64_t qb, int64_t qt,
                                                                            int64_t qh, int T, uint32_t* keys) {
  const int lane = threadIdx.x & 31;
  const int64_t unit = blockIdx.y;
  const int h = (int)(unit % v.H), t = (int)(unit / v.H % T), b = (int)(unit / v.H / T);
  const int P = 1 << v.page_log;
  const int sees = max(0, held_tokens(v, b) - T + 1 + t), n = (sees + P - 1) >> v.page_log;
  const uint16_t* rows = q + b * qb + t * qt + (int64_t)h * v.G * qh + 4 * lane;
  float top = 0.f;
  for (int g = 0; g < v.G; ++g)
    for (int e = 0; e < 4; ++e) top = max_nan(top, fabsf(row_to_float(rows[g * qh + e], v.half)));
  for (int k = 16; k; k >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, k));
  const bool fine = top <= 3.402823466e38f;
  const float unit_q = power(7 - exponent_of(fine ? top : 0.f));
  for (int j = blockIdx.x * kScoreWarps + (threadIdx.x >> 5); j < n; j += gridDim.x * kScoreWarps) {
    const int page = page_of(v, b, j);
    uint32_t key = order_key(-__int_as_float(0x7f800000));
    if (page >= 0) {
      const uint16_t* bound = (const uint16_t*)(block_of(v, page, h) + (uint32_t)(P >> 4) * sub_bytes(v.ng)) + 4 * lane;
      float lo[4], hi[4], big = 0.f;
      for (int e = 0; e < 4; ++e) {
        lo[e] = row_to_float(bound[e], v.half);
        hi[e] = row_to_float(bound[kD + e], v.half);
        big = max_nan(big, max_nan(fabsf(lo[e]), fabsf(hi[e])));
      }
      for (int k = 16; k; k >>= 1) big = max_nan(big, __shfl_xor_sync(0xffffffffu, big, k));
      if (!(big <= 3.402823466e38f)) {
        key = order_key(__int_as_float(0x7f800000));
      } else {
        const int ep = exponent_of(big);
        const float unit_p = power(7 - ep);
        int best = INT32_MIN;
        for (int g = 0; g < v.G; ++g) {
          int sum = 0;
          for (int e = 0; e < 4; ++e) {
            const int x = fine ? whole(row_to_float(rows[g * qh + e], v.half), unit_q) : 0;
            sum += max(x * whole(lo[e], unit_p), x * whole(hi[e], unit_p));
          }
          best = max(best, __reduce_add_sync(0xffffffffu, sum));
        }
        key = order_key((float)best * power(ep));
      }
    }
    if (lane == 0) keys[unit * v.max_pages + j] = key;
  }
}

constexpr int kPickThreads = 256;

// One CTA: one (request, query token, head).  The key of the last page that is kept is found digit by digit (8 bits at
// a time, from above); pages above it are kept, and of those equal to it the lowest.
__global__ void __launch_bounds__(kPickThreads) akv_paged_pick_kernel(PagedView v, int T, int sink, int recent, const uint32_t* keys,
                                                                      int32_t* sel, int32_t* count, int top) {
  const int64_t unit = blockIdx.x;
  const int t = (int)(unit / v.H % T), b = (int)(unit / v.H / T);
  const int P = 1 << v.page_log, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sees = max(0, held_tokens(v, b) - T + 1 + t), n = (sees + P - 1) >> v.page_log;
  int32_t* out = sel + unit * top;
  const int kept = min(n, top);
  if (tid == 0) count[unit] = kept;
  for (int i = kept + tid; i < top; i += blockDim.x) out[i] = -1;
  if (n <= top) {
    for (int i = tid; i < n; i += blockDim.x) out[i] = i;
    return;
  }
  const uint32_t* key = keys + unit * v.max_pages;
  const int first = sink, last = n - recent;  // pages that the score decides about
  int want = top - sink - recent;             // of them, how many
  __shared__ int hist[256];
  __shared__ int s_digit, s_want;
  __shared__ int part[kPickThreads / 32][2];
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int i = first + tid; i < last; i += blockDim.x) {
      const uint32_t k = key[i];
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(hist + (k >> shift & 255), 1);
    }
    __syncthreads();
    if (tid == 0) {
      int left = want, d = 255;
      while (hist[d] < left) left -= hist[d--];
      s_digit = d;
      s_want = left;
    }
    __syncthreads();
    prefix |= (uint32_t)s_digit << shift;
    want = s_want;
    __syncthreads();
  }
  // prefix: the last kept key; want: how many of those equal to it (none at all where nothing was wanted)
  const bool any = top - sink - recent > 0;
  int at = 0, ties = 0;
  for (int i0 = 0; i0 < n; i0 += blockDim.x) {
    const int i = i0 + tid;
    const bool mid = i >= first && i < last;
    const uint32_t k = mid ? key[i] : 0;
    const bool tie = any && mid && k == prefix;
    const bool sure = i < n && (!mid || (any && k > prefix));
    const uint32_t mt = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) part[warp][0] = __popc(mt);
    __syncthreads();
    int before = ties, all = 0;
    for (int w = 0; w < kPickThreads / 32; ++w) {
      if (w < warp) before += part[w][0];
      all += part[w][0];
    }
    const bool keep = sure || (tie && before + __popc(mt & ((1u << lane) - 1)) < want);
    ties += all;
    const uint32_t mk = __ballot_sync(0xffffffffu, keep);
    if (lane == 0) part[warp][1] = __popc(mk);
    __syncthreads();
    int place = at;
    all = 0;
    for (int w = 0; w < kPickThreads / 32; ++w) {
      if (w < warp) place += part[w][1];
      all += part[w][1];
    }
    if (keep) out[place + __popc(mk & ((1u << lane) - 1))] = i;
    at += all;
  }
}

}  // namespace

size_t paged_select_ws_bytes(const PagedView& v, int32_t T) {
  return ((size_t)v.rows * T * v.H * v.max_pages * 4 + 255) & ~(size_t)255;
}

int launch_paged_select(const PagedView& v, const akv_rows& q, int32_t T, int32_t sink, int32_t recent, const akv_selection& sel,
                        void* ws, void* stream) {
  const int64_t units = (int64_t)v.rows * T * v.H;
  if (units > 65535) return (int)cudaErrorInvalidConfiguration;
  const int blocks = (v.max_pages + kScoreWarps * 4 - 1) / (kScoreWarps * 4);
  akv_paged_score_kernel<<<dim3(blocks < 1024 ? blocks : 1024, (unsigned)units), 32 * kScoreWarps, 0, (cudaStream_t)stream>>>(
      v, (const uint16_t*)q.ptr, q.stride_b, q.stride_t, q.stride_h, T, (uint32_t*)ws);
  akv_paged_pick_kernel<<<(unsigned)units, kPickThreads, 0, (cudaStream_t)stream>>>(v, T, sink, recent, (const uint32_t*)ws, sel.pages,
                                                                                   sel.count, sel.top);
  return (int)cudaGetLastError();
}

}  // namespace akv
