// Choice of the pages that a query attends: a score per page in whole numbers, then the best of them.
//
// The score reads the pages' bounds once (512 bytes a page and head) and does 2 G x 128 multiply-adds on them, in bytes:
// with a query row split into its positive and its negative part, the larger of q lo and q hi in each dimension is
// q+ hi + q- lo, two four-way byte products.  Whole numbers make the sums exact in any order, so that the choice is the
// same on every machine.  The choice itself finds the key of the last page kept bit by bit.
#include "akv_paged.cuh"

namespace akv {
namespace {

__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 .. 127
// Exponent e of a = f 2^e, f in [0.5, 1), clamped to +-100 (a finite, >= 0; subnormal and zero: -100).
__device__ __forceinline__ int exponent_of(float a) { return min(max((int)(__float_as_uint(a) >> 23) - 126, -100), 100); }

// Float order as unsigned order (no NaN; one zero).
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kScoreThreads = 128;
constexpr int kPageLanes = 8;                               // lanes of a page: dimensions 8 u .. and 64 + 8 u ..
constexpr int kAtOnce = kScoreThreads / kPageLanes;         // pages of a CTA at a time
constexpr int kRowsAtOnce = 8;                              // query rows whose sums are reduced together

template <bool HALF>
__device__ __forceinline__ float value(uint32_t w, int hi) {
  if (HALF) return __half2float(__ushort_as_half((unsigned short)(hi ? w >> 16 : w)));
  return __uint_as_float(hi ? w & 0xffff0000u : w << 16);
}

// Four values of two words times `unit` -> whole numbers in bytes (clamped to +-127 where `clamp`).
template <bool HALF>
__device__ __forceinline__ uint32_t whole4(uint32_t w0, uint32_t w1, float unit, bool clamp) {
  float t[4] = {value<HALF>(w0, 0) * unit, value<HALF>(w0, 1) * unit, value<HALF>(w1, 0) * unit, value<HALF>(w1, 1) * unit};
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (clamp) t[i] = fminf(fmaxf(t[i], -127.f), 127.f);
    b[i] = __float_as_uint(t[i] + 12582912.f);  // 1.5 2^23: the rounded number in the low bits
  }
  return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}

template <bool HALF>
__global__ void __launch_bounds__(kScoreThreads) akv_paged_score_kernel(PagedView v, const uint16_t* q, int64_t qb, int64_t qt,
                                                                        int64_t qh, int T, int chunks, int per_cta, uint32_t* keys) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ __align__(16) uint32_t q_words[];  // [rows to a multiple of 8][8 lanes][4 positive, 4 negative]
  __shared__ float q_max[kScoreThreads / 32];
  const int unit = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const int h = unit % v.H, t = unit / v.H % T, b = unit / v.H / T;
  const int P = 1 << v.page_log, tid = threadIdx.x, lane = tid & 31, u = tid & 7;
  const int sees = max(0, held_tokens(v, b) - T + 1 + t), n = (sees + P - 1) >> v.page_log;
  const int j0 = chunk * per_cta, j1 = min(n, j0 + per_cta);
  if (j0 >= j1) return;
  const uint32_t bounds_at = (uint32_t)(P >> 4) * sub_bytes(v.ng);
  struct Bounds {
    uint4 lo0, lo1, hi0, hi1;
    bool there;
  };
  auto load = [&](int j) {
    Bounds x;
    x.lo0 = x.lo1 = x.hi0 = x.hi1 = make_uint4(0, 0, 0, 0);
    const int page = j < j1 ? page_of(v, b, j) : -1;
    x.there = page >= 0;
    if (x.there) {
      const uint4* at = (const uint4*)(block_of(v, page, h) + bounds_at) + u;
      x.lo0 = at[0], x.lo1 = at[8], x.hi0 = at[16], x.hi1 = at[24];
    }
    return x;
  };
  Bounds next = load(j0 + tid / kPageLanes);

  // the query rows as bytes
  const uint16_t* rows = q + b * qb + t * qt + (int64_t)h * v.G * qh;
  float top = 0.f;
  for (int i = tid; i < v.G * kD; i += kScoreThreads) top = max_nan(top, fabsf(row_to_float(rows[(int64_t)(i >> 7) * qh + (i & 127)], HALF)));
  for (int k = 16; k; k >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, k));
  if (lane == 0) q_max[tid >> 5] = top;
  __syncthreads();
  top = max_nan(max_nan(q_max[0], q_max[1]), max_nan(q_max[2], q_max[3]));
  const bool fine = top <= 3.402823466e38f;
  const float unit_q = power(7 - exponent_of(fine ? top : 0.f));
  const int padded = (v.G + kRowsAtOnce - 1) / kRowsAtOnce * kRowsAtOnce;
  for (int i = tid; i < padded * 32; i += kScoreThreads) {  // word: dimensions 4 k .. of a row
    const int g = i >> 5, k = i & 31;
    uint32_t pos = 0, neg = 0;
    if (g < v.G && fine) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int x = min(max(__float2int_rn(row_to_float(rows[g * qh + 4 * k + e], HALF) * unit_q), -127), 127);
        pos |= (uint32_t)(max(x, 0) & 255) << 8 * e;
        neg |= (uint32_t)(min(x, 0) & 255) << 8 * e;
      }
    }
    uint32_t* to = q_words + (g * 8 + (k & 15) / 2) * 8 + 2 * (k >> 4) + (k & 1);
    to[0] = pos;
    to[4] = neg;
  }
  __syncthreads();

  for (int j = j0 + tid / kPageLanes; j - tid / kPageLanes < j1; j += kAtOnce) {
    const Bounds x = next;
    next = load(j + kAtOnce);
    const uint32_t w[16] = {x.lo0.x, x.lo0.y, x.lo0.z, x.lo0.w, x.lo1.x, x.lo1.y, x.lo1.z, x.lo1.w,
                            x.hi0.x, x.hi0.y, x.hi0.z, x.hi0.w, x.hi1.x, x.hi1.y, x.hi1.z, x.hi1.w};
    uint32_t big = 0;  // largest magnitudes of the even and of the odd values, as their bits
#pragma unroll
    for (int i = 0; i < 16; ++i) big = __vmaxu2(big, w[i] & 0x7fff7fffu);
#pragma unroll
    for (int k = 1; k < kPageLanes; k *= 2) big = __vmaxu2(big, __shfl_xor_sync(0xffffffffu, big, k));
    big = max(big & 0xffffu, big >> 16);
    const bool number = big < (HALF ? 0x7c00u : 0x7f80u);
    const float most = value<HALF>(number ? big : 0u, 0);
    const int ep = exponent_of(most);
    const float unit_p = power(7 - ep);
    const bool clamp = __any_sync(0xffffffffu, most * unit_p >= 127.5f);
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      lo[k] = whole4<HALF>(w[2 * k], w[2 * k + 1], unit_p, clamp);
      hi[k] = whole4<HALF>(w[8 + 2 * k], w[8 + 2 * k + 1], unit_p, clamp);
    }
    int best = INT32_MIN;
    for (int g0 = 0; g0 < v.G; g0 += kRowsAtOnce) {
      int sum[kRowsAtOnce];
#pragma unroll
      for (int g = 0; g < kRowsAtOnce; ++g) {
        sum[g] = 0;
        if (g0 + g < v.G) {
          const uint4 qp = *(const uint4*)(q_words + ((g0 + g) * 8 + u) * 8), qn = *(const uint4*)(q_words + ((g0 + g) * 8 + u) * 8 + 4);
          sum[g] = __dp4a((int)hi[0], (int)qp.x, sum[g]);
          sum[g] = __dp4a((int)hi[1], (int)qp.y, sum[g]);
          sum[g] = __dp4a((int)hi[2], (int)qp.z, sum[g]);
          sum[g] = __dp4a((int)hi[3], (int)qp.w, sum[g]);
          sum[g] = __dp4a((int)lo[0], (int)qn.x, sum[g]);
          sum[g] = __dp4a((int)lo[1], (int)qn.y, sum[g]);
          sum[g] = __dp4a((int)lo[2], (int)qn.z, sum[g]);
          sum[g] = __dp4a((int)lo[3], (int)qn.w, sum[g]);
        }
      }
      // over the page's lanes: at each step a lane keeps half of its rows, in the end one, lane u row bits of u reversed
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int give = u & 1 ? sum[k] : sum[k + 4], keep = u & 1 ? sum[k + 4] : sum[k];
        sum[k] = keep + __shfl_xor_sync(0xffffffffu, give, 1);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int give = u & 2 ? sum[k] : sum[k + 2], keep = u & 2 ? sum[k + 2] : sum[k];
        sum[k] = keep + __shfl_xor_sync(0xffffffffu, give, 2);
      }
      const int give = u & 4 ? sum[0] : sum[1], keep = u & 4 ? sum[1] : sum[0];
      const int s = keep + __shfl_xor_sync(0xffffffffu, give, 4);
      const int row = g0 + 4 * (u & 1) + (u & 2) + (u >> 2);
      if (row < v.G) best = max(best, s);
    }
#pragma unroll
    for (int k = 1; k < kPageLanes; k *= 2) best = max(best, __shfl_xor_sync(0xffffffffu, best, k));
    if (u == 0 && j < j1) {
      const float inf = __int_as_float(0x7f800000);
      keys[(int64_t)unit * v.max_pages + j] = order_key(!x.there ? -inf : number ? (float)best * power(ep) : inf);
    }
  }
}

constexpr int kPickThreads = 512, kPickWarps = kPickThreads / 32;
constexpr uint32_t kForced = 0xffffffffu;  // above every score

// Sum over the CTA of x; `part` alternates between two buffers, so one barrier does.
__device__ __forceinline__ int block_sum(int x, int* part) {
  x = __reduce_add_sync(0xffffffffu, x);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int w = 0; w < kPickWarps; ++w) s += part[w];
  return s;
}
// Sum over the threads before.
__device__ __forceinline__ int block_before(int x, int* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = x;
#pragma unroll
  for (int h = 1; h < 32; h *= 2) {
    const int o = __shfl_up_sync(0xffffffffu, inc, h);
    if (lane >= h) inc += o;
  }
  if (lane == 31) part[warp] = inc;
  __syncthreads();
  int s = inc - x;
#pragma unroll
  for (int w = 0; w < kPickWarps; ++w) s += w < warp ? part[w] : 0;
  return s;
}

// One CTA: one (request, query token, head).  A thread holds `each` neighbouring pages, in registers where they are KEPT
// at most.
template <int KEPT>
__global__ void __launch_bounds__(kPickThreads) akv_paged_pick_kernel(PagedView v, int T, int sink, int recent, const uint32_t* keys,
                                                                      int32_t* sel, int32_t* count, int top) {
  __shared__ int part[2][kPickWarps];
  __shared__ uint32_t ends[2][kPickWarps];
  const int64_t unit = blockIdx.x;
  const int t = (int)(unit / v.H % T), b = (int)(unit / v.H / T);
  const int P = 1 << v.page_log, tid = threadIdx.x;
  const int sees = max(0, held_tokens(v, b) - T + 1 + t), n = (sees + P - 1) >> v.page_log;
  int32_t* out = sel + unit * top;
  const int kept = min(n, top);
  if (tid == 0) count[unit] = kept;
  for (int i = kept + tid; i < top; i += kPickThreads) out[i] = -1;
  if (n <= top) {
    for (int i = tid; i < n; i += kPickThreads) out[i] = i;
  }
  // waited for in any case: what follows in the stream may write where the scores are still being written
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (n <= top) return;
  const uint32_t* key = keys + unit * v.max_pages;
  const int each = (n + kPickThreads - 1) / kPickThreads, i0 = tid * each, i1 = min(n, i0 + each);
  uint32_t mine[KEPT > 0 ? KEPT : 1];
  auto at = [&](int i) { return i < sink || i >= n - recent ? kForced : key[i]; };
  if (KEPT > 0) {
#pragma unroll
    for (int k = 0; k < (KEPT > 0 ? KEPT : 1); ++k) mine[k] = i0 + k < i1 ? at(i0 + k) : 0u;  // (0: below every score)
  }
  auto each_key = [&](auto f) {
    if (KEPT > 0) {
#pragma unroll
      for (int k = 0; k < (KEPT > 0 ? KEPT : 1); ++k)
        if (i0 + k < i1) f(i0 + k, mine[k]);
    } else {
      for (int i = i0; i < i1; ++i) f(i, at(i));
    }
  };
  // the range of the keys that are not forced
  uint32_t low = kForced, high = 0;
  each_key([&](int, uint32_t k) {
    if (k != kForced) low = min(low, k), high = max(high, k);
  });
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  if ((tid & 31) == 0) ends[0][tid >> 5] = low, ends[1][tid >> 5] = high;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPickWarps; ++w) low = min(low, ends[0][w]), high = max(high, ends[1][w]);
  // the largest key `last` of which at least `top` pages have it or more; its bits above the first that differs are known
  // (n > top >= sink + recent, so there is a page that is not forced)
  uint32_t last = low;
  int turn = 0;
  bool exact = false;  // exactly `top` pages have `last` or more
  if (low != high) {
    const int bit0 = 31 - __clz(low ^ high);
    last = low >> bit0 >> 1 << bit0 << 1;
    for (int bit = bit0; bit >= 0 && !exact; --bit) {
      const uint32_t probe = last | 1u << bit;
      int c = 0;
      each_key([&](int, uint32_t k) { c += k >= probe; });
      c = block_sum(c, part[turn ^= 1]);
      if (c >= top) last = probe;
      exact = c == top;
    }
  }
  int above = 0, ties = 0;
  each_key([&](int, uint32_t k) {
    above += exact ? k >= last : k > last;
    ties += !exact && k == last;
  });
  const int room = top - block_sum(above, part[turn ^= 1]);  // for pages with the key `last`, the lowest first
  int tie = block_before(ties, part[turn ^= 1]);
  const int my_ties = min(max(room - tie, 0), ties);
  int place = block_before(above + my_ties, part[turn ^= 1]);
  each_key([&](int i, uint32_t k) {
    bool keep = exact ? k >= last : k > last;
    if (!exact && k == last) keep = tie++ < room;
    if (keep) out[place++] = i;
  });
}

}  // namespace

size_t paged_select_ws_bytes(const PagedView& v, int32_t T) {
  return ((size_t)v.rows * T * v.H * v.max_pages * 4 + 255) & ~(size_t)255;
}

int launch_paged_select(const PagedView& v, const akv_rows& q, int32_t T, int32_t sink, int32_t recent, const akv_selection& sel,
                        void* ws, void* stream) {
  const int64_t units = (int64_t)v.rows * T * v.H;
  cudaStream_t s = (cudaStream_t)stream;
  // A CTA prepares the query rows (its price) for as many pages as leave 8 CTAs for each SM, at least 16 and at most 256.
  int64_t per_cta = (units * v.max_pages + 8 * 152 - 1) / (8 * 152);
  per_cta = (per_cta + kAtOnce - 1) / kAtOnce * kAtOnce;
  if (per_cta > 256) per_cta = 256;
  const int64_t chunks = ((int64_t)v.max_pages + per_cta - 1) / per_cta;
  if (units * chunks > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  const size_t smem = (size_t)((v.G + kRowsAtOnce - 1) / kRowsAtOnce) * kRowsAtOnce * 64 * 4;
  auto score = v.half ? akv_paged_score_kernel<true> : akv_paged_score_kernel<false>;
  score<<<(unsigned)(units * chunks), kScoreThreads, smem, s>>>(v, (const uint16_t*)q.ptr, q.stride_b, q.stride_t, q.stride_h, T,
                                                                (int)chunks, (int)per_cta, (uint32_t*)ws);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return (int)e;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute pdl{};
  pdl.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)units);
  cfg.blockDim = dim3(kPickThreads);
  cfg.stream = s;
  cfg.attrs = &pdl;
  cfg.numAttrs = 1;
  auto pick = v.max_pages <= 4 * kPickThreads    ? akv_paged_pick_kernel<4>
              : v.max_pages <= 16 * kPickThreads ? akv_paged_pick_kernel<16>
                                                 : akv_paged_pick_kernel<0>;
  return (int)cudaLaunchKernelEx(&cfg, pick, v, T, sink, recent, (const uint32_t*)ws, sel.pages, sel.count, sel.top);
}

}  // namespace akv
