// Query rows as operands of the paged cache's products on the fifth-generation tensor cores, once for all CTAs that multiply with them.
//
// A warp a row: its rotation, its power of two, its halves and its sums are some 300 instructions, which every CTA of a unit would
// repeat (256 rows of 8 heads for 152 CTAs: 18 us of 60).  A row's record lies as akv_paged_tc.cuh's operands have it, without their swizzle.
// Beside it, in a CTA of its own: for which groups the plan of shared pages is worth following.
#include "akv_paged.cuh"
#include "akv_paged_tc.cuh"

namespace akv {
namespace {

constexpr int kWarps = 8, kSide = 2;  // rows of a warp, side by side

struct QueryArgs {
  PagedView v;
  const uint16_t* q;
  const float* lse;
  uint8_t* records;
  int64_t qb, qt, qh, total;
  uint32_t sign;
  int T, aligned, sms;
  akv_share share;
  int32_t* shared;  // null: no share
};

// Whether reading a group's pages once pays.  Its time row by row goes by each member's units of 8 or 16 query rows (the second 1.5 times the first),
// shared by blocks of 128 rows of the whole group, at 3.5 times a unit of 8.  Microseconds row by row and shared of groups over 32 k tokens each, 8 KV
// heads: 12 pairs of 8 query rows 181 and 263, 8 of three 179 and 188, 6 of four 171 and 151, 3 of eight 169 and 97; of 16 query rows 12 pairs 262
// and 269 (rotated 308 and 280), 8 of three 261 and 198.
//   The launch of the shared part takes some 15 us until it has ended by itself where its caches are cold, as what it reads then is: all groups together have
// to save as much (4 query heads; a group of 32 rows over 4 k tokens 44 shared, 50 not; of 8 rows 38 and 32; 4 rows over 16 k tokens 44 and 38).
constexpr int kUnit8 = 2, kUnit16 = 3, kBlock = 7;  // of a tile of 128 tokens and a KV head, in half units of 8
constexpr int kWorth = 43;                          // what an SM saves at least, in those
__device__ __forceinline__ int64_t saved(const PagedView& v, int T, int tokens, int size) {
  const int rows = T * v.G;
  const int64_t alone = (int64_t)size * (rows <= 8 ? kUnit8 : (rows + 15) / 16 * kUnit16), together = ((int64_t)size * rows + 127) / 128 * kBlock;
  return max((int64_t)0, alone - together) * ((tokens + 127) / 128) * v.H;
}
__device__ __forceinline__ void choose(const QueryArgs& a) {
  __shared__ int64_t part[kWarps];
  const PagedView& v = a.v;
  const bool always = a.share.flags & AKV_SHARE_ALWAYS;
  auto pages = [&](int b) { return min(max(a.share.pages[b], 0), v.max_pages); };
  auto saves = [&](int b) { return saved(v, a.T, pages(b) << v.page_log, min(max(a.share.size[b], 0), v.rows)); };
  int64_t sum = 0;
  if (!always)
    for (int b = threadIdx.x; b < v.rows; b += 32 * kWarps)
      if (a.share.leader[b] == b) sum += saves(b);
#pragma unroll
  for (int m = 1; m < 32; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = sum;
  __syncthreads();
  sum = 0;
  for (int w = 0; w < kWarps; ++w) sum += part[w];
  const bool worth = sum >= (int64_t)kWorth * a.sms;
  for (int b = threadIdx.x; b < v.rows; b += 32 * kWarps) a.shared[b] = always || (worth && saves(b) > 0) ? pages(b) : 0;
}

template <int NG, bool HILO>
__global__ void __launch_bounds__(32 * kWarps) akv_paged_queries_kernel(const __grid_constant__ QueryArgs a) {
  launch_dependents();
  wait_for_stream();
  const PagedView& v = a.v;
  if (a.shared && blockIdx.x == gridDim.x - 1) {
    choose(a);
    return;
  }
  const int lane = threadIdx.x & 31, hq = v.H * v.G;
  const int64_t row0 = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * kSide;
  float x[kSide][4];
  bool counts[kSide];
#pragma unroll
  for (int r = 0; r < kSide; ++r) {
    const int64_t row = row0 + r;
    uint2 raw = make_uint2(0, 0);
    float lse = 0.f;
    if (row < a.total) {
      const int64_t bt = row / hq;
      const uint16_t* q = a.q + bt / a.T * a.qb + bt % a.T * a.qt + row % hq * a.qh + 4 * lane;
      raw = a.aligned ? *(const uint2*)q : make_uint2(q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16);
      if (a.lse) lse = a.lse[row];
    }
    bool fine = fabsf(lse) < __builtin_huge_valf();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[r][e] = row_to_float((uint16_t)((e < 2 ? raw.x : raw.y) >> (16 * (e & 1))), v.half);
      fine = fine && fabsf(x[r][e]) < __builtin_huge_valf();
    }
    // where lse is given, a row without a finite one, or with an infinity or a NaN of its own, is zeros and does not count
    counts[r] = !a.lse || __all_sync(0xffffffffu, fine);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[r][e] = counts[r] ? __uint_as_float(__float_as_uint(x[r][e]) ^ a.sign ^ (HILO ? sign_flip(v, 4 * lane + e) : 0u)) : 0.f;
  }
  if (HILO) {  // q' = H (s o q) / 16
    wht_rows(x, lane);
#pragma unroll
    for (int r = 0; r < kSide; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[r][e] *= 0.0625f;
  }
  float big[kSide], sum[kSide];
#pragma unroll
  for (int r = 0; r < kSide; ++r) {
    big[r] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = fabsf(x[r][e]);
      if (y <= 3.402823466e38f) big[r] = fmaxf(big[r], y);  // an infinite or NaN row spoils itself alone
    }
    sum[r] = (x[r][0] + x[r][1]) + (x[r][2] + x[r][3]);
  }
#pragma unroll
  for (int r = 0; r < kSide; ++r) big[r] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(big[r])));
#pragma unroll
  for (int m = 1; m < 32 / NG; m *= 2)
#pragma unroll
    for (int r = 0; r < kSide; ++r) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], m);
#pragma unroll
  for (int r = 0; r < kSide; ++r) {
    // times 2^(7 - e), e the largest value's exponent: below 2^7 (the sums below 2^14), exact in fp16 down to 2^-23 of that
    const int up = 7 - min(max((int)(__float_as_uint(big[r]) >> 23) - 126, -100), 128);
    const float unit = pow2(up);
    uint4 f[2];
    f[1] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int h = 0; h < (HILO ? 2 : 1); ++h) {
      uint32_t y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float z = x[r][e] * unit, own = h ? z - __half2float(__float2half_rn(z)) : z;
        const float other = __shfl_xor_sync(0xffffffffu, own, 1);
        y[e] = lane & 1 ? half2_bits(other, own) : half2_bits(own, other);
      }
      f[h] = make_uint4(y[0], y[1], y[2], y[3]);
    }
    if (row0 + r >= a.total) continue;
    // lanes 2 x, 2 x + 1 hold dimensions 8 x .. of word j = x / 4, t = x % 4: chunk 4 j + t of the row; the odd lane writes the low half
    uint8_t* to = a.records + (row0 + r) * kQueryRecord;
    *(uint4*)(to + (lane & 1) * 256 + 16 * (lane >> 1)) = f[lane & 1];
    // the 16 more dimensions (a group's sum in three parts p: p0 p1 p2 p0 p1 of each), and the row's numbers
    const float s0 = __shfl_sync(0xffffffffu, sum[r], 0) * unit, s1 = NG == 2 ? __shfl_sync(0xffffffffu, sum[r], 16) * unit : 0.f;
    if (lane == 0) {
      uint32_t p[2][3];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        float z = g ? s1 : s0;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const __half y = __float2half_rn(z);
          p[g][i] = __half_as_ushort(y);
          z -= __half2float(y);
        }
      }
      *(uint4*)(to + 512) = make_uint4(p[0][0] | p[0][1] << 16, p[0][2] | p[0][0] << 16, p[0][1] | p[1][0] << 16, p[1][1] | p[1][2] << 16);
      *(uint4*)(to + 528) = make_uint4(p[1][0] | p[1][1] << 16, 0, 0, 0);
      *(float2*)(to + 544) = make_float2(pow2(-up), counts[r] ? 1.f : 0.f);
    }
  }
}

}  // namespace

int launch_paged_queries(const PagedView& v, const akv_rows& q, int32_t T, bool negative, const float* lse, const akv_share* share, int32_t* shared,
                         void* records, void* stream) {
  QueryArgs a{};
  if (share) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&a.sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return (int)e;
    a.share = *share;
    a.shared = shared;
  }
  a.v = v;
  a.q = (const uint16_t*)q.ptr;
  a.qb = q.stride_b, a.qt = q.stride_t, a.qh = q.stride_h;
  a.lse = lse;
  a.records = (uint8_t*)records;
  a.total = (int64_t)v.rows * T * v.H * v.G;
  a.sign = negative ? 0x80000000u : 0u;
  a.T = T;
  a.aligned = (uintptr_t)q.ptr % 8 == 0 && q.stride_b % 4 == 0 && q.stride_t % 4 == 0 && q.stride_h % 4 == 0;
  const dim3 grid((unsigned)((a.total + kWarps * kSide - 1) / (kWarps * kSide)) + (share ? 1 : 0));
  auto* kernel = v.rotate ? (v.ng == 2 ? akv_paged_queries_kernel<2, true> : akv_paged_queries_kernel<1, true>)
                          : (v.ng == 2 ? akv_paged_queries_kernel<2, false> : akv_paged_queries_kernel<1, false>);
  return launch_after(kernel, grid, 32 * kWarps, 0, stream, a);
}

}  // namespace akv
