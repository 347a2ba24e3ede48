// Choice of the pages that a query attends: a score per page in whole numbers, then the best of them.
//
// The score reads the pages' bounds once (512 bytes a page and head) and does 2 G x 128 multiply-adds on them: with a
// query row split into its positive and its negative part, the larger of q lo and q hi in each dimension is
// q+ hi + q- lo, two products.  The numbers are at most 127, exact in bf16 and fp16, and the sums at most 2^22, exact in
// fp32: the tensor cores add them up without rounding, in any order, so that the choice is the same on every machine.
// What costs is turning the bounds into whole numbers (three operations a pair); a warp does it once for all query rows.
// 8 x 2048 pages of 8 heads: 20 to 22 us, 3.1 to 3.3 TB/s.  The page format bounds it: a plain read of 512-byte pieces 9.7 KB
// apart, as bounds inside the pages' blocks are, reaches 3.35 TB/s in any order and at any number of CTAs.
// The choice finds the key of the last page kept, 8 bits of its range a pass: 6 us for 512 pages and 8 us for 2048,
// latency alone.
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

constexpr int kScoreThreads = 128, kScoreWarps = kScoreThreads / 32;
constexpr int kWarpPages = 16;                          // pages of a warp at a time: the rows of its products
constexpr int kAtOnce = kWarpPages * kScoreWarps;
constexpr int kSteps = 16;                              // products over 16 dimensions: 8 of the largest, 8 of the smallest

template <bool HALF>
__device__ __forceinline__ float value(uint32_t w, int hi) {
  if (HALF) return __half2float(__ushort_as_half((unsigned short)(hi ? w >> 16 : w)));
  return __uint_as_float(hi ? w & 0xffff0000u : w << 16);
}
// The pair of larger magnitudes (a NaN is passed on; the signs mean nothing).
template <bool HALF>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  uint32_t r;
  if (HALF) asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Two values times a power of two (the product of both factors), at most 128 in magnitude, as whole numbers of the same
// type: at 128 and above (fp16: 1024) its numbers are 1 apart, so adding 128 away from zero rounds to nearest even.
template <bool HALF>
__device__ __forceinline__ uint32_t whole2(uint32_t w, uint32_t unit, uint32_t unit_first) {
  uint32_t far = w & 0x80008000u, r;
  if (HALF) {
    far |= 0x64006400u;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(unit_first));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(r), "r"(unit), "r"(far));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(far));
  } else {
    far |= 0x43004300u;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w), "r"(unit), "r"(far));
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(far));
  }
  return r;
}
template <bool HALF>
__device__ __forceinline__ uint32_t clamp2(uint32_t w) {  // to +-127
  uint32_t r;
  if (HALF) asm("min.f16x2 %0, %1, %2;\n max.f16x2 %0, %0, %3;" : "=&r"(r) : "r"(w), "r"(0x57f057f0u), "r"(0xd7f0d7f0u));
  else asm("min.bf16x2 %0, %1, %2;\n max.bf16x2 %0, %0, %3;" : "=&r"(r) : "r"(w), "r"(0x42fe42feu), "r"(0xc2fec2feu));
  return r;
}

template <bool HALF>
__global__ void __launch_bounds__(kScoreThreads, 3) akv_paged_score_kernel(PagedView v, const uint16_t* q, int64_t qb, int64_t qt,
                                                                           int64_t qh, int T, int chunks, int per_cta, uint32_t* keys) {
  launch_dependents();
  wait_for_stream();
  extern __shared__ __align__(16) uint2 q_frag[];  // [blocks of 8 rows][kSteps][32 lanes]
  __shared__ float q_max[kScoreWarps];
  const int unit = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
  const int h = unit % v.H, t = unit / v.H % T, b = unit / v.H / T;
  const int P = 1 << v.page_log, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g8 = lane >> 2, t4 = lane & 3;
  const int sees = max(0, held_tokens(v, b) - T + 1 + t), n = (sees + P - 1) >> v.page_log;
  const int j0 = chunk * per_cta, j1 = min(n, j0 + per_cta);
  if (j0 >= j1) return;
  const uint32_t bounds_at = (uint32_t)(P >> 4) * sub_bytes(v.ng);
  // this lane's pages: g8 and g8 + 8 of the warp's sixteen
  auto find = [&](int j) { return j < j1 ? v.table[(int64_t)b * v.table_stride + j] : -1; };
  int j = j0 + kWarpPages * warp + g8;
  int page[2] = {find(j), find(j + 8)};
  uint32_t w[2][2][16];  // the lane's two pages; their largest, their smallest keys; four chunks of four words
  bool there[2];
  auto load = [&]() {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      there[x] = (uint32_t)page[x] < (uint32_t)v.n_pages;
      const uint4* at = (const uint4*)(block_of(v, there[x] ? page[x] : 0, h) + bounds_at) + t4;
#pragma unroll
      for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint4 y = there[x] ? at[16 * (1 - side) + 4 * c] : make_uint4(0, 0, 0, 0);
          w[x][side][4 * c] = y.x, w[x][side][4 * c + 1] = y.y, w[x][side][4 * c + 2] = y.z, w[x][side][4 * c + 3] = y.w;
        }
    }
  };
  load();  // (under way while the queries are prepared)
  page[0] = find(j + kAtOnce), page[1] = find(j + kAtOnce + 8);

  // the query rows as whole numbers
  const uint16_t* rows = q + b * qb + t * qt + (int64_t)h * v.G * qh;
  float top = 0.f;
  for (int i = tid; i < v.G * kD; i += kScoreThreads) top = max_nan(top, fabsf(row_to_float(rows[(int64_t)(i >> 7) * qh + (i & 127)], HALF)));
  for (int k = 16; k; k >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, k));
  if (lane == 0) q_max[warp] = top;
  __syncthreads();
  top = max_nan(max_nan(q_max[0], q_max[1]), max_nan(q_max[2], q_max[3]));
  const bool fine = top <= 3.402823466e38f;
  const float unit_q = power(7 - exponent_of(fine ? top : 0.f));
  const int blocks = (v.G + 7) / 8;
  for (int i = tid; i < blocks * 8 * 32; i += kScoreThreads) {
    // steps s (the largest) and s + 8 (the smallest): chunk t4 + 4 (s / 2) of 8 dimensions, its half s % 2
    const int l = i & 31, s = i >> 5 & 7, row = i / 256 * 8 + (l >> 2);
    uint32_t pos[2] = {0, 0}, neg[2] = {0, 0};
    if (row < v.G && fine) {
      const uint16_t* x = rows + row * qh + 8 * ((l & 3) + 4 * (s >> 1)) + 4 * (s & 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = fminf(fmaxf(rintf(row_to_float(x[e], HALF) * unit_q), -127.f), 127.f);
        pos[e >> 1] |= (uint32_t)float_to_row(fmaxf(y, 0.f), HALF) << 16 * (e & 1);
        neg[e >> 1] |= (uint32_t)float_to_row(fminf(y, 0.f), HALF) << 16 * (e & 1);
      }
    }
    uint2* to = q_frag + (i / 256 * kSteps + s) * 32 + l;
    to[0] = make_uint2(pos[0], pos[1]);
    to[8 * 32] = make_uint2(neg[0], neg[1]);
  }
  __syncthreads();

  for (; j - g8 < j1; j += kAtOnce) {
    bool number[2];
    float most[2];
    int ep[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t big = larger<HALF>(w[x][0][0], w[x][1][0]);
#pragma unroll
      for (int i = 1; i < 16; ++i) big = larger<HALF>(big, larger<HALF>(w[x][0][i], w[x][1][i]));
      big = larger<HALF>(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = larger<HALF>(big, __shfl_xor_sync(0xffffffffu, big, 2));
      big = max(big & 0x7fffu, big >> 16 & 0x7fffu);
      number[x] = big < (HALF ? 0x7c00u : 0x7f80u);
      most[x] = value<HALF>(number[x] ? big : 0u, 0);
      ep[x] = exponent_of(most[x]);
    }
    bool clamp = false;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      // 2^(7 - e) as a pair; in fp16, whose numbers go from 2^-24 to 2^15, in two factors
      const int up = 7 - ep[x], first = HALF ? max(up - 15, 0) : 0;
      const uint32_t unit = HALF ? (uint32_t)(up - first + 15) << 10 : (uint32_t)(up + 127) << 7;
      const uint32_t unit_first = (uint32_t)(first + 15) << 10;
      clamp = clamp || most[x] * power(up) >= 127.5f;
#pragma unroll
      for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int i = 0; i < 16; ++i) w[x][side][i] = whole2<HALF>(w[x][side][i], unit * 0x10001u, unit_first * 0x10001u);
    }
    if (__any_sync(0xffffffffu, clamp)) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
          for (int i = 0; i < 16; ++i) w[x][side][i] = clamp2<HALF>(w[x][side][i]);
    }
    float best[2] = {__int_as_float(0xff800000), __int_as_float(0xff800000)};
    for (int r = 0; r < blocks; ++r) {
      float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};  // two chains of products
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const uint2 y = q_frag[(r * kSteps + s) * 32 + lane];
        const int side = s >> 3, i = 2 * (s & 7);
        if (HALF)
          asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                       : "+f"(d[side][0]), "+f"(d[side][1]), "+f"(d[side][2]), "+f"(d[side][3])
                       : "r"(w[0][side][i]), "r"(w[1][side][i]), "r"(w[0][side][i + 1]), "r"(w[1][side][i + 1]), "r"(y.x), "r"(y.y));
        else
          asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                       : "+f"(d[side][0]), "+f"(d[side][1]), "+f"(d[side][2]), "+f"(d[side][3])
                       : "r"(w[0][side][i]), "r"(w[1][side][i]), "r"(w[0][side][i + 1]), "r"(w[1][side][i + 1]), "r"(y.x), "r"(y.y));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (8 * r + 2 * t4 + (e & 1) < v.G) best[e >> 1] = fmaxf(best[e >> 1], d[0][e] + d[1][e]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      best[x] = fmaxf(best[x], __shfl_xor_sync(0xffffffffu, best[x], 1));
      best[x] = fmaxf(best[x], __shfl_xor_sync(0xffffffffu, best[x], 2));
      const float inf = __int_as_float(0x7f800000);
      if (t4 == 0 && j + 8 * x < j1)
        keys[(int64_t)unit * v.max_pages + j + 8 * x] = order_key(!there[x] ? -inf : number[x] ? best[x] * power(ep[x]) : inf);
    }
    load();
    page[0] = find(j + 2 * kAtOnce), page[1] = find(j + 2 * kAtOnce + 8);
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
  __shared__ int hist[256], found[3];
  launch_dependents();
  wait_for_stream();
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
    return;
  }
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
  // the range of the keys that are not forced (n > top >= sink + recent, so there is one)
  uint32_t low = kForced, high = 0;
  each_key([&](int, uint32_t k) {
    if (k != kForced) low = min(low, k), high = max(high, k);
  });
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  if ((tid & 31) == 0) ends[0][tid >> 5] = low, ends[1][tid >> 5] = high;
  if (tid < 256) hist[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPickWarps; ++w) low = min(low, ends[0][w]), high = max(high, ends[1][w]);
  // The range is narrowed to a 256th a pass: the part that holds the last page kept.  In the end either all pages with
  // `last` or more are kept (exact), or `last` is the one key of its part and the lowest pages that have it are.
  int want = top - sink - recent;
  uint32_t last = kForced;
  bool exact = want == 0;
  while (!exact) {
    const int bits = 32 - __clz(high - low), shift = max(0, bits - 8);
    each_key([&](int, uint32_t k) {
      if (k >= low && k <= high) atomicAdd(hist + (k - low >> shift), 1);
    });
    __syncthreads();
    const int mine_h = tid < 256 ? hist[255 - tid] : 0;  // from the highest part down
    const int before = block_before(mine_h, part[0]);
    if (tid < 256) {
      hist[255 - tid] = 0;
      if (before < want && before + mine_h >= want) found[0] = 255 - tid, found[1] = before, found[2] = mine_h;
    }
    __syncthreads();
    low += (uint32_t)found[0] << shift;
    high = min(high, low + ((1u << shift) - 1));
    want -= found[1];
    last = low;
    exact = found[2] == want;
    if (shift == 0) break;
  }
  int turn = 0;
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
  // A CTA prepares the query rows (its price) for as many pages as leave three CTAs for each SM, 64 to 1024.
  int64_t per_cta = (units * v.max_pages + 3 * 152 - 1) / (3 * 152);
  per_cta = (per_cta + kAtOnce - 1) / kAtOnce * kAtOnce;
  if (per_cta > 1024) per_cta = 1024;
  const int64_t chunks = ((int64_t)v.max_pages + per_cta - 1) / per_cta;
  if (units * chunks > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  const size_t smem = (size_t)((v.G + 7) / 8) * kSteps * 32 * sizeof(uint2);
  auto score = v.half ? akv_paged_score_kernel<true> : akv_paged_score_kernel<false>;
  const int err = launch_after(score, dim3((unsigned)(units * chunks)), kScoreThreads, smem, stream, v, (const uint16_t*)q.ptr, q.stride_b,
                               q.stride_t, q.stride_h, T, (int)chunks, (int)per_cta, (uint32_t*)ws);
  if (err) return err;
  auto pick = v.max_pages <= 4 * kPickThreads    ? akv_paged_pick_kernel<4>
              : v.max_pages <= 8 * kPickThreads ? akv_paged_pick_kernel<8>
              : v.max_pages <= 16 * kPickThreads ? akv_paged_pick_kernel<16>
                                                 : akv_paged_pick_kernel<0>;
  return launch_after(pick, dim3((unsigned)units), kPickThreads, 0, stream, v, T, sink, recent, (const uint32_t*)ws, sel.pages, sel.count,
                      sel.top);
}

}  // namespace akv
