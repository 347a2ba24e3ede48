// Attention weights that the tokens of a paged cache got, added to their scores.
//
// The softmax's normaliser is known (lse), so a token's weight needs its own key alone: one pass over the key codes and their
// parameters, no reference, no join, and every score is written by one lane.  Units (request, KV head) are cut into tiles of
// 128 tokens, the tiles of all units into equal contiguous ranges, one per CTA; in a CTA a warp takes sub-blocks of 16
// tokens, straight from memory to the tensor cores' operands (nibbles as fp16 subnormals, as in the attention).
#include <cuda_runtime.h>

#include "akv_paged.cuh"

namespace akv {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kTileTokens = 128, kTileSubs = 8;
constexpr int kBlocks = 8;  // blocks of 8 query rows in shared memory at a time
constexpr float kInf = __builtin_huge_valf();

struct WeightArgs {
  PagedView v;
  const uint16_t* q;
  const float* lse;
  const float* was;
  float* now;
  int64_t qb, qt, qh, wb, wh, nb, nh;
  float scale, decay;  // scale: sm_scale log2(e)
  int T, rows;         // rows: query rows of a unit, T G
};

struct Smem {
  uint4 frag[2][kBlocks][4][32];     // query operand: high, low halves
  float qsum[8 * kBlocks][2];        // sums of a query row over each group of dimensions, times scale
  float qscale[8 * kBlocks];         // what its products count; 0 for rows that add nothing
  float lse2[8 * kBlocks];           // lse in log2 units; +infinity for rows that add nothing
  int64_t part[kWarps];
  int64_t place[2];
};

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float word_scale(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)w)); }
__device__ __forceinline__ float word_min(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
__device__ __forceinline__ uint32_t comp(const uint4& x, int j) { return j == 0 ? x.x : j == 1 ? x.y : j == 2 ? x.z : x.w; }
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }  // -126 .. 127
__device__ __forceinline__ bool finite_word(uint32_t w) { return (w & 0x7c00u) != 0x7c00u && (w & 0x7c000000u) != 0x7c000000u; }

// Query rows row0 .. of unit (b, h) as operands, a warp per row; up to `blocks` blocks of 8.
template <int NG, bool HILO>
__device__ __forceinline__ void load_queries(const WeightArgs& a, Smem& S, int b, int h, int row0, int blocks) {
  const PagedView& v = a.v;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int rr = warp; rr < 8 * blocks; rr += kWarps) {
    float x[4] = {0.f, 0.f, 0.f, 0.f}, lse = kInf;
    const int row = row0 + rr;
    if (row < a.rows) {
      const int t = row / v.G, g = row % v.G;
      const uint16_t* at = a.q + b * a.qb + t * a.qt + (int64_t)(h * v.G + g) * a.qh + 4 * lane;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = row_to_float(at[e], v.half);
      lse = a.lse[((int64_t)b * a.T + t) * (v.H * v.G) + h * v.G + g];
    }
    if (HILO) {  // q' = H (s o q) / 16
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(__float_as_uint(x[e]) ^ sign_flip(v, 4 * lane + e));
      wht_32x4(x, lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= 0.0625f;
    }
    // a row with no finite lse, or with an infinity or a NaN of its own, adds nothing
    const bool fine = fabsf(lse) < kInf && fabsf(x[0]) < kInf && fabsf(x[1]) < kInf && fabsf(x[2]) < kInf && fabsf(x[3]) < kInf;
    const bool counts = __all_sync(0xffffffffu, fine);
    float big = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!counts) x[e] = 0.f;
      big = fmaxf(big, fabsf(x[e]));
    }
    big = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(big)));
    const int e2 = min(max((int)(__float_as_uint(big) >> 23) - 126, -100), 128);
    const float up = pow2(14 - e2);  // below 2^14, exact in fp16 down to 2^-23 of that
    float sum = (x[0] + x[1]) + (x[2] + x[3]);
#pragma unroll
    for (int s = 1; s < 32 / NG; s *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if (lane % (32 / NG) == 0) S.qsum[rr][lane / (32 / NG)] = sum * a.scale;
    if (lane == 0) {
      S.qscale[rr] = a.scale * pow2(e2 - 10) * 1048576.f;  // codes count 2^-24, queries 2^(14 - e2)
      S.lse2[rr] = counts ? lse * 1.4426950408889634f : kInf;
    }
    uint4 f[HILO ? 2 : 1];
#pragma unroll
    for (int lo = 0; lo < (HILO ? 2 : 1); ++lo) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // nibble e: odd ones stand for 16 times their value
        const float y = x[e] * (e & 1 ? up * 0.0625f : up);
        const float hi = __half2float(__float2half_rn(y));
        const float mine = lo ? y - hi : y;
        const float other = __shfl_xor_sync(0xffffffffu, mine, 1);
        w[e] = lane & 1 ? half2_bits(other, mine) : half2_bits(mine, other);
      }
      f[lo] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    // lanes 2 x and 2 x + 1 hold dimensions 8 x ..: word j = x / 4, operand lane 4 row + x % 4
    const int to = 4 * (rr & 7) + (lane >> 1 & 3);
    if (!(lane & 1)) S.frag[0][rr >> 3][lane >> 3][to] = f[0];
    if (HILO && (lane & 1)) S.frag[1][rr >> 3][lane >> 3][to] = f[HILO ? 1 : 0];
  }
}

template <int NG>
struct Sub {  // key codes and parameters of a sub-block, a lane's part: tokens g8, g8 + 8
  uint4 c[2];
  uint32_t w[2][NG];
  bool there;
};

template <int NG, bool HILO>
__global__ void __launch_bounds__(kThreads, 2) akv_paged_weights_kernel(const __grid_constant__ WeightArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Smem& S = *reinterpret_cast<Smem*>(smem_raw);
  constexpr uint32_t kSub = 2048 + 128 * NG;
  const PagedView& v = a.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
  launch_dependents();
  wait_for_stream();

  // ---- the CTA's range of tiles: row by row, its heads in turn
  auto tiles_of = [&](int b) { return (held_tokens(v, b) + kTileTokens - 1) / kTileTokens; };
  const int strip = (v.rows + kThreads - 1) / kThreads, b0 = min(v.rows, tid * strip), b1 = min(v.rows, b0 + strip);
  int64_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += (int64_t)tiles_of(b) * v.H;
  int64_t inc = mine, before, total = 0;
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    const int64_t o = __shfl_up_sync(0xffffffffu, inc, s);
    if (lane >= s) inc += o;
  }
  if (lane == 31) S.part[warp] = inc;
  __syncthreads();
  before = inc - mine;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += S.part[w];
    total += S.part[w];
  }
  const int64_t lo = blockIdx.x * total / gridDim.x, hi = (blockIdx.x + 1) * total / gridDim.x;
  if (lo >= hi) return;
  if (lo >= before && lo < before + mine) {
    int64_t rest = lo - before;
    int b = b0;
    for (;; ++b) {
      const int64_t here = (int64_t)tiles_of(b) * v.H;
      if (rest < here) break;
      rest -= here;
    }
    S.place[0] = b, S.place[1] = rest;
  }
  __syncthreads();
  int b = (int)S.place[0];
  int64_t at = S.place[1];  // tile of the row's H x tiles

  for (int64_t k = lo; k < hi;) {
    const int held = held_tokens(v, b), tiles = tiles_of(b), h = (int)(at / tiles), t0 = (int)(at % tiles);
    const int n = (int)min((int64_t)(tiles - t0), hi - k);  // tiles of this unit
    const int sees0 = held - a.T + 1;                        // tokens that the first query token sees
    const int sub1 = min((t0 + n) * kTileSubs, (held + 15) >> 4);
    for (int row0 = 0; row0 < a.rows; row0 += 8 * kBlocks) {
      const int blocks = min(kBlocks, (a.rows - row0 + 7) >> 3);
      __syncthreads();
      load_queries<NG, HILO>(a, S, b, h, row0, blocks);
      __syncthreads();
      auto load = [&](int s) {
        Sub<NG> x{};
        const int page = s < sub1 ? page_of(v, b, 16 * s >> v.page_log) : -1;
        x.there = page >= 0;
        if (x.there) {
          const uint8_t* base = block_of(v, page, h) + (uint64_t)((16 * s & ((1 << v.page_log) - 1)) >> 4) * kSub;
          x.c[0] = *(const uint4*)(base + 16 * lane);
          x.c[1] = *(const uint4*)(base + 512 + 16 * lane);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint8_t* p = base + 2048 + 8 * NG * (g8 + 8 * y);
            if (NG == 2) {
              const uint2 w = *(const uint2*)p;
              x.w[y][0] = w.x, x.w[y][NG - 1] = w.y;
            } else {
              x.w[y][0] = *(const uint32_t*)p;
            }
          }
        }
        return x;
      };
      Sub<NG> next = load(t0 * kTileSubs + warp);
      for (int s = t0 * kTileSubs + warp; s < sub1; s += kWarps) {
        const Sub<NG> x = next;
        next = load(s + kWarps);
        const bool edge = 16 * s + 16 > sees0;
        float sum[2] = {0.f, 0.f};
#pragma unroll 1
        for (int nt = 0; nt < blocks; ++nt) {
          // logits of tokens g8 and g8 + 8, query rows 2 t4 and 2 t4 + 1; sums of 64 dimensions, the low halves first
          float l[4];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int part = HILO ? 1 : 0; part >= 0; --part)
#pragma unroll
              for (int j = 2 * half; j < 2 * half + 2; ++j) {
                const uint4 q = S.frag[part][nt][j][lane];
                const uint32_t x0 = comp(x.c[0], j), x1 = comp(x.c[1], j), y0 = x0 >> 8, y1 = x1 >> 8;
                mma_16816(d, x0 & 0x000f000fu, x1 & 0x000f000fu, y0 & 0x000f000fu, y1 & 0x000f000fu, q.x, q.z);
                mma_16816(d, x0 & 0x00f000f0u, x1 & 0x00f000f0u, y0 & 0x00f000f0u, y1 & 0x00f000f0u, q.y, q.w);
              }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float unit = word_scale(x.w[e >> 1][half * (NG - 1)]);
              l[e] = half ? fmaf(unit, d[e], l[e]) : unit * d[e];
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 8 * nt + 2 * t4 + (e & 1);
            float y = fmaf(word_min(x.w[e >> 1][0]), S.qsum[r][0], -S.lse2[r]);
            if (NG == 2) y = fmaf(word_min(x.w[e >> 1][NG - 1]), S.qsum[r][NG - 1], y);
            float p = exp2_fast(fmaf(l[e], S.qscale[r], y));
            if (edge && 16 * s + g8 + 8 * (e >> 1) >= sees0 + (row0 + r) / v.G) p = 0.f;
            sum[e >> 1] += p;
          }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 1);
          sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 2);
          const int i = 16 * s + g8 + 8 * y;
          if (t4 == 0 && i < held) {
            bool fine = x.there;
#pragma unroll
            for (int g = 0; g < NG; ++g) fine = fine && finite_word(x.w[y][g]);
            float* to = a.now + b * a.nb + h * a.nh + i;
            const float old = row0 ? *to : a.was ? a.decay * a.was[b * a.wb + h * a.wh + i] : 0.f;
            *to = fine ? old + sum[y] : old;
          }
        }
      }
    }
    k += n;
    at += n;
    while (k < hi && at >= (int64_t)tiles_of(b) * v.H) at = 0, ++b;  // (rows without tokens have no tiles)
  }
}

template <int NG, bool HILO>
int launch(const WeightArgs& a, int sms, void* stream) {
  auto* kernel = akv_paged_weights_kernel<NG, HILO>;
  static_assert(sizeof(Smem) <= 48 * 1024, "shared memory without an attribute");
  return launch_after(kernel, dim3(2 * sms), kThreads, sizeof(Smem), stream, a);
}

}  // namespace

int launch_paged_weights(const PagedView& v, const akv_rows& q, const float* lse, int32_t T, float sm_scale, float decay,
                         const akv_scores* was, const akv_scores& now, void* stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return (int)e;
  WeightArgs a{};
  a.v = v;
  a.q = (const uint16_t*)q.ptr;
  a.qb = q.stride_b, a.qt = q.stride_t, a.qh = q.stride_h;
  a.lse = lse;
  if (was) a.was = was->ptr, a.wb = was->stride_b, a.wh = was->stride_h;
  a.now = now.ptr, a.nb = now.stride_b, a.nh = now.stride_h;
  a.scale = (float)((double)sm_scale * 1.4426950408889634);
  a.decay = decay;
  a.T = T;
  a.rows = T * v.G;
  if (v.rotate) return v.ng == 2 ? launch<2, true>(a, sms, stream) : launch<1, true>(a, sms, stream);
  return v.ng == 2 ? launch<2, false>(a, sms, stream) : launch<1, false>(a, sms, stream);
}

}  // namespace akv
