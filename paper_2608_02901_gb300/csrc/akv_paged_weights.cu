// Attention weights that the tokens of a paged cache got, added to their scores.
//
// The softmax's normaliser is known (lse), so a token's weight needs its own key alone: one pass over the key codes and their
// parameters, no reference, no join, and every score is written by one thread.  Two kernels:
//   up to 16 query rows a unit (a decode step): warp-level products of 16 tokens and 8 rows, codes straight from memory into operands
//     (nibbles as fp16 subnormals, as in the attention).  8 requests of 128 k tokens, 8 x 8 heads, rotated: 197 us, 671 MB (3.4 TB/s); an instruction is
//     issued in 67 % of the cycles, ALU 45 %, FMA 31 %, tensor 29 %: the unpacking, the sums' way into logits and the two halves' products.
//   more rows (a prompt's last tokens): S = K Q^T on the fifth-generation tensor cores with the tokens as rows.  A thread owns a token:
//     it turns the codes into its lane of the operand in tensor memory, applies the token's scales to the products behind them,
//     and adds its weights up along its lane without a shuffle; the queries are the columns.  64 query tokens, 8 x 4 heads, over 32 k tokens:
//     48.5 us (53 with 16 columns a load), 8 of them until the first product; then a block's 17 products take 550 cycles to issue, its weights 700.
// In both, tiles of all units (request, KV head) go in equal contiguous ranges to the CTAs.
//   With codes in the products and scales outside, a logit is k (a_0 S_0 + a_1 S_1 + m_0 sum q_0 + m_1 sum q_1) over the groups of dimensions, with
// c - 7.5 for c and m + 7.5 a for m (of many rows twice that), and a weight 2 to that less lse, which is subtracted in such parts that it
// costs no rounding of its own.  Codes from 0 up would make sums that are larger than what they leave.
//   Warp-level products cut their sums off at 24 bits of the largest term.  So of few rows the high halves of the queries are whole numbers of
// 11 bits times a power of two of the row: their sums with codes are exact, and begin at -7.5 times the row's sum, which centres the codes;
// the low halves (of rows that are not rotated too) have sums of their own.  With both halves' products in one sum, and codes from 0 up, a
// weight was off by 1e-6 to 5e-6 of its size, now by 1e-7 to 5e-7, for 4 to 7 % of the time of up to 8 rows and 20 % of 16 rows that are not rotated.
#include <cuda_runtime.h>

#include <atomic>

#include "akv_device.cuh"
#include "akv_paged.cuh"
#include "akv_paged_tc.cuh"

namespace akv {
namespace {

constexpr int kTile = 128;                           // tokens of a tile
constexpr float kInf = __builtin_huge_valf();

struct WeightArgs {
  PagedView v;
  const uint16_t* q;
  const uint8_t* queries;  // many rows: their records
  const float* lse;
  const float* was;
  float* now;
  int64_t qb, qt, qh, wb, wh, nb, nh;
  float scale, decay;  // scale: sm_scale log2(e)
  int T, rows;         // rows: query rows of a unit, T G
  int aligned;         // every query row begins at a multiple of 8 bytes
};

// A unit's share of a CTA: tiles t0 .. t0 + n - 1 of request b, head h.
struct Segment {
  int b, h, held, tiles, t0, n;
};
__device__ __forceinline__ int tiles_of(const WeightArgs& a, int b) { return (held_tokens(a.v, b) + kTile - 1) / kTile; }
__device__ __forceinline__ void open(const WeightArgs& a, Segment& s) {
  s.held = held_tokens(a.v, s.b);
  s.tiles = (s.held + kTile - 1) / kTile;
}
// The segment after s, `left` tiles of the CTA's range still to go (> 0).
__device__ __forceinline__ void next_segment(const WeightArgs& a, Segment& s, int64_t left) {
  s.t0 = 0;
  if (++s.h == a.v.H) {
    s.h = 0;
    do ++s.b;
    while (s.b + 1 < a.v.rows && tiles_of(a, s.b) == 0);  // (rows without tokens have no tiles)
    open(a, s);
  }
  s.n = (int)min((int64_t)s.tiles, left);
}

// The CTA's range lo .. hi - 1 of all units' tiles, and its first segment; false: none.  All threads call it.
template <int kThreads>
__device__ __forceinline__ bool plan(const WeightArgs& a, int64_t* part, int64_t* place, Segment& seg, int64_t& lo, int64_t& hi) {
  const PagedView& v = a.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int strip = (v.rows + kThreads - 1) / kThreads, b0 = min(v.rows, tid * strip), b1 = min(v.rows, b0 + strip);
  int64_t mine = 0, total = 0;
  for (int b = b0; b < b1; ++b) mine += (int64_t)tiles_of(a, b) * v.H;
  int64_t inc = mine;
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    const int64_t o = __shfl_up_sync(0xffffffffu, inc, s);
    if (lane >= s) inc += o;
  }
  if (lane == 31) part[warp] = inc;
  __syncthreads();
  int64_t before = inc - mine;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += part[w];
    total += part[w];
  }
  lo = blockIdx.x * total / gridDim.x, hi = (blockIdx.x + 1) * total / gridDim.x;
  if (lo >= hi) return false;
  if (lo >= before && lo < before + mine) {
    int64_t rest = lo - before;
    int b = b0;
    for (;; ++b) {
      const int64_t here = (int64_t)tiles_of(a, b) * v.H;
      if (rest < here) break;
      rest -= here;
    }
    place[0] = b, place[1] = rest;
  }
  __syncthreads();
  seg.b = (int)place[0];
  open(a, seg);
  seg.h = (int)(place[1] / seg.tiles), seg.t0 = (int)(place[1] % seg.tiles);
  seg.n = (int)min((int64_t)(seg.tiles - seg.t0), hi - lo);
  return true;
}

// A query row as it lies in memory, four values a lane.
struct RowRaw {
  uint2 x;
  float lse;
};
__device__ __forceinline__ RowRaw fetch_row(const WeightArgs& a, const Segment& seg, int row) {
  RowRaw r{make_uint2(0, 0), kInf};
  if (row < a.rows) {
    const PagedView& v = a.v;
    const int lane = threadIdx.x & 31, t = row / v.G, g = row % v.G;
    const uint16_t* q = a.q + seg.b * a.qb + t * a.qt + (int64_t)(seg.h * v.G + g) * a.qh + 4 * lane;
    r.x = a.aligned ? *(const uint2*)q : make_uint2(q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16);
    r.lse = a.lse[((int64_t)seg.b * a.T + t) * (v.H * v.G) + seg.h * v.G + g];
  }
  return r;
}
// R rows' values, rotated where the cache is, times the sign of the scale; zeros, and lse infinite, where a row adds nothing: no finite lse, or an
// infinity or a NaN of its own.
template <bool HILO, int R>
__device__ __forceinline__ void open_rows(const WeightArgs& a, const RowRaw (&raw)[R], float (&x)[R][4], float (&lse)[R]) {
  const PagedView& v = a.v;
  const int lane = threadIdx.x & 31;
  const uint32_t sign = a.scale < 0.f ? 0x80000000u : 0u;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    lse[r] = raw[r].lse;
    bool fine = fabsf(lse[r]) < kInf;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[r][e] = row_to_float((uint16_t)((e < 2 ? raw[r].x.x : raw[r].x.y) >> (16 * (e & 1))), v.half);
      fine = fine && fabsf(x[r][e]) < kInf;
    }
    const bool counts = __all_sync(0xffffffffu, fine);
    if (!counts) lse[r] = kInf;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[r][e] = counts ? __uint_as_float(__float_as_uint(x[r][e]) ^ sign ^ (HILO ? sign_flip(v, 4 * lane + e) : 0u)) : 0.f;
  }
  if (HILO) {  // q' = H (s o q) / 16
    wht_rows(x, lane);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[r][e] *= 0.0625f;
  }
}
// lse in log2 units as fp32 and what that leaves out.
__device__ __forceinline__ void lse_log2(float lse, float& hi, float& lo) {
  constexpr float c = 1.44269504f, c_rest = 1.92596299e-8f;  // log2(e) in two parts
  hi = lse * c;
  lo = fabsf(lse) < kInf ? fmaf(lse, c, -hi) + lse * c_rest : 0.f;
}
__device__ __forceinline__ bool finite_word(uint32_t w) { return (w & 0x7c00u) != 0x7c00u && (w & 0x7c000000u) != 0x7c000000u; }
__device__ __forceinline__ float word_scale(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)w)); }
__device__ __forceinline__ float word_min(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
__device__ __forceinline__ uint32_t comp(const uint4& x, int j) { return j == 0 ? x.x : j == 1 ? x.y : j == 2 ? x.z : x.w; }

// ---- few query rows -----------------------------------------------------------------------------
// A warp takes two sub-blocks of 16 tokens at a time (of 16 rows one), the next on their way meanwhile, their pages known a step earlier still.

constexpr int kFewWarps = 8, kFewThreads = 32 * kFewWarps;

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int NT>
struct FewSmem {
  uint4 frag[2][NT][4][32];     // query operand: high, low halves
  // of a row, in what its products count: sums over each group, what its two sums of products begin at, the part of -lse that goes with them;
  // what they count, the rest of -lse
  float2 qsum[8 * NT], start[2][8 * NT], k[8 * NT];
  float lse_in[8 * NT];
  int64_t part[kFewWarps], place[2];
};

template <int NG>
struct Sub {  // key codes and parameters of a sub-block, a lane's part: tokens g8, g8 + 8
  uint4 c[2];
  uint32_t w[2][NG];
};

template <int NG, int NT, bool HILO>
__global__ void __launch_bounds__(kFewThreads, 2) akv_paged_weights_few_kernel(const __grid_constant__ WeightArgs a) {
  __shared__ FewSmem<NT> S;
  constexpr uint32_t kSub = 2048 + 128 * NG;
  constexpr int kSubs = NT == 1 ? 2 : 1, kStep = kFewWarps * kSubs;  // (two of 16 rows spill)
  const PagedView& v = a.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
  launch_dependents();
  wait_for_stream();
  Segment seg;
  int64_t lo, hi;
  if (!plan<kFewThreads>(a, S.part, S.place, seg, lo, hi)) return;

  for (int64_t at = lo; at < hi;) {
    const int first = seg.t0 * (kTile / 16), end = min((seg.t0 + seg.n) * (kTile / 16), (seg.held + 15) >> 4);
    auto page_at = [&](int s) {  // as the table says (looked at when it is used)
      return s < end ? v.table[(int64_t)seg.b * v.table_stride + (16 * s >> v.page_log)] : -1;
    };
    auto place = [&](int s, int page) {
      return block_of(v, page, seg.h) + (uint64_t)((16 * s & ((1 << v.page_log) - 1)) >> 4) * kSub;
    };
    auto load = [&](int s, int page) {  // (no token, or a page that is none of the pool's: NaN parameters)
      Sub<NG> x;
      if ((uint32_t)page < (uint32_t)v.n_pages) {
        const uint8_t* base = place(s, page);
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
      } else {
        x.c[0] = x.c[1] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int g = 0; g < NG; ++g) x.w[y][g] = 0x7e007e00u;
      }
      return x;
    };
    const int mine = first + kSubs * warp;
    int page[kSubs], far[kSubs];
    Sub<NG> next[kSubs];
#pragma unroll
    for (int i = 0; i < kSubs; ++i) page[i] = page_at(mine + i);
#pragma unroll
    for (int i = 0; i < kSubs; ++i) {
      next[i] = load(mine + i, page[i]);
      page[i] = page_at(mine + kStep + i);
      far[i] = page_at(mine + 2 * kStep + i);
    }

    // ---- queries: a warp per row, four dimensions a lane
    __syncthreads();
#pragma unroll 1
    for (int rr = warp; rr < 8 * NT; rr += kFewWarps) {
      const RowRaw raw[1] = {fetch_row(a, seg, rr)};
      float x1[1][4], lse1[1];
      open_rows<HILO>(a, raw, x1, lse1);
      float(&x)[4] = x1[0];
      const float lse = lse1[0];
      float big = fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3])));
      big = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(big)));
      const int e2 = min(max((int)(__float_as_uint(big) >> 23) - 126, -100), 128);
      const float up = pow2(14 - e2);  // below 2^14, exact in fp16 down to 2^-23 of that
      // What the products count.  Rows of zeros, and scales of (nearly) zero, have logits below 1e-27, and what -lse has below 2^-8 would not
      // go with their products: such rows are zeros, whose products count 1.
      float k = fabsf(a.scale) * pow2(e2 - 10) * 1048576.f;
      if (!(k > 2e-33f)) {
        k = 1.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = 0.f;
      }
      // the high half is a multiple of 2^-11 of the largest's power of two: sums of its products with codes are exact in 24 bits
      float high[4], sum[2];
#pragma unroll
      for (int e = 0; e < 4; ++e) high[e] = 8.f * rintf(x[e] * (0.125f * up));
      sum[0] = (high[0] + high[1]) + (high[2] + high[3]);
      sum[1] = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[1] += fmaf(x[e], up, -high[e]);
#pragma unroll
      for (int s = 1; s < 32 / NG; s *= 2)
#pragma unroll
        for (int y = 0; y < 2; ++y) sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], s);
      // (codes count 2^-24 in the products, and so does what is added to them)
      if (lane % (32 / NG) == 0) {
        const int g = lane / (32 / NG);
        constexpr float c = 5.9604644775390625e-8f;
        ((float*)&S.qsum[rr])[g] = (sum[0] + sum[1]) * c;
        S.start[g][rr] = make_float2(-7.5f * c * sum[0], -7.5f * c * sum[1]);
      }
      if (lane == 0) {
        float l, rest;
        lse_log2(lse, l, rest);
        const float coarse = fabsf(l) < 8192.f ? rintf(l * 256.f) * 0.00390625f : l;
        const float in = (rest + (l - coarse)) / k;  // (below 1e30 but for an lse beyond 8192, or a row that adds nothing)
        S.k[rr] = make_float2(k, -coarse), S.lse_in[rr] = fabsf(in) < 1e30f ? -in : 0.f;
      }
      uint4 f[2];
#pragma unroll
      for (int low = 0; low < 2; ++low) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // nibble e: odd ones stand for 16 times their value
          const float own = (low ? fmaf(x[e], up, -high[e]) : high[e]) * (e & 1 ? 0.0625f : 1.f);
          const float other = __shfl_xor_sync(0xffffffffu, own, 1);
          w[e] = lane & 1 ? half2_bits(other, own) : half2_bits(own, other);
        }
        f[low] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      // lanes 2 x and 2 x + 1 hold dimensions 8 x ..: word j = x / 4, operand lane 4 row + x % 4
      const int to = 4 * (rr & 7) + (lane >> 1 & 3);
      if (!(lane & 1)) S.frag[0][rr >> 3][lane >> 3][to] = f[0];
      if (lane & 1) S.frag[1][rr >> 3][lane >> 3][to] = f[1];
    }
    __syncthreads();

    const float* was = a.was ? a.was + seg.b * a.wb + seg.h * a.wh : nullptr;
    float* now = a.now + seg.b * a.nb + seg.h * a.nh;
    const int sees0 = seg.held - a.T + 1;  // tokens that the first query token sees
#pragma unroll 1
    for (int s0 = mine; s0 < end; s0 += kStep) {
      Sub<NG> x[kSubs];
#pragma unroll
      for (int i = 0; i < kSubs; ++i) x[i] = next[i];
#pragma unroll
      for (int i = 0; i < kSubs; ++i) {
        next[i] = load(s0 + kStep + i, page[i]);
        page[i] = far[i];
        far[i] = page_at(s0 + 3 * kStep + i);
      }
      float old[kSubs][2], sum[kSubs][2];
#pragma unroll
      for (int i = 0; i < kSubs; ++i)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int tok = 16 * (s0 + i) + g8 + 8 * y;
          old[i][y] = was && t4 == 0 && tok < seg.held && s0 + i < end ? was[tok] : 0.f;
          sum[i][y] = 0.f;
        }
      const bool edge = 16 * (s0 + kSubs) > sees0;  // some row may not see some token
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        // products of tokens g8 and g8 + 8 with query rows 2 t4 and 2 t4 + 1 over a group of dimensions, the high halves' and the low ones'
        // apart: the first are whole numbers of 22 bits, the second's cut does not count
        float z[kSubs][4], d[kSubs][4], rest[kSubs][4];
        float2 k[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) k[r] = S.k[8 * nt + 2 * t4 + r];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int g = NG == 2 ? j >> 1 : 0;
          if (j == 0 || (NG == 2 && j == 2)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 y = S.start[g][8 * nt + 2 * t4 + (e & 1)];
#pragma unroll
              for (int i = 0; i < kSubs; ++i) d[i][e] = y.x, rest[i][e] = y.y;
            }
          }
          const uint4 q0 = S.frag[0][nt][j][lane], q1 = S.frag[1][nt][j][lane];
#pragma unroll
          for (int i = 0; i < kSubs; ++i) {
            const uint32_t x0 = comp(x[i].c[0], j), x1 = comp(x[i].c[1], j), y0 = x0 >> 8, y1 = x1 >> 8;
            const uint32_t e0 = x0 & 0x000f000fu, e1 = x1 & 0x000f000fu, e2 = y0 & 0x000f000fu, e3 = y1 & 0x000f000fu;
            const uint32_t o0 = x0 & 0x00f000f0u, o1 = x1 & 0x00f000f0u, o2 = y0 & 0x00f000f0u, o3 = y1 & 0x00f000f0u;
            mma_16816(d[i], e0, e1, e2, e3, q0.x, q0.z);
            mma_16816(rest[i], e0, e1, e2, e3, q1.x, q1.z);
            mma_16816(d[i], o0, o1, o2, o3, q0.y, q0.w);
            mma_16816(rest[i], o0, o1, o2, o3, q1.y, q1.w);
          }
          // a (c - 7.5) . q + (m + 7.5 a) sum q
          if (j == 3 || (NG == 2 && j == 1)) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int row = 8 * nt + 2 * t4 + r;
              const float qsum = g ? S.qsum[row].y : S.qsum[row].x, lse_in = S.lse_in[row];
#pragma unroll
              for (int i = 0; i < kSubs; ++i)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                  const float scale = word_scale(x[i].w[y][g]), mid = fmaf(7.5f, scale, word_min(x[i].w[y][g]));
                  float& to = z[i][2 * y + r];
                  to = fmaf(mid, qsum, g ? to : lse_in);
                  to = fmaf(scale, d[i][2 * y + r] + rest[i][2 * y + r], to);
                }
            }
          }
        }
#pragma unroll
        for (int i = 0; i < kSubs; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[i][e] = fmaf(z[i][e], k[e & 1].x, k[e & 1].y);
        if (edge) {
#pragma unroll
          for (int i = 0; i < kSubs; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (16 * (s0 + i) + g8 + 8 * (e >> 1) >= sees0 + (8 * nt + 2 * t4 + (e & 1)) / v.G) z[i][e] = -kInf;
        }
#pragma unroll
        for (int i = 0; i < kSubs; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[i][e >> 1] += exp2_fast(z[i][e]);
      }
#pragma unroll
      for (int i = 0; i < kSubs; ++i)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          sum[i][y] += __shfl_xor_sync(0xffffffffu, sum[i][y], 1);
          sum[i][y] += __shfl_xor_sync(0xffffffffu, sum[i][y], 2);
          const int tok = 16 * (s0 + i) + g8 + 8 * y;
          if (t4 == 0 && tok < seg.held && s0 + i < end) {
            bool fine = true;
#pragma unroll
            for (int g = 0; g < NG; ++g) fine = fine && finite_word(x[i].w[y][g]);
            now[tok] = fine ? fmaf(a.decay, old[i][y], sum[i][y]) : a.decay * old[i][y];
          }
        }
    }
    at += seg.n;
    if (at < hi) next_segment(a, seg, hi - at);
  }
}

// ---- many query rows ----------------------------------------------------------------------------
// Two warpgroups take the tiles in turn, a warp for each issues its products, 32 columns a time into two buffers.  Queries of up to 256 rows lie in shared memory as
// operands; a unit with more goes over its tiles again for each 256.

constexpr int W = 2, kWorkers = 4 * W, kThreads = 128 * (W + 1);
constexpr int kCols = 32, kBlocks = 8, kHeld = kBlocks * kCols;  // query rows of a product, and in shared memory
// Tensor memory: the warpgroups' keys, then of each two buffers of sums over the first group of dimensions (or all), the second, and the rest
constexpr uint32_t kColK = 0, kColS = 64 * W, kColsS = 3 * kCols;
constexpr float kOnes = 16.f;  // the dimensions that carry lse count 16

struct Smem {
  uint8_t q[2][4 * kPanel];  // 128 rows each: high, then low halves
  uint8_t qx[2][kExtra], kx[W][kExtra];
  alignas(16) float k[kHeld], lse[kHeld];  // what a row's products count; the part of -lse behind them (-infinity: the row adds nothing)
  int sees[kHeld];             // tokens that it sees
  int behind[kBlocks];         // whether a block has rows with such a part
  uint64_t k_full[W], s_full[W][2], s_free[W][2], drained[W];
  int64_t part[4 * W + 4], place[2];
  uint32_t tmem;
  int failed;
};

template <int NG, bool HILO>
__global__ void __launch_bounds__(kThreads, 1) akv_paged_weights_kernel(const __grid_constant__ WeightArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Smem& S = *reinterpret_cast<Smem*>(smem_raw + (1024u - (smem_u32(smem_raw) & 1023u)) % 1024u);
  constexpr uint32_t kSub = 2048 + 128 * NG;
  const PagedView& v = a.v;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  volatile int* failed = &S.failed;
  launch_dependents();
  if (tid == 0) {
    for (int w = 0; w < W; ++w) {
      mbar_init(smem_u32(&S.k_full[w]), 4);
      for (int b = 0; b < 2; ++b) {
        mbar_init(smem_u32(&S.s_full[w][b]), 1);
        mbar_init(smem_u32(&S.s_free[w][b]), 4);
      }
    }
    for (int w = 0; w < W; ++w) mbar_init(smem_u32(&S.drained[w]), 1);
    S.failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_stream();
  Segment seg;
  int64_t lo, hi;
  if (!plan<kThreads>(a, S.part, S.place, seg, lo, hi)) return;
  if (warp == kWorkers) tc_alloc(smem_u32(&S.tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, S.tmem, 0);
  const int passes = (a.rows + kHeld - 1) / kHeld;
  auto rows_of = [&](int pass) { return min(kHeld, a.rows - pass * kHeld); };
  auto columns = [](int rows, int block) { return min(kCols, (rows - block * kCols + 15) & ~15); };

  if (warp >= kWorkers && warp < kWorkers + W) {
    // ---- the products of a warpgroup's tiles, a block of columns after the other.  Keys of a tile tell that the queries are there
    // too: every warp of the warpgroup has passed the barrier behind them.  (A barrier for queries alone would go on without the
    // warp where its warpgroup has no tile, and two phases of it look alike.)
    const int w = warp - kWorkers;
    uint32_t n_k = 0, n_s = 0;
    bool ok = true;
    const uint32_t k = tmem + kColK + 64 * w, d0 = tmem + kColS + 2 * kColsS * w;
    const uint64_t dkx = plain_desc(smem_u32(S.kx[w]));
    for (int64_t at = lo; ok && at < hi;) {
      for (int pass = 0; ok && pass < passes; ++pass) {
        const int rows = rows_of(pass), blocks = (rows + kCols - 1) / kCols;
#pragma unroll 1
        for (int i = w; ok && i < seg.n; i += W) {
          ok = mbar_wait_w(smem_u32(&S.k_full[w]), n_k++ & 1) && !warp_failed(failed);
#pragma unroll 1
          for (int block = 0; ok && block < blocks; ++block, ++n_s) {
            const uint32_t n = (uint32_t)columns(rows, block), idesc = (1u << 4) | ((n >> 3) << 17) | ((128u >> 4) << 24);
            const int held_at = block * kCols / 128, row_at = block * kCols % 128;  // the block's rows
            const uint32_t b = n_s & 1;
            ok = mbar_wait_w(smem_u32(&S.s_free[w][b]), (n_s >> 1 & 1) ^ 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              const uint32_t d = d0 + kColsS * b;
              const uint64_t dq = sw128_desc(smem_u32(S.q[held_at]) + 128 * row_at);
              auto product = [&](uint32_t to, int first_step, int steps, uint64_t desc, bool first) {
#pragma unroll
                for (int i = 0; i < steps; ++i) {
                  const int kk = first_step + i;
                  tc_mma_ts(to, k + 8 * kk, desc + (((uint32_t)(kk >> 2) * kPanel + (uint32_t)(kk & 3) * 32) >> 4), idesc, !first || i > 0);
                }
              };
              constexpr uint64_t low = 2 * kPanel >> 4;
#pragma unroll
              for (int g = 0; g < NG; ++g) {
                if (HILO) product(d + kCols * g, 8 / NG * g, 8 / NG, dq + low, true);
                product(d + kCols * g, 8 / NG * g, 8 / NG, dq, !HILO);
              }
              tc_mma(d + 2 * kCols, dkx, plain_desc(smem_u32(S.qx[held_at]) + extra_at(row_at)), idesc, 0);
              tc_commit(smem_u32(&S.s_full[w][b]));
            }
            __syncwarp();
          }
        }
      }
      at += seg.n;
      if (at < hi) next_segment(a, seg, hi - at);
    }
    if (!ok) *failed = 1;
    if (elect_one()) tc_commit(smem_u32(&S.drained[w]));
    __syncwarp();
    mbar_wait_w(smem_u32(&S.drained[w]), 0);  // nothing is under way when tensor memory is given back
  } else if (warp < kWorkers) {
    // ---- a warpgroup, a thread a token
    const int w = warp >> 2, token = tid & 127;
    const uint32_t lane_at = tmem + ((uint32_t)((warp & 3) * 32) << 16), tK = lane_at + kColK + 64 * w, tS0 = lane_at + kColS + 2 * kColsS * w;
    const uint32_t kx_at = smem_u32(S.kx[w]) + extra_at(token);
    const KeyCodes codes;
    uint32_t n_s = 0;
    uint4 kc[4];
    uint32_t kw[NG];
    int page;
    auto page_at = [&](const Segment& s, int i) {  // as the table says (looked at when it is used)
      const int tok = (s.t0 + i) * kTile + token;
      return i < s.n && tok < s.held ? v.table[(int64_t)s.b * v.table_stride + (tok >> v.page_log)] : -1;
    };
    auto load = [&](const Segment& s, int i, int pg) {
      if ((uint32_t)pg < (uint32_t)v.n_pages) {
        const int tok = (s.t0 + i) * kTile + token;
        const uint8_t* p = block_of(v, pg, s.h) + (uint64_t)((tok & ((1 << v.page_log) - 1)) >> 4) * kSub;
        const uint4* k = (const uint4*)(p + 64 * (tok & 15));
#pragma unroll
        for (int t = 0; t < 4; ++t) kc[t] = k[t];
        if (NG == 2) {
          const uint2 x = *(const uint2*)(p + 2048 + 16 * (tok & 15));
          kw[0] = x.x, kw[NG - 1] = x.y;
        } else {
          kw[0] = *(const uint32_t*)(p + 2048 + 8 * (tok & 15));
        }
      } else {  // no token, or a page that is none of the pool's: adds nothing
#pragma unroll
        for (int t = 0; t < 4; ++t) kc[t] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < NG; ++g) kw[g] = 0x7e007e00u;
      }
    };
    load(seg, w, page_at(seg, w));
    page = page_at(seg, w + W);
    for (int64_t at = lo; at < hi;) {
      Segment after = seg;
      const bool more = at + seg.n < hi;
      if (more) next_segment(a, after, hi - at - seg.n);
      const float* was = a.was ? a.was + seg.b * a.wb + seg.h * a.wh : nullptr;
      float* now = a.now + seg.b * a.nb + seg.h * a.nh;
      for (int pass = 0; pass < passes; ++pass) {
        const int rows = rows_of(pass), blocks = (rows + kCols - 1) / kCols;
        // queries as operands (the products of the pass before have been waited for by every warpgroup)
        named_sync(1, 32 * kWorkers);
        if (tid < kBlocks) S.behind[tid] = 0;
        named_sync(1, 32 * kWorkers);
        const int padded = (blocks - 1) * kCols + columns(rows, blocks - 1);
        auto record_of = [&](int rr) {
          const int row = pass * kHeld + rr, t = row / v.G, g = row % v.G;
          return rr < rows ? a.queries + (((int64_t)seg.b * a.T + t) * (v.H * v.G) + seg.h * v.G + g) * kQueryRecord : nullptr;
        };
        float2 own = make_float2(1.f, 0.f);
        float lse = kInf;
        if (tid < rows) {
          const int row = pass * kHeld + tid;
          own = *(const float2*)(record_of(tid) + 544);
          lse = a.lse[((int64_t)seg.b * a.T + row / v.G) * (v.H * v.G) + seg.h * v.G + row % v.G];
        }
#pragma unroll 1
        for (int r0 = 16 * warp; r0 < padded; r0 += 16 * kWorkers)  // (padded is a multiple of 16)
          place_queries<HILO, 16>(
              lane, record_of(r0 + (lane & 15)),
              [&](int r, int& row, uint32_t& panels, uint32_t& extra) {
                row = (r0 + r) & 127, panels = smem_u32(S.q[r0 >> 7]), extra = smem_u32(S.qx[r0 >> 7]);
              });
        named_sync(1, 32 * kWorkers);
        // -lse goes with the products in three parts where it fits them (rows so small that it does not: behind them); a thread a row
        if (tid < padded) {
          if (own.y == 0.f) lse = kInf;
          const float k = 0.5f * fabsf(a.scale) * own.x, inv = 1.f / (k * kOnes);  // (keys enter twice as large)
          float l, rest;
          lse_log2(lse, l, rest);
          float in = -l * inv, in_rest = (fmaf(-in * kOnes, k, -l) - rest) * inv;
          const bool fits = fabsf(in) < 32768.f;
          if (!fits) in = in_rest = 0.f, S.behind[tid / kCols] = 1;
          uint16_t* to = (uint16_t*)(S.qx[tid >> 7] + extra_at(tid & 127) + 2048) + 2;
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            const __half p = __float2half_rn(in);
            to[i] = __half_as_ushort(p);
            in = in - __half2float(p) + (i == 0 ? in_rest : 0.f);
          }
          S.k[tid] = k, S.lse[tid] = fits ? 0.f : -l;
          S.sees[tid] = min(seg.held, seg.held - a.T + 1 + (pass * kHeld + tid) / v.G);
        }
        proxy_fence();
        __syncwarp();
        named_sync(1, 32 * kWorkers);

        bool ok = true;
#pragma unroll 1
        for (int i = w; i < seg.n; i += W) {
          // ---- the token's codes into tensor memory
          bool fine = true;
          float scale[NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) fine = fine && finite_word(kw[g]);
          uint32_t words[NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) words[g] = fine ? kw[g] : 0u, scale[g] = word_scale(words[g]);
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            float x[32];
#pragma unroll
            for (int jj = 0; jj < 2; ++jj)
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                const uint32_t word = comp(kc[t], 2 * p + jj), x2 = word << 1, y2 = word >> 7;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[16 * jj + 4 * t + e] = __uint_as_float(bits(codes(x2, y2, e)));
              }
            tm_st32(tK + 32 * p, x);
          }
          // (2 m + 15 a beyond fp16's range: 2^-5 of it, and of lse)
          bool big = false;
#pragma unroll
          for (int g = 0; g < NG; ++g) big = big || scale[g] > 2048.f || fabsf(word_min(words[g])) > 16384.f;
          const float down = big ? kLargeDown : 1.f, back = big ? 32.f : 1.f;
          uint4 first, second;
          key_extra<NG>(words, down, false, kOnes * down, first, second);
          sts128(kx_at, first);
          sts128(kx_at + 2048, second);
          tm_wait_st();
          tc_fence_before();
          proxy_fence();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&S.k_full[w]));
          // the warpgroup's next tile is under way meanwhile
          if (i + W < seg.n) {
            load(seg, i + W, page);
            page = page_at(seg, i + 2 * W);
          }
          const int tok = (seg.t0 + i) * kTile + token;
          const bool held = tok < seg.held;
          float old = 0.f;
          if (held) old = pass ? now[tok] : was ? a.decay * was[tok] : 0.f;
          const bool edge = (seg.t0 + i + 1) * kTile > seg.held - a.T + 1;  // some row may not see some token
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float2 s0 = make_float2(scale[0], scale[0]), s1 = make_float2(scale[NG - 1], scale[NG - 1]), b2 = make_float2(back, back);
#pragma unroll 1
          for (int block = 0; block < blocks; ++block) {
            const uint32_t b = n_s & 1, use = n_s >> 1 & 1, tS = tS0 + kColsS * b;
            ++n_s;
            if (!ok || warp_failed(failed) || !mbar_wait_w(smem_u32(&S.s_full[w][b]), use)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const int n = columns(rows, block);
            const bool behind = edge || *(volatile int*)&S.behind[block];
            const float* ks = &S.k[block * kCols];
            // the logits, in log2 units less lse, of two columns
            auto logit = [&](float x0, float x1, float y0, float y1, float z0, float z1, float2 k) {
              float2 l = __fmul2_rn(make_float2(z0, z1), b2);  // (by a power of two)
              if (NG == 2) l = __ffma2_rn(s1, make_float2(y0, y1), l);
              return __fmul2_rn(__ffma2_rn(s0, make_float2(x0, x1), l), k);
            };
            if (n == kCols && !behind) {
              float x[NG == 2 ? 3 : 2][32];
              tm_ld32xn(tS, x);
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const float4 k = *(const float4*)(ks + e);
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                  float2 l = logit(x[0][e + i], x[0][e + i + 1], x[NG - 1][e + i], x[NG - 1][e + i + 1], x[NG][e + i], x[NG][e + i + 1],
                                   i ? make_float2(k.z, k.w) : make_float2(k.x, k.y));
                  l.x = exp2_fast(l.x), l.y = exp2_fast(l.y);
                  sum[i >> 1] = __fadd2_rn(sum[i >> 1], l);
                }
              }
            } else {
#pragma unroll 1
              for (int c = 0; c < n; c += 16) {
                float x[16], y[16], z[16];
                tm_ld16x3(tS + c, tS + (NG - 1) * kCols + c, tS + 2 * kCols + c, x, y, z);
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                  const int at = block * kCols + c + e;
                  float2 l = logit(x[e], x[e + 1], y[e], y[e + 1], z[e], z[e + 1], *(const float2*)(ks + c + e));
                  if (behind) {
                    const float2 lse = *(const float2*)&S.lse[at];
                    const int2 sees = *(const int2*)&S.sees[at];
                    l.x = tok < sees.x ? l.x + lse.x : -kInf;
                    l.y = tok < sees.y ? l.y + lse.y : -kInf;
                  }
                  l.x = exp2_fast(l.x), l.y = exp2_fast(l.y);
                  sum[e >> 1 & 1] = __fadd2_rn(sum[e >> 1 & 1], l);
                }
              }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&S.s_free[w][b]));
          }
          if (held) now[tok] = ok ? (fine ? old + ((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y)) : old) : __int_as_float(0x7fffffff);
        }
        if (!ok) *failed = 1;
        // the first tile of what comes next
        if (pass + 1 < passes) {
          load(seg, w, page_at(seg, w));
          page = page_at(seg, w + W);
        } else if (more) {
          load(after, w, page_at(after, w));
          page = page_at(after, w + W);
        }
      }
      at += seg.n;
      seg = after;
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kWorkers) tc_dealloc(tmem, 512);
}

// Query rows up to which the first kernel is the faster one: 16 rows over 325 k tokens of 8 heads 86 us there, 118 in the second; the first has no
// registers for more.
constexpr int kFew = 16;

template <int NG, bool HILO>
int launch(const WeightArgs& a, int dev, int sms, void* stream) {
  if (a.rows <= 8) return launch_after(akv_paged_weights_few_kernel<NG, 1, HILO>, dim3(2 * sms), kFewThreads, 0, stream, a);
  if (a.rows <= kFew) return launch_after(akv_paged_weights_few_kernel<NG, 2, HILO>, dim3(2 * sms), kFewThreads, 0, stream, a);
  auto* kernel = akv_paged_weights_kernel<NG, HILO>;
  constexpr size_t smem = sizeof(Smem) + 1024;
  static_assert(smem <= 232448, "shared memory of a CTA");
  static std::atomic<uint64_t> ready{0};  // devices on which the kernel's shared memory has been set
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return (int)e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_after(kernel, dim3(sms), kThreads, smem, stream, a);
}

}  // namespace

size_t paged_weights_ws_bytes(const PagedView& v, int32_t T) {
  return T * v.G <= kFew ? 256 : ((size_t)v.rows * T * v.H * v.G * kQueryRecord + 255) & ~(size_t)255;
}

int launch_paged_weights(const PagedView& v, const akv_rows& q, const float* lse, int32_t T, float sm_scale, float decay,
                         const akv_scores* was, const akv_scores& now, void* ws, void* stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return (int)e;
  WeightArgs a{};
  a.v = v;
  a.q = (const uint16_t*)q.ptr;
  a.qb = q.stride_b, a.qt = q.stride_t, a.qh = q.stride_h;
  a.aligned = (uintptr_t)q.ptr % 8 == 0 && q.stride_b % 4 == 0 && q.stride_t % 4 == 0 && q.stride_h % 4 == 0;
  a.lse = lse;
  if (was) a.was = was->ptr, a.wb = was->stride_b, a.wh = was->stride_h;
  a.now = now.ptr, a.nb = now.stride_b, a.nh = now.stride_h;
  a.scale = (float)((double)sm_scale * 1.4426950408889634);
  a.decay = decay;
  a.T = T;
  a.rows = T * v.G;
  if (a.rows > kFew) {
    a.queries = (const uint8_t*)ws;
    const int err = launch_paged_queries(v, q, T, sm_scale < 0.f, lse, nullptr, nullptr, ws, stream);
    if (err) return err;
  }
  if (v.rotate) return v.ng == 2 ? launch<2, true>(a, dev, sms, stream) : launch<1, true>(a, dev, sms, stream);
  return v.ng == 2 ? launch<2, false>(a, dev, sms, stream) : launch<1, false>(a, dev, sms, stream);
}

}  // namespace akv
