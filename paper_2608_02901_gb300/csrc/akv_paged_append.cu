// Paged 4-bit cache: quantising new tokens into their pages, and reading rows back.
//
// Both move a row between 256 dense bytes and 64 + 4 NG held ones; what bounds them is the operations per value (16
// an element appended with rotation, 10 read back, where the bytes alone would leave room for 14), so the layout saves
// those.  Four lanes share a row: lane u of them holds dimensions 32 c + 8 u + n (c < 4, n < 8), so that
//   - the dense side is four 16-byte accesses a lane, 64 contiguous bytes a row each time;
//   - the key codes of a lane are the 16 contiguous bytes of its row's words 4 u .. 4 u + 3, the value codes (after an
//     exchange with the neighbouring token's lanes, whose halves share the words) one 16-byte unit;
//   - a warp's 8 rows are operands of the tensor cores as they were loaded, and its products come back in the same
//     places: four of the rotation's seven stages are products with the signs of a 16 x 16 Hadamard matrix (exact
//     products, fp32 sums), the other three additions within a lane, and no value is shuffled.
#include "akv_paged.cuh"

namespace akv {
namespace {

constexpr int kRowLanes = 4;
constexpr int kMaxThreads = 128;

struct RowsIO {
  uint16_t* ptr;
  int64_t sb, st, sh;
  int vec;  // every row 16-byte aligned
};

// Two fp32 at a time (each rounded as its own).
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

template <bool HALF>
__device__ __forceinline__ void mma_rows(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  const float z = 0.f;
  if (HALF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(z));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(z));
}

// The second operand of the rotation's products: signs (-1)^(bits that input and output share) of four dimension bits.
// Inputs: lane t has bits 3 and 4, register r bit 1, the pair's halves bit `first` (0 or 2); outputs: column g has bits
// 3 and 4 in g / 2, column parity bit 0 (first 0) or bit 1 (first 2), tile n bit 1 or bit 2.
template <bool HALF>
__device__ __forceinline__ void hadamard_operand(int lane, int first, uint32_t (&b)[2][2]) {
  const int g = lane >> 2, t = lane & 3;
  const uint32_t one = HALF ? 0x3c00u : 0x3f80u, far = (uint32_t)__popc(t & (g >> 1)) & 1u;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (uint32_t r = 0; r < 2; ++r) {
      const uint32_t tile = (uint32_t)n, parity = (uint32_t)g & 1u;
      const uint32_t low = far ^ (r & (first ? parity : tile));        // the pair's half 0
      const uint32_t high = low ^ (first ? tile : parity);             // and half 1
      b[n][r] = (one | low << 15) | (one | high << 15) << 16;
    }
}

// H (s o x) of the warp's 8 rows, x as loaded with its signs flipped: word 4 c + m is dimensions 32 c + 8 u + 2 m and
// the next, y[8 c + n] dimension 32 c + 8 u + n.  fp32 sums.
template <bool HALF>
__device__ __forceinline__ void rotate_rows(const uint32_t (&w)[16], const uint32_t (&b)[2][2], float (&y)[32]) {
  uint64_t p[16];  // p[4 c + 2 d2 + d1]: a pair of neighbouring dimensions
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int n = 0; n < 2; ++n) {  // bits 0, 1, 3, 4; the tile's lower rows are the dimensions with bit 2
      float d[4];
      mma_rows<HALF>(d, w[4 * c], w[4 * c + 2], w[4 * c + 1], w[4 * c + 3], b[n][0], b[n][1]);
      p[4 * c + n] = pair(d[0], d[1]);
      p[4 * c + 2 + n] = pair(d[2], d[3]);
    }
  const uint64_t minus = pair(-1.f, -1.f);
#pragma unroll
  for (int h = 2; h < 16; h *= 2)  // bits 2, 5, 6
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!(i & h)) {
        const uint64_t a = p[i], q = p[i | h];
        p[i] = add2(a, q);
        p[i | h] = fma2(q, minus, a);
      }
#pragma unroll
  for (int i = 0; i < 16; ++i) unpair(p[i], y[2 * i], y[2 * i + 1]);
}

template <bool HALF>
__device__ __forceinline__ float lo_half(uint32_t w) {
  return HALF ? __half2float(__ushort_as_half((unsigned short)w)) : __uint_as_float(w << 16);
}
template <bool HALF>
__device__ __forceinline__ float hi_half(uint32_t w) {
  return HALF ? __half2float(__ushort_as_half((unsigned short)(w >> 16))) : __uint_as_float(w & 0xffff0000u);
}
template <bool HALF>
__device__ __forceinline__ uint32_t pack_rows(float a, float b) {
  if (HALF) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Smaller and larger of two pairs of rows' values (a NaN is passed on).
template <bool HALF>
__device__ __forceinline__ uint32_t min_rows(uint32_t a, uint32_t b) {
  uint32_t r;
  if (HALF) asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <bool HALF>
__device__ __forceinline__ uint32_t max_rows(uint32_t a, uint32_t b) {
  uint32_t r;
  if (HALF) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float min3_nan(float a, float b, float c) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Signs of the rotation as pairs of rows' sign bits, in shared memory: word 16 u + 4 c + m is dimensions
// 32 c + 8 u + 2 m and the next.  Called by every thread of the CTA.
__device__ __forceinline__ void fill_signs(const PagedView& v, uint32_t* sign) {
  for (int i = threadIdx.x; i < 64; i += blockDim.x) {
    const int d = 32 * (i >> 2 & 3) + 8 * (i >> 4) + 2 * (i & 3);
    const uint32_t bits = (uint32_t)((d < 64 ? v.sign_bits[0] : v.sign_bits[1]) >> (d & 63)) & 3u;
    sign[i] = (bits & 1u) << 15 | (bits & 2u) << 30;
  }
  __syncthreads();
}

// A row's values (as given, packed; signs flipped where rotated) -> this lane's codes, word c: dimensions 32 c + 8 u + n
// in nibble n, and the words (scale | minimum << 16) of the row's groups.
template <int NG, bool ROT, bool HALF>
__device__ __forceinline__ void quantise(const uint32_t (&w)[16], const uint32_t (&b)[2][2], int u, uint32_t (&codes)[4], uint32_t (&word)[NG]) {
  float x[32];
  if (ROT) {
    rotate_rows<HALF>(w, b, x);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[2 * i] = lo_half<HALF>(w[i]), x[2 * i + 1] = hi_half<HALF>(w[i]);
  }
  constexpr float kUnit = ROT ? 0.125f : 1.f;  // v = x times this (exact: a power of two)
  constexpr int kEach = 32 / NG;
  float lo[NG], hi[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    if (ROT) {
      lo[g] = hi[g] = x[g * kEach];
#pragma unroll
      for (int i = 1; i + 1 < kEach; i += 2) {
        lo[g] = min3_nan(lo[g], x[g * kEach + i], x[g * kEach + i + 1]);
        hi[g] = max3_nan(hi[g], x[g * kEach + i], x[g * kEach + i + 1]);
      }
      lo[g] = min_nan(lo[g], x[g * kEach + kEach - 1]);
      hi[g] = max_nan(hi[g], x[g * kEach + kEach - 1]);
    } else {
      uint32_t a = w[g * kEach / 2], c = a;
#pragma unroll
      for (int i = 1; i < kEach / 2; ++i) {
        a = min_rows<HALF>(a, w[g * kEach / 2 + i]);
        c = max_rows<HALF>(c, w[g * kEach / 2 + i]);
      }
      lo[g] = min_nan(lo_half<HALF>(a), hi_half<HALF>(a));
      hi[g] = max_nan(lo_half<HALF>(c), hi_half<HALF>(c));
    }
  }
  // over the row's lanes; of two groups, lanes with an odd u are left with the second
  float my_lo = lo[0], my_hi = hi[0];
  if (NG == 2) {
    my_lo = u & 1 ? lo[NG - 1] : lo[0];
    my_hi = u & 1 ? hi[NG - 1] : hi[0];
  }
  my_lo = min_nan(my_lo, __shfl_xor_sync(0xffffffffu, NG == 2 && !(u & 1) ? lo[NG - 1] : lo[0], 1));
  my_hi = max_nan(my_hi, __shfl_xor_sync(0xffffffffu, NG == 2 && !(u & 1) ? hi[NG - 1] : hi[0], 1));
  my_lo = min_nan(my_lo, __shfl_xor_sync(0xffffffffu, my_lo, 2)) * kUnit;
  my_hi = max_nan(my_hi, __shfl_xor_sync(0xffffffffu, my_hi, 2)) * kUnit;
  const bool my_fine = fabsf(my_lo) <= 3.402823466e38f && fabsf(my_hi) <= 3.402823466e38f;  // no infinity, no NaN
  const __half mh = __float2half_rn(fminf(fmaxf(my_lo, -65504.f), 65504.f));
  const float my_m = __half2float(mh);
  const __half ah = __float2half_rn(fminf(__fdiv_rn(fmaxf(__fsub_rn(my_hi, my_m), 0.f), 15.f), 65504.f));
  const float my_a = __half2float(ah);
  const uint32_t my_word = my_fine ? (uint32_t)__half_as_ushort(ah) | (uint32_t)__half_as_ushort(mh) << 16 : 0x7e007e00u;
  const float my_inv = my_a > 0.f && my_fine ? __frcp_rn(my_a) : 0.f;
  // the ends of the range: between them (every step of t is monotone) no code needs clamping
  const bool inside = my_fine && __fmul_rn(__fsub_rn(my_lo, my_m), my_inv) >= -0.5f && __fmul_rn(__fsub_rn(my_hi, my_m), my_inv) < 15.5f;
  float inv[NG], m[NG];
  if (NG == 2) {
    const float o_inv = __shfl_xor_sync(0xffffffffu, my_inv, 1);
    const uint32_t o_word = __shfl_xor_sync(0xffffffffu, my_word, 1);
    inv[0] = u & 1 ? o_inv : my_inv;
    inv[NG - 1] = u & 1 ? my_inv : o_inv;
    word[0] = u & 1 ? o_word : my_word;
    word[NG - 1] = u & 1 ? my_word : o_word;
  } else {
    inv[0] = my_inv;
    word[0] = my_word;
  }
#pragma unroll
  for (int g = 0; g < NG; ++g) m[g] = __half2float(__ushort_as_half((unsigned short)(word[g] >> 16)));
  const bool clamp = !__all_sync(0xffffffffu, inside);
  const uint64_t magic = pair(12582912.f, 12582912.f), unit = pair(kUnit, kUnit);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const uint64_t inv2 = pair(inv[g], inv[g]), minus_m = pair(-m[g], -m[g]);
#pragma unroll
    for (int c = g * 4 / NG; c < (g + 1) * 4 / NG; ++c) {
      // t + 1.5 2^23 has the rounded code in its low bits; the rest sums up to a constant over the eight nibbles
      uint64_t t[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) t[n] = mul2(fma2(pair(x[8 * c + 2 * n], x[8 * c + 2 * n + 1]), unit, minus_m), inv2);
      if (clamp) {  // (a NaN becomes 0)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          float t0, t1;
          unpair(t[n], t0, t1);
          t[n] = pair(fminf(fmaxf(t0, 0.f), 15.f), fminf(fmaxf(t1, 0.f), 15.f));
        }
      }
      uint32_t sum = 0, bias = 0;
#pragma unroll
      for (int n = 3; n >= 0; --n) {
        float t0, t1;
        unpair(add2(t[n], magic), t0, t1);
        sum = (sum << 4) + __float_as_uint(t1);
        sum = (sum << 4) + __float_as_uint(t0);
        bias = (bias << 4) + 0x4B400000u;
        bias = (bias << 4) + 0x4B400000u;
      }
      codes[c] = sum - bias;
    }
  }
}

__device__ __forceinline__ void load_row(const RowsIO& R, int64_t at, int u, uint32_t (&w)[16]) {
  const uint16_t* row = R.ptr + at + 8 * u;
  if (R.vec) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint4 x = *(const uint4*)(row + 32 * c);
      w[4 * c] = x.x, w[4 * c + 1] = x.y, w[4 * c + 2] = x.z, w[4 * c + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = row[32 * (i >> 2) + 2 * (i & 3)] | (uint32_t)row[32 * (i >> 2) + 2 * (i & 3) + 1] << 16;
  }
}

// One CTA: one page of one request that gets new tokens, one head; its keys, then its values, or (sides 1) one of them.
// The row after the present one is loaded while that is worked on.  Seven CTAs an SM: 128K rotated tokens of 8 heads take
// 162 us (4.2 TB/s).
template <int NG, bool ROT, bool HALF>
__global__ void __launch_bounds__(kMaxThreads, 7) akv_paged_append_kernel(PagedView v, RowsIO K, RowsIO V, int T, const int32_t* n_new,
                                                                          int pages_each, int sides) {
  __shared__ __align__(16) uint32_t sign[64];
  launch_dependents();
  if (ROT) fill_signs(v, sign);
  wait_for_stream();
  const int part = sides == 1 ? blockIdx.x & 1 : 0, cta = sides == 1 ? blockIdx.x >> 1 : blockIdx.x;
  const int slot = cta % pages_each, bh = cta / pages_each;
  const int h = bh % v.H, b = bh / v.H;
  const int P = 1 << v.page_log;
  const int held = held_tokens(v, b);
  const int n = min(min(max(n_new ? n_new[b] : T, 0), T), (v.max_pages << v.page_log) - held);
  const int j = (held >> v.page_log) + slot;  // table position
  const int i0 = max(0, held - (j << v.page_log)), i1 = min(P, held + n - (j << v.page_log));  // places in the page
  if (i0 >= i1) return;
  const int page = page_of(v, b, j);  // (looked at once the first rows are under way)
  constexpr uint32_t kSub = 2048 + 128 * NG;
  const int u = threadIdx.x & 3, row = threadIdx.x / kRowLanes;
  const int at_once = blockDim.x / kRowLanes;  // rows: the page's, or 32
  const int turns_log = max(0, v.page_log - 5), turns = sides << turns_log;
  const int64_t to = (int64_t)(j << v.page_log) - held;  // token of the page's first place, among the new ones
  const int64_t base_k = b * K.sb + h * K.sh + to * K.st, base_v = b * V.sb + h * V.sh + to * V.st;

  auto load = [&](int turn, uint32_t (&w)[16]) {  // (a row that is not there leaves what was: nothing of it is stored)
    const int side = part + (turn >> turns_log), i = (turn & ((1 << turns_log) - 1)) * at_once + row;
    if (turn < turns && i >= i0 && i < i1) {
      if (side) load_row(V, base_v + i * V.st, u, w);
      else load_row(K, base_k + i * K.st, u, w);
    }
  };
  uint32_t signs[2][2];
  if (ROT) hadamard_operand<HALF>(threadIdx.x & 31, 0, signs);
  uint32_t next[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) next[k] = 0;
  load(0, next);
  if (page < 0 || (v.refs && v.refs[page] > 1)) return;  // (never over what another request holds)
  uint8_t* block = block_of(v, page, h);
#pragma unroll 1
  for (int turn = 0; turn < turns; ++turn) {
    uint32_t w[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) w[k] = next[k];
    load(turn + 1, next);
    const int side = part + (turn >> turns_log), i = (turn & ((1 << turns_log) - 1)) * at_once + row;
    const bool there = i >= i0 && i < i1;
    if (!__any_sync(0xffffffffu, there)) continue;
    if (ROT) {
#pragma unroll
      for (int k = 0; k < 16; ++k) w[k] ^= sign[16 * u + k];
    }
    uint32_t c[4], word[NG];
    quantise<NG, ROT, HALF>(w, signs, u, c, word);
    uint8_t* s = block + (uint32_t)(i >> 4) * kSub;
    const int i16 = i & 15;
    if (side == 0) {
      if (there) *(uint4*)(s + 64 * i16 + 16 * u) = make_uint4(c[0], c[1], c[2], c[3]);
    } else {
      // c[j]: s = j / 2, g = u + 4 (j % 2); words 2 s + u' of unit g hold the even token's half, then the odd one's
      const bool odd = i & 1, both = __shfl_xor_sync(0xffffffffu, (int)there, 4) && there;
      const uint32_t o0 = __shfl_xor_sync(0xffffffffu, odd ? c[0] : c[1], 4), o1 = __shfl_xor_sync(0xffffffffu, odd ? c[2] : c[3], 4);
      uint8_t* unit = s + 1024 + 512 * (i16 >> 3) + 16 * (4 * u + ((i16 & 7) >> 1));
      if (both) {  // the even token's lanes write unit u, the odd one's u + 4
        const uint32_t a0 = odd ? o0 : c[0], b0 = odd ? c[1] : o0, a1 = odd ? o1 : c[2], b1 = odd ? c[3] : o1;
        *(uint4*)(unit + (odd ? 256 : 0)) = make_uint4(__byte_perm(a0, b0, 0x5410), __byte_perm(a0, b0, 0x7632),
                                                       __byte_perm(a1, b1, 0x5410), __byte_perm(a1, b1, 0x7632));
      } else if (there) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint16_t* at = (uint16_t*)(unit + 256 * (k & 1) + 8 * (k >> 1)) + odd;
          at[0] = (uint16_t)c[k];
          at[2] = (uint16_t)(c[k] >> 16);
        }
      }
    }
    if (there && u == 0) {
      uint32_t* at = (uint32_t*)(s + 2048) + 2 * NG * i16 + NG * side;
#pragma unroll
      for (int g = 0; g < NG; ++g) at[g] = word[g];
    }
  }
  if (!v.bounds || part != 0) return;
  // The page's bounds: the keys once more, which the caches hold; a thread takes 16 bytes of every eighth row (128K tokens:
  // 162 us in all, 198 with 4 bytes of every other row, 140 without bounds; read first, or between keys and values, 170 to 187).
  __shared__ __align__(16) uint4 red[kMaxThreads / 32][2][16];
  const int at = threadIdx.x & 15, warp = threadIdx.x >> 5, rows = blockDim.x >> 4;
  uint4 lo, hi;
  lo.x = lo.y = lo.z = lo.w = HALF ? 0x7c007c00u : 0x7f807f80u;  // + and - infinity
  hi.x = hi.y = hi.z = hi.w = lo.x | 0x80008000u;
  auto take = [&](const uint4& a, const uint4& b) {  // (a page with a NaN has the score +infinity)
    lo.x = min_rows<HALF>(lo.x, a.x), lo.y = min_rows<HALF>(lo.y, a.y), lo.z = min_rows<HALF>(lo.z, a.z), lo.w = min_rows<HALF>(lo.w, a.w);
    hi.x = max_rows<HALF>(hi.x, b.x), hi.y = max_rows<HALF>(hi.y, b.y), hi.z = max_rows<HALF>(hi.z, b.z), hi.w = max_rows<HALF>(hi.w, b.w);
  };
  const uint16_t* x = K.ptr + base_k + 8 * at;
#pragma unroll 4
  for (int i = i0 + (threadIdx.x >> 4); i < i1; i += rows) {
    uint4 w;
    const uint16_t* y = x + i * K.st;
    if (K.vec) {
      w = *(const uint4*)y;
    } else {
      w.x = y[0] | (uint32_t)y[1] << 16, w.y = y[2] | (uint32_t)y[3] << 16;
      w.z = y[4] | (uint32_t)y[5] << 16, w.w = y[6] | (uint32_t)y[7] << 16;
    }
    take(w, w);
  }
  auto other = [&](const uint4& w) {
    return make_uint4(__shfl_xor_sync(0xffffffffu, w.x, 16), __shfl_xor_sync(0xffffffffu, w.y, 16),
                      __shfl_xor_sync(0xffffffffu, w.z, 16), __shfl_xor_sync(0xffffffffu, w.w, 16));
  };
  take(other(lo), other(hi));
  if (!(threadIdx.x & 16)) red[warp][0][at] = lo, red[warp][1][at] = hi;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  for (int w = 1; w < (int)blockDim.x >> 5; ++w) take(red[w][0][at], red[w][1][at]);
  uint4* to_b = (uint4*)(block + (uint32_t)(P >> 4) * kSub) + at;
  if (i0 != 0) take(to_b[0], to_b[16]);  // what the page held before
  to_b[0] = lo;
  to_b[16] = hi;
}

// H v^ / 16 of the warp's 8 rows from their codes: over the six bits of a group H v^ = a (H c) + 64 m at dimension 0, and
// the codes' sums are whole numbers, exact; bit 6 joins the groups.  Nibbles are taken in place as fp16 subnormals,
// c 2^-24 or (odd dimensions) c 2^-20.
template <int NG>
__device__ __forceinline__ void unrotate_codes(const uint32_t (&c)[4], const uint32_t (&b)[2][2], const float (&scale)[NG],
                                               const float (&low)[NG], int u, float (&y)[32]) {
  uint64_t p[16];  // p[4 c + 2 d2 + d0]: the pair of bit 1
  const uint64_t up = pair(0.0625f, 0.0625f), down = pair(-0.0625f, -0.0625f), minus = pair(-1.f, -1.f);
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int n = 0; n < 2; ++n) {  // bits 1, 2, 3, 4; the tile's lower rows are the odd dimensions; then bit 0
      const uint32_t x = c[k], z = c[k] >> 8;
      float d[4];
      mma_rows<true>(d, x & 0x000f000fu, x & 0x00f000f0u, z & 0x000f000fu, z & 0x00f000f0u, b[n][0], b[n][1]);
      const uint64_t even = pair(d[0], d[1]), odd = pair(d[2], d[3]);
      p[4 * k + 2 * n] = fma2(odd, up, even);
      p[4 * k + 2 * n + 1] = fma2(odd, down, even);
    }
#pragma unroll
  for (int i = 0; i < 16; ++i)  // bit 5
    if (!(i & 4)) {
      const uint64_t a = p[i], q = p[i | 4];
      p[i] = add2(a, q);
      p[i | 4] = fma2(q, minus, a);
    }
  const float a0 = scale[0] * 1048576.f, a1 = scale[NG - 1] * 1048576.f;  // 2^24 / 16
  const uint64_t s0 = pair(a0, a0), s1 = pair(a1, a1);
  const float m0 = u == 0 ? low[0] * 4.f : 0.f, m1 = u == 0 ? low[NG - 1] * 4.f : 0.f;  // 64 / 16
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // bit 6
    uint64_t q = mul2(p[i + 8], s1), r = q;
    if (i == 0) {  // dimension 0 of each group
      q = fma2(p[8], s1, pair(m0 + m1, 0.f));
      r = fma2(p[8], s1, pair(m1 - m0, 0.f));
    }
    const uint64_t a = fma2(p[i], s0, q), d = fma2(r, minus, mul2(p[i], s0));
    const int c0 = i >> 2, d2 = i >> 1 & 1, d0 = i & 1, at = 8 * c0 + 4 * d2 + d0;
    unpair(a, y[at], y[at + 2]);
    unpair(d, y[at + 16], y[at + 18]);
  }
}

constexpr int kReadTurns = 8;  // rows a thread reads back at most (128K rotated tokens of 8 heads: 140 us with four, 132
                               // with eight; 120 us, 5.7 TB/s, since seven CTAs share an SM)

template <int NG, bool ROT, bool HALF>
__global__ void __launch_bounds__(kMaxThreads, 7) akv_paged_read_kernel(PagedView v, const int32_t* start, RowsIO K, RowsIO V, int T,
                                                                        int chunks, int turns) {
  constexpr int kRowsAtOnce = kMaxThreads / kRowLanes;
  const int side = blockIdx.x & 1;
  const int chunk = (blockIdx.x >> 1) % chunks;
  const int bh = (blockIdx.x >> 1) / chunks;
  const int h = bh % v.H, b = bh / v.H;
  const int u = threadIdx.x & 3;
  __shared__ __align__(16) uint32_t sign[64];
  launch_dependents();
  if (ROT) fill_signs(v, sign);
  wait_for_stream();
  const int64_t first = start ? (int64_t)start[b] : 0;
  const int held = held_tokens(v, b), P = 1 << v.page_log;
  const RowsIO& R = side ? V : K;
  auto token = [&](int turn) { return (chunk * turns + turn) * kRowsAtOnce + (int)threadIdx.x / kRowLanes; };
  auto find = [&](int turn) {
    const int t = token(turn);
    const int64_t pos = first + t;
    return turn < turns && t < T && pos >= 0 && pos < held ? page_of(v, b, (int)(pos >> v.page_log)) : -1;
  };
  struct Held {
    uint4 y, z;  // a key's codes; the two units that hold a value's
    uint32_t words[NG];
  };
  auto fetch = [&](int turn, int page) {
    Held r;
    r.y = r.z = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int g = 0; g < NG; ++g) r.words[g] = 0;
    if (page < 0) return r;
    const int i = (int)((first + token(turn)) & (P - 1)), i16 = i & 15;
    const uint8_t* s = block_of(v, page, h) + (uint32_t)(i >> 4) * (2048 + 128 * NG);
    const uint32_t* at = (const uint32_t*)(s + 2048) + 2 * NG * i16 + NG * side;
#pragma unroll
    for (int g = 0; g < NG; ++g) r.words[g] = at[g];
    if (side == 0) {
      r.y = *(const uint4*)(s + 64 * i16 + 16 * u);
    } else {
      const uint8_t* unit = s + 1024 + 512 * (i16 >> 3) + 16 * (4 * u + ((i16 & 7) >> 1));
      r.y = *(const uint4*)unit;
      r.z = *(const uint4*)(unit + 256);
    }
    return r;
  };
  uint32_t signs[2][2];
  if (ROT) hadamard_operand<true>(threadIdx.x & 31, 2, signs);
  // the page of the row after the next and the codes of the next are under way while a row is worked on
  int page = find(0), page1 = find(1);
  Held ahead = fetch(0, page);
#pragma unroll 1
  for (int turn = 0; turn < turns; ++turn) {
    const Held r = ahead;
    const int t = token(turn);
    const bool there = page >= 0, odd = (first + t) & 1;
    ahead = fetch(turn + 1, page1);
    page = page1;
    page1 = find(turn + 2);
    float x[32];
    {
      uint32_t c[4] = {r.y.x, r.y.y, r.y.z, r.y.w};
      const uint32_t* words = r.words;
      float scale[NG], low[NG];
      if (side) {
        const uint32_t pick = odd ? 0x7632 : 0x5410;
        c[0] = __byte_perm(r.y.x, r.y.y, pick);
        c[1] = __byte_perm(r.z.x, r.z.y, pick);
        c[2] = __byte_perm(r.y.z, r.y.w, pick);
        c[3] = __byte_perm(r.z.z, r.z.w, pick);
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        scale[g] = __half2float(__ushort_as_half((unsigned short)words[g]));
        low[g] = __half2float(__ushort_as_half((unsigned short)(words[g] >> 16)));
      }
      if (ROT) {
        unrotate_codes<NG>(c, signs, scale, low, u, x);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float a24 = scale[k * NG / 4] * 16777216.f, a20 = scale[k * NG / 4] * 1048576.f, m = low[k * NG / 4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {  // nibbles q and q + 4, in place, as fp16 subnormals: c 2^-24, odd ones c 2^-20
            const uint32_t y = (q & 2 ? c[k] >> 8 : c[k]) & (q & 1 ? 0x00f000f0u : 0x000f000fu);
            const __half2 hh = *reinterpret_cast<const __half2*>(&y);
            x[8 * k + q] = fmaf(__low2float(hh), q & 1 ? a20 : a24, m);
            x[8 * k + q + 4] = fmaf(__high2float(hh), q & 1 ? a20 : a24, m);
          }
        }
      }
    }
    uint32_t w[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) w[k] = pack_rows<HALF>(x[2 * k], x[2 * k + 1]);
    if (ROT && there) {  // (a row that is not there is +0)
#pragma unroll
      for (int k = 0; k < 16; ++k) w[k] ^= sign[16 * u + k];
    }
    if (t >= T) continue;
    uint16_t* row = R.ptr + b * R.sb + t * R.st + h * R.sh + 8 * u;
    if (R.vec) {
#pragma unroll
      for (int k = 0; k < 4; ++k) *(uint4*)(row + 32 * k) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        row[32 * (k >> 2) + 2 * (k & 3)] = (uint16_t)w[k];
        row[32 * (k >> 2) + 2 * (k & 3) + 1] = (uint16_t)(w[k] >> 16);
      }
    }
  }
}

template <bool HALF>
auto append_kernel(const PagedView& v) {
  return v.rotate ? (v.ng == 2 ? akv_paged_append_kernel<2, true, HALF> : akv_paged_append_kernel<1, true, HALF>)
                  : (v.ng == 2 ? akv_paged_append_kernel<2, false, HALF> : akv_paged_append_kernel<1, false, HALF>);
}
template <bool HALF>
auto read_kernel(const PagedView& v) {
  return v.rotate ? (v.ng == 2 ? akv_paged_read_kernel<2, true, HALF> : akv_paged_read_kernel<1, true, HALF>)
                  : (v.ng == 2 ? akv_paged_read_kernel<2, false, HALF> : akv_paged_read_kernel<1, false, HALF>);
}

RowsIO rows_io(const akv_rows& r) {
  RowsIO io{(uint16_t*)r.ptr, r.stride_b, r.stride_t, r.stride_h, 0};
  io.vec = ((uintptr_t)r.ptr % 16) == 0 && (r.stride_b | r.stride_t | r.stride_h) % 8 == 0;
  return io;
}

}  // namespace

int launch_paged_append(const PagedView& v, const akv_rows& K, const akv_rows& V, int32_t T, const int32_t* n_new, void* stream) {
  const int P = 1 << v.page_log;
  int64_t each = ((int64_t)T + P - 2) / P + 1;  // pages that T tokens can touch
  if (each > v.max_pages) each = v.max_pages;
  // keys and values by one CTA where there are CTAs enough for the GPU (four an SM) all the same
  const int sides = each * v.H * v.rows >= 4 * 152 ? 2 : 1;
  const int64_t grid = (sides == 1 ? 2 : 1) * each * v.H * v.rows;
  if (grid > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  const int threads = P * kRowLanes < kMaxThreads ? P * kRowLanes : kMaxThreads;
  auto kernel = v.half ? append_kernel<true>(v) : append_kernel<false>(v);
  return launch_after(kernel, dim3((unsigned)grid), threads, 0, stream, v, rows_io(K), rows_io(V), T, n_new, (int)each, sides);
}

int launch_paged_read(const PagedView& v, const int32_t* start, const akv_rows& K, const akv_rows& V, int32_t T, void* stream) {
  const int64_t chunks = ((int64_t)T + kMaxThreads / kRowLanes - 1) / (kMaxThreads / kRowLanes);
  // more rows a thread only where the grid stays above a few waves: then a row's page and codes are under way while
  // others are worked on, else the rows of a small call would wait for one another
  const int turns = chunks * v.H * v.rows >= 8192 ? kReadTurns : 1;
  const int64_t each = (chunks + turns - 1) / turns;
  const int64_t grid = 2 * each * v.H * v.rows;
  if (grid > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  auto kernel = v.half ? read_kernel<true>(v) : read_kernel<false>(v);
  return launch_after(kernel, dim3((unsigned)grid), kMaxThreads, 0, stream, v, start, rows_io(K), rows_io(V), T, (int)each, turns);
}

}  // namespace akv
