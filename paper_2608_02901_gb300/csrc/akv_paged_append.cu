// Paged 4-bit cache: quantising new tokens into their pages, and reading rows back.
//
// Both move a row between 256 dense bytes and 64 + 4 NG held ones.  Four lanes share a row: lane u of them holds
// dimensions 32 c + 8 u + n (c < 4, n < 8), so that
//   - the dense side is four 16-byte accesses a lane, 64 contiguous bytes a row each time;
//   - the key codes of a lane are the 16 contiguous bytes of its row's words 4 u .. 4 u + 3, the value codes (after an
//     exchange with the neighbouring token's lanes, whose halves share the words) one 16-byte unit;
//   - the rotation needs shuffles for two of its seven stages only (8 and 16), the minimum and maximum of a group two.
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

// The codec's butterfly of a row over four lanes: x[8 c + n] is dimension 32 c + 8 u + n.
__device__ __forceinline__ void wht_4x32(float (&x)[32], int u) {
  const uint64_t minus = pair(-1.f, -1.f);
#pragma unroll
  for (int i = 0; i < 32; i += 2) {  // stage 1
    const float a = x[i], b = x[i + 1];
    x[i] = __fadd_rn(a, b);
    x[i + 1] = __fsub_rn(a, b);
  }
  uint64_t p[16];  // pairs of neighbouring dimensions
#pragma unroll
  for (int i = 0; i < 16; ++i) p[i] = pair(x[2 * i], x[2 * i + 1]);
  auto stage = [&](int h) {  // h: distance in pairs
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!(i & h)) {
        const uint64_t a = p[i], b = p[i | h];
        p[i] = add2(a, b);
        p[i | h] = fma2(b, minus, a);
      }
  };
  stage(1);  // 2
  stage(2);  // 4
#pragma unroll
  for (int h = 1; h < 4; h *= 2) {  // 8, 16: the lane with the bit holds b of a + b, a - b
    const uint64_t sign = u & h ? minus : pair(1.f, 1.f);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float a, b;
      unpair(p[i], a, b);
      const uint64_t o = pair(__shfl_xor_sync(0xffffffffu, a, h), __shfl_xor_sync(0xffffffffu, b, h));
      p[i] = fma2(p[i], sign, o);
    }
  }
  stage(4);  // 32
  stage(8);  // 64
#pragma unroll
  for (int i = 0; i < 16; ++i) unpair(p[i], x[2 * i], x[2 * i + 1]);
}

__device__ __forceinline__ float lo_half(uint32_t w, int half) {
  return half ? __half2float(__ushort_as_half((unsigned short)w)) : __uint_as_float(w << 16);
}
__device__ __forceinline__ float hi_half(uint32_t w, int half) {
  return half ? __half2float(__ushort_as_half((unsigned short)(w >> 16))) : __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack_rows(float a, float b, int half) {
  if (half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Smaller and larger of two pairs of rows' values (a NaN is left out).
__device__ __forceinline__ uint32_t min_rows(uint32_t a, uint32_t b, int half) {
  uint32_t r;
  if (half) asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_rows(uint32_t a, uint32_t b, int half) {
  uint32_t r;
  if (half) asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Signs of the rotation as pairs of rows' sign bits: word 4 c + m of lane u is dimensions 32 c + 8 u + 2 m, + 1.
__device__ __forceinline__ void sign_words(const PagedView& v, int u, uint32_t (&w)[16]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t bits = (uint32_t)(v.sign_bits[c >> 1] >> (32 * (c & 1) + 8 * u));
#pragma unroll
    for (int m = 0; m < 4; ++m) w[4 * c + m] = (bits >> (2 * m) & 1u) << 15 | (bits >> (2 * m + 1) & 1u) << 31;
  }
}

// A row's values (packed as stored, signs flipped) -> this lane's codes, word c: dimensions 32 c + 8 u + n in nibble n,
// and the words (scale | minimum << 16) of the row's groups.
template <int NG, bool ROT>
__device__ __forceinline__ void quantise(const uint32_t (&w)[16], int half, int u, uint32_t (&codes)[4], uint32_t (&word)[NG]) {
  float x[32];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[2 * i] = lo_half(w[i], half), x[2 * i + 1] = hi_half(w[i], half);
  if (ROT) {
    wht_4x32(x, u);
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] *= 0.125f;
  }
  constexpr int kEach = 32 / NG;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    float lo = x[g * kEach], hi = lo;
#pragma unroll
    for (int i = 1; i < kEach; ++i) {
      lo = min_nan(lo, x[g * kEach + i]);
      hi = max_nan(hi, x[g * kEach + i]);
    }
#pragma unroll
    for (int h = 1; h < kRowLanes; h *= 2) {
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, h));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, h));
    }
    const bool fine = fabsf(lo) <= 3.402823466e38f && fabsf(hi) <= 3.402823466e38f;  // no infinity, no NaN
    const __half mh = __float2half_rn(fminf(fmaxf(lo, -65504.f), 65504.f));
    const float m = __half2float(mh);
    const __half ah = __float2half_rn(fminf(__fdiv_rn(fmaxf(__fsub_rn(hi, m), 0.f), 15.f), 65504.f));
    const float a = __half2float(ah);
    word[g] = fine ? (uint32_t)__half_as_ushort(ah) | (uint32_t)__half_as_ushort(mh) << 16 : 0x7e007e00u;
    const float inv = a > 0.f ? __frcp_rn(a) : 0.f;
    const uint64_t inv2 = pair(inv, inv), minus_m = pair(-m, -m), magic = pair(12582912.f, 12582912.f);
#pragma unroll
    for (int c = g * 4 / NG; c < (g + 1) * 4 / NG; ++c) {
      // c + 1.5 2^23 has the rounded code in its low bits; the exponents' sum over the eight nibbles is a constant
      uint32_t sum = 0;
#pragma unroll
      for (int n = 6; n >= 0; n -= 2) {
        float t0, t1;
        unpair(mul2(add2(pair(x[8 * c + n], x[8 * c + n + 1]), minus_m), inv2), t0, t1);
        t0 = fminf(fmaxf(t0, 0.f), 15.f);
        t1 = fminf(fmaxf(t1, 0.f), 15.f);
        unpair(add2(pair(t0, t1), magic), t0, t1);
        sum = (sum << 4) + __float_as_uint(t1);
        sum = (sum << 4) + __float_as_uint(t0);
      }
      uint32_t bias = 0;
#pragma unroll
      for (int n = 0; n < 8; ++n) bias = (bias << 4) + 0x4B400000u;
      codes[c] = fine ? sum - bias : 0u;
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

// One step over the rows of a warp (lanes 2 kWords apart): a lane gives away one half of its 2 kWords words and joins the
// other half with its partner's.
template <int kWords>
__device__ __forceinline__ void join_rows(uint32_t (&lo)[16], uint32_t (&hi)[16], int& first, int lane, int half) {
  const bool up = lane & 2 * kWords;
#pragma unroll
  for (int k = 0; k < kWords; ++k) {
    const uint32_t ol = __shfl_xor_sync(0xffffffffu, up ? lo[k] : lo[k + kWords], 2 * kWords);
    const uint32_t oh = __shfl_xor_sync(0xffffffffu, up ? hi[k] : hi[k + kWords], 2 * kWords);
    lo[k] = min_rows(up ? lo[k + kWords] : lo[k], ol, half);
    hi[k] = max_rows(up ? hi[k + kWords] : hi[k], oh, half);
  }
  first += up ? kWords : 0;
}

// One CTA: the keys or the values of one page of one request that gets new tokens, one head.
template <int NG, bool ROT>
__global__ void __launch_bounds__(kMaxThreads, 4) akv_paged_append_kernel(PagedView v, RowsIO K, RowsIO V, int T, const int32_t* n_new,
                                                                          int pages_each) {
  const int side = blockIdx.x & 1;
  const int slot = (blockIdx.x >> 1) % pages_each;
  const int bh = (blockIdx.x >> 1) / pages_each;
  const int h = bh % v.H, b = bh / v.H;
  const int P = 1 << v.page_log;
  const int held = held_tokens(v, b);
  const int n = min(min(max(n_new ? n_new[b] : T, 0), T), (v.max_pages << v.page_log) - held);
  const int j = (held >> v.page_log) + slot;  // table position
  const int i0 = max(0, held - (j << v.page_log)), i1 = min(P, held + n - (j << v.page_log));  // places in the page
  if (i0 >= i1) return;
  const int page = page_of(v, b, j);
  if (page < 0) return;
  uint8_t* block = block_of(v, page, h);
  constexpr uint32_t kSub = 2048 + 128 * NG;
  const RowsIO& R = side ? V : K;
  const int lane = threadIdx.x & 31, u = lane & 3;
  const int rows_at_once = blockDim.x / kRowLanes;
  const int64_t base = b * R.sb + h * R.sh + ((int64_t)(j << v.page_log) - held) * R.st;
  const bool bounds = v.bounds && side == 0;
  const uint32_t none_lo = v.half ? 0x7c007c00u : 0x7f807f80u, none_hi = none_lo | 0x80008000u;  // + and - infinity
  uint32_t lo[16], hi[16], sign[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) lo[i] = none_lo, hi[i] = none_hi;
  if (ROT) sign_words(v, u, sign);

  for (int i_at = 0; i_at < P; i_at += rows_at_once) {
    const int i = i_at + threadIdx.x / kRowLanes;
    const bool there = i >= i0 && i < i1;
    if (!__any_sync(0xffffffffu, there)) continue;
    uint32_t w[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) w[k] = 0;
    if (there) {
      load_row(R, base + i * R.st, u, w);
      if (bounds) {
#pragma unroll
        for (int k = 0; k < 16; ++k) lo[k] = min_rows(lo[k], w[k], v.half), hi[k] = max_rows(hi[k], w[k], v.half);
      }
    }
    if (ROT) {
#pragma unroll
      for (int k = 0; k < 16; ++k) w[k] ^= sign[k];
    }
    uint32_t c[4], word[NG];
    quantise<NG, ROT>(w, v.half, u, c, word);
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
  if (!bounds) return;
  // over the 8 rows of a warp, after which a lane has two words (of the smallest, and of the largest) left; then over
  // the warps
  int first = 0;
  join_rows<8>(lo, hi, first, lane, v.half);
  join_rows<4>(lo, hi, first, lane, v.half);
  join_rows<2>(lo, hi, first, lane, v.half);
  __shared__ uint32_t red[kMaxThreads / 32][2][64];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = first + k, at = 16 * (i >> 2) + 4 * u + (i & 3);  // dimensions 32 c + 8 u + 2 m as pair 16 c + 4 u + m
    red[threadIdx.x >> 5][0][at] = lo[k];
    red[threadIdx.x >> 5][1][at] = hi[k];
  }
  __syncthreads();
  for (int k = threadIdx.x; k < 128; k += blockDim.x) {
    const int most = k >> 6, at = k & 63;
    uint32_t x = red[0][most][at];
    for (unsigned w = 1; w < blockDim.x / 32; ++w) x = most ? max_rows(x, red[w][1][at], v.half) : min_rows(x, red[w][0][at], v.half);
    uint32_t* to = (uint32_t*)(block + (uint32_t)(P >> 4) * kSub) + k;
    if (i0 != 0) x = most ? max_rows(x, *to, v.half) : min_rows(x, *to, v.half);  // what the page held before
    *to = x;
  }
}

template <int NG, bool ROT>
__global__ void __launch_bounds__(kMaxThreads, 4) akv_paged_read_kernel(PagedView v, const int32_t* start, RowsIO K, RowsIO V, int T,
                                                                        int chunks) {
  constexpr int kRowsAtOnce = kMaxThreads / kRowLanes;
  const int side = blockIdx.x & 1;
  const int chunk = (blockIdx.x >> 1) % chunks;
  const int bh = (blockIdx.x >> 1) / chunks;
  const int h = bh % v.H, b = bh / v.H;
  const int u = threadIdx.x & 3, t = chunk * kRowsAtOnce + threadIdx.x / kRowLanes;
  const int64_t pos = (start ? (int64_t)start[b] : 0) + t;
  const int P = 1 << v.page_log;
  int page = -1;
  if (t < T && pos >= 0 && pos < held_tokens(v, b)) page = page_of(v, b, (int)(pos >> v.page_log));
  const int i = (int)(pos & (P - 1)), i16 = i & 15;
  float x[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) x[e] = 0.f;
  if (page >= 0) {
    const uint8_t* s = block_of(v, page, h) + (uint32_t)(i >> 4) * (2048 + 128 * NG);
    uint32_t c[4];
    if (side == 0) {
      const uint4 k = *(const uint4*)(s + 64 * i16 + 16 * u);
      c[0] = k.x, c[1] = k.y, c[2] = k.z, c[3] = k.w;
    } else {
      const uint8_t* unit = s + 1024 + 512 * (i16 >> 3) + 16 * (4 * u + ((i16 & 7) >> 1));
      const uint4 y = *(const uint4*)unit, z = *(const uint4*)(unit + 256);
      const uint32_t pick = i & 1 ? 0x7632 : 0x5410;
      c[0] = __byte_perm(y.x, y.y, pick);
      c[1] = __byte_perm(z.x, z.y, pick);
      c[2] = __byte_perm(y.z, y.w, pick);
      c[3] = __byte_perm(z.z, z.w, pick);
    }
    const uint32_t* words = (const uint32_t*)(s + 2048) + 2 * NG * i16 + NG * side;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t w = words[g];
      const float a = __half2float(__ushort_as_half((unsigned short)w)), m = __half2float(__ushort_as_half((unsigned short)(w >> 16)));
      const float a24 = a * 16777216.f, a20 = a * 1048576.f;
#pragma unroll
      for (int k = g * 4 / NG; k < (g + 1) * 4 / NG; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // nibbles q and q + 4, in place, as fp16 subnormals: c 2^-24, odd ones c 2^-20
          const uint32_t y = (q & 2 ? c[k] >> 8 : c[k]) & (q & 1 ? 0x00f000f0u : 0x000f000fu);
          const __half2 hh = *reinterpret_cast<const __half2*>(&y);
          x[8 * k + q] = fmaf(__low2float(hh), q & 1 ? a20 : a24, m);
          x[8 * k + q + 4] = fmaf(__high2float(hh), q & 1 ? a20 : a24, m);
        }
    }
  }
  uint32_t w[16];
  if (ROT) {
    wht_4x32(x, u);
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] *= 0.0625f;
  }
#pragma unroll
  for (int k = 0; k < 16; ++k) w[k] = pack_rows(x[2 * k], x[2 * k + 1], v.half);
  if (ROT) {
    uint32_t sign[16];
    sign_words(v, u, sign);
#pragma unroll
    for (int k = 0; k < 16; ++k) w[k] ^= sign[k];
    if (page < 0)
#pragma unroll
      for (int k = 0; k < 16; ++k) w[k] = 0;  // (no negative zeros)
  }
  if (t >= T) return;
  const RowsIO& R = side ? V : K;
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
  const int64_t grid = 2 * each * v.H * v.rows;
  if (grid > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  const int threads = P * kRowLanes < kMaxThreads ? P * kRowLanes : kMaxThreads;
  auto* kernel = v.rotate ? (v.ng == 2 ? akv_paged_append_kernel<2, true> : akv_paged_append_kernel<1, true>)
                          : (v.ng == 2 ? akv_paged_append_kernel<2, false> : akv_paged_append_kernel<1, false>);
  kernel<<<(unsigned)grid, threads, 0, (cudaStream_t)stream>>>(v, rows_io(K), rows_io(V), T, n_new, (int)each);
  return (int)cudaGetLastError();
}

int launch_paged_read(const PagedView& v, const int32_t* start, const akv_rows& K, const akv_rows& V, int32_t T, void* stream) {
  const int64_t each = ((int64_t)T + kMaxThreads / kRowLanes - 1) / (kMaxThreads / kRowLanes);
  const int64_t grid = 2 * each * v.H * v.rows;
  if (grid > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  auto* kernel = v.rotate ? (v.ng == 2 ? akv_paged_read_kernel<2, true> : akv_paged_read_kernel<1, true>)
                          : (v.ng == 2 ? akv_paged_read_kernel<2, false> : akv_paged_read_kernel<1, false>);
  kernel<<<(unsigned)grid, kMaxThreads, 0, (cudaStream_t)stream>>>(v, start, rows_io(K), rows_io(V), T, (int)each);
  return (int)cudaGetLastError();
}

}  // namespace akv
