// Paged 4-bit cache: quantising new tokens into their pages, and reading rows back.
//
// Both move a row between 256 dense bytes and 64 + 4 NG held ones and do a few operations per value, so the bytes
// bound them.  Eight lanes share a row, 16 dimensions each: the dense side is two 16-byte accesses a lane, the minimum
// and maximum of a group two or three shuffles, the rotation's last three stages 16 shuffles each (four lanes with 32
// dimensions would need fewer, and twice the registers).
#include "akv_paged.cuh"

namespace akv {
namespace {

constexpr int kRowLanes = 8;
constexpr int kThreads = 256;
constexpr int kRowsAtOnce = kThreads / kRowLanes;

struct RowsIO {
  uint16_t* ptr;
  int64_t sb, st, sh;
  int vec;  // every row 16-byte aligned
};

__device__ __forceinline__ void load_row16(const uint16_t* row, int vec, int half, float (&x)[16]) {
  if (vec) {
    const uint4 a = ((const uint4*)row)[0], b = ((const uint4*)row)[1];
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = row_to_float((uint16_t)w[i], half);
      x[2 * i + 1] = row_to_float((uint16_t)(w[i] >> 16), half);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = row_to_float(row[i], half);
  }
}

// Codes (a nibble each, 16 dimensions of this lane) and the lane's group word (scale | minimum << 16).
__device__ __forceinline__ void quantise(const PagedView& v, float (&x)[16], int u, uint32_t (&codes)[2], uint32_t& word) {
  if (v.rotate) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = __uint_as_float(__float_as_uint(x[e]) ^ sign_flip(v, 16 * u + e));
    wht_8x16(x, u);
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= 0.125f;
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) {
    lo = min_nan(lo, x[e]);
    hi = max_nan(hi, x[e]);
  }
  for (int h = 1; h < kRowLanes / v.ng; h *= 2) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, h));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, h));
  }
  const bool fine = fabsf(lo) <= 3.402823466e38f && fabsf(hi) <= 3.402823466e38f;  // no infinity, no NaN
  const __half mh = __float2half_rn(fminf(fmaxf(lo, -65504.f), 65504.f));
  const float m = __half2float(mh);
  const __half ah = __float2half_rn(fminf(__fdiv_rn(fmaxf(__fsub_rn(hi, m), 0.f), 15.f), 65504.f));
  const float a = __half2float(ah);
  const float inv = a > 0.f && fine ? __frcp_rn(a) : 0.f;
  codes[0] = codes[1] = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float t = __fmul_rn(__fsub_rn(x[e], m), inv);
    const int c = fine ? min(max(__float2int_rn(t), 0), 15) : 0;
    codes[e >> 3] |= (uint32_t)c << 4 * (e & 7);
  }
  word = fine ? (uint32_t)__half_as_ushort(ah) | (uint32_t)__half_as_ushort(mh) << 16 : 0x7e007e00u;
}

// One CTA: one page of one request that gets new tokens, one head.
__global__ void __launch_bounds__(kThreads) akv_paged_append_kernel(PagedView v, RowsIO K, RowsIO V, int T, const int32_t* n_new,
                                                                    int pages_each) {
  const int slot = blockIdx.x % pages_each;
  const int h = blockIdx.x / pages_each % v.H;
  const int b = blockIdx.x / pages_each / v.H;
  const int P = 1 << v.page_log;
  const int held = held_tokens(v, b);
  const int n = min(min(max(n_new ? n_new[b] : T, 0), T), (v.max_pages << v.page_log) - held);
  const int j = (held >> v.page_log) + slot;  // table position
  const int t0 = max(0, (j << v.page_log) - held), t1 = min(n, ((j + 1) << v.page_log) - held);
  if (t0 >= t1) return;
  const int page = page_of(v, b, j);
  if (page < 0) return;
  uint8_t* block = block_of(v, page, h);
  const int u = threadIdx.x % kRowLanes, r = threadIdx.x / kRowLanes;
  const uint32_t sub = sub_bytes(v.ng);

  float lo[16], hi[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) lo[e] = __int_as_float(0x7f800000), hi[e] = __int_as_float(0xff800000);
  for (int t = t0; t < t1; t += kRowsAtOnce) {
    const bool there = t + r < t1;  // (whole warps stay for the shuffles)
    const int tt = there ? t + r : t1 - 1;
    const int i = held + tt & P - 1;  // place in the page
    uint8_t* s = block + (uint32_t)(i >> 4) * sub;
    const int i16 = i & 15;
    float x[16];
    uint32_t c[2], word;
    load_row16(K.ptr + b * K.sb + tt * K.st + h * K.sh + 16 * u, K.vec, v.half, x);
#pragma unroll
    for (int e = 0; e < 16; ++e) lo[e] = fminf(lo[e], x[e]), hi[e] = fmaxf(hi[e], x[e]);
    quantise(v, x, u, c, word);
    if (there) {
#pragma unroll
      for (int k = 0; k < 2; ++k)  // dimensions 16 u + 8 k ..: j = u / 2, t = 2 (u % 2) + k
        *(uint32_t*)(s + 64 * i16 + 4 * (4 * (2 * (u & 1) + k) + (u >> 1))) = c[k];
      if (u % (kRowLanes / v.ng) == 0) *(uint32_t*)(s + 2048 + 4 * (2 * v.ng * i16 + u / (kRowLanes / v.ng))) = word;
    }
    load_row16(V.ptr + b * V.sb + tt * V.st + h * V.sh + 16 * u, V.vec, v.half, x);
    quantise(v, x, u, c, word);
    if (there) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // s = u / 4, g = 2 (u % 4) + k
        const int at = 1024 + value_place(i16, u >> 2, 2 * (u & 3) + k, 0);
        *(uint16_t*)(s + at) = (uint16_t)c[k];
        *(uint16_t*)(s + at + 4) = (uint16_t)(c[k] >> 16);
      }
      if (u % (kRowLanes / v.ng) == 0) *(uint32_t*)(s + 2048 + 4 * (2 * v.ng * i16 + v.ng + u / (kRowLanes / v.ng))) = word;
    }
  }
  if (!v.bounds) return;
  __shared__ float red[2][kRowsAtOnce][kD];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    red[0][r][16 * u + e] = lo[e];
    red[1][r][16 * u + e] = hi[e];
  }
  __syncthreads();
  {  // thread d of side 0 or 1: the column over the rows, with what the page held before
    const int side = threadIdx.x / kD, d = threadIdx.x % kD;
    float x = red[side][0][d];
    for (int k = 1; k < kRowsAtOnce; ++k) x = side ? fmaxf(x, red[1][k][d]) : fminf(x, red[0][k][d]);
    uint16_t* at = (uint16_t*)(block + (uint32_t)(P >> 4) * sub) + side * kD + d;
    if ((held + t0 & P - 1) != 0) {
      const float was = row_to_float(*at, v.half);
      x = side ? fmaxf(x, was) : fminf(x, was);
    }
    *at = float_to_row(x, v.half);
  }
}

__global__ void __launch_bounds__(kThreads) akv_paged_read_kernel(PagedView v, const int32_t* start, RowsIO K, RowsIO V, int T,
                                                                  int chunks) {
  const int chunk = blockIdx.x % chunks;
  const int h = blockIdx.x / chunks % v.H;
  const int b = blockIdx.x / chunks / v.H;
  const int u = threadIdx.x % kRowLanes, t = chunk * kRowsAtOnce + threadIdx.x / kRowLanes;
  const int64_t pos = (start ? (int64_t)start[b] : 0) + t;
  const int P = 1 << v.page_log;
  int page = -1;
  if (t < T && pos >= 0 && pos < held_tokens(v, b)) page = page_of(v, b, (int)(pos >> v.page_log));
  const int i = (int)(pos & P - 1), i16 = i & 15;
  const uint8_t* s = page < 0 ? nullptr : block_of(v, page, h) + (uint32_t)(i >> 4) * sub_bytes(v.ng);
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
    if (s) {
      uint32_t c[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (side == 0) {
          c[k] = *(const uint32_t*)(s + 64 * i16 + 4 * (4 * (2 * (u & 1) + k) + (u >> 1)));
        } else {
          const int at = 1024 + value_place(i16, u >> 2, 2 * (u & 3) + k, 0);
          c[k] = *(const uint16_t*)(s + at) | (uint32_t)*(const uint16_t*)(s + at + 4) << 16;
        }
      }
      const uint32_t w = *(const uint32_t*)(s + 2048 + 4 * (2 * v.ng * i16 + side * v.ng + u / (kRowLanes / v.ng)));
      const float a = row_to_float((uint16_t)w, 1), m = row_to_float((uint16_t)(w >> 16), 1);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = fmaf((float)(c[e >> 3] >> 4 * (e & 7) & 15), a, m);
    }
    if (v.rotate) {
      wht_8x16(x, u);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = __uint_as_float(__float_as_uint(x[e] * 0.0625f) ^ sign_flip(v, 16 * u + e));
    }
    if (t < T) {
      const RowsIO& R = side ? V : K;
      uint16_t* row = R.ptr + b * R.sb + t * R.st + h * R.sh + 16 * u;
      if (R.vec) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = float_to_row(x[2 * e], v.half) | (uint32_t)float_to_row(x[2 * e + 1], v.half) << 16;
        ((uint4*)row)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        ((uint4*)row)[1] = make_uint4(w[4], w[5], w[6], w[7]);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) row[e] = float_to_row(x[e], v.half);
      }
    }
  }
}

RowsIO rows_io(const akv_rows& r) {
  RowsIO io{(uint16_t*)r.ptr, r.stride_b, r.stride_t, r.stride_h, 0};
  io.vec = ((uintptr_t)r.ptr % 16) == 0 && (r.stride_b | r.stride_t | r.stride_h) % 8 == 0;
  return io;
}

// CTAs of a launch over rows x heads x each, or an error where they are too many.
int64_t grid_of(const PagedView& v, int64_t each) { return each * v.H * v.rows; }

}  // namespace

int launch_paged_append(const PagedView& v, const akv_rows& K, const akv_rows& V, int32_t T, const int32_t* n_new, void* stream) {
  const int P = 1 << v.page_log;
  int64_t each = ((int64_t)T + P - 2) / P + 1;  // pages that T tokens can touch
  if (each > v.max_pages) each = v.max_pages;
  const int64_t grid = grid_of(v, each);
  if (grid > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  akv_paged_append_kernel<<<(unsigned)grid, kThreads, 0, (cudaStream_t)stream>>>(v, rows_io(K), rows_io(V), T, n_new, (int)each);
  return (int)cudaGetLastError();
}

int launch_paged_read(const PagedView& v, const int32_t* start, const akv_rows& K, const akv_rows& V, int32_t T, void* stream) {
  const int64_t each = ((int64_t)T + kRowsAtOnce - 1) / kRowsAtOnce;
  const int64_t grid = grid_of(v, each);
  if (grid > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  akv_paged_read_kernel<<<(unsigned)grid, kThreads, 0, (cudaStream_t)stream>>>(v, start, rows_io(K), rows_io(V), T, (int)each);
  return (int)cudaGetLastError();
}

}  // namespace akv
