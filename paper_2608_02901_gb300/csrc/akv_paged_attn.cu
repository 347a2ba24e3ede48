// Attention over the paged 4-bit cache.
#include "akv_paged.cuh"

namespace akv {
namespace {

constexpr float kNegInf = -__builtin_huge_valf();

// One CTA of 128 threads: one query row.  Chunks of 128 tokens: a thread scores one token, then holds one dimension
// of the output.  fp32 throughout.
__global__ void __launch_bounds__(kD) akv_paged_attn_kernel(PagedView v, const uint16_t* q, int64_t qb, int64_t qt, int64_t qh,
                                                            uint16_t* out, int64_t ob, int64_t ot, int64_t oh, float* lse, int T,
                                                            float sm_scale, const int32_t* sel, const int32_t* count, int top) {
  const int Hq = v.H * v.G;
  const int hq = blockIdx.x % Hq, t = blockIdx.x / Hq % T, b = blockIdx.x / Hq / T;
  const int h = hq / v.G, d = threadIdx.x, lane = d & 31, warp = d >> 5;
  const int P = 1 << v.page_log;
  const int sees = max(0, held_tokens(v, b) - T + 1 + t);
  __shared__ float qs[kD], p[kD], red[4], ys[kD];
  __shared__ const uint8_t* sub_of[kD];
  const float x0 = row_to_float(q[b * qb + t * qt + hq * qh + d], v.half);
  if (v.rotate) {
    ys[d] = __uint_as_float(__float_as_uint(x0) ^ sign_flip(v, d));
    __syncthreads();
    if (warp == 0) {
      float x[4];
      for (int e = 0; e < 4; ++e) x[e] = ys[4 * lane + e];
      wht_32x4(x, lane);
      for (int e = 0; e < 4; ++e) qs[4 * lane + e] = x[e] * 0.0625f;
    }
  } else {
    qs[d] = x0;
  }
  const int64_t unit = ((int64_t)b * T + t) * v.H + h;
  const int n_sel = sel ? min(max(count[unit], 0), top) : 0;
  const int n = sel ? n_sel << v.page_log : sees;
  float m = kNegInf, l = 0.f, y = 0.f;
  bool bad = false;
  for (int i0 = 0; i0 < n; i0 += kD) {
    __syncthreads();
    const int i = i0 + d;
    int pos = i, j = i >> v.page_log;
    bool there = i < n;
    if (there && sel) {
      j = sel[unit * top + j];
      there = (uint32_t)j < (uint32_t)v.max_pages;
      pos = there ? (j << v.page_log) + (i & P - 1) : 0;
    }
    there = there && pos < sees;
    const int page = there ? page_of(v, b, j) : -1;
    bad = bad || (there && page < 0);
    const uint8_t* sub = page < 0 ? nullptr : block_of(v, page, h) + (uint32_t)((pos & P - 1) >> 4) * sub_bytes(v.ng);
    sub_of[d] = sub;
    float s = kNegInf;
    if (sub) {
      s = 0.f;
      for (int g = 0; g < v.ng; ++g) {
        const uint32_t w = *(const uint32_t*)(sub + 2048 + 4 * (2 * v.ng * (pos & 15) + g));
        const float a = row_to_float((uint16_t)w, 1), mn = row_to_float((uint16_t)(w >> 16), 1);
        for (int e = g * kD / v.ng; e < (g + 1) * kD / v.ng; ++e) s += qs[e] * fmaf((float)key_code(sub, pos & 15, e), a, mn);
      }
      s *= sm_scale;
    }
    float top_s = s;
    for (int k = 16; k; k >>= 1) top_s = max_nan(top_s, __shfl_xor_sync(0xffffffffu, top_s, k));
    if (lane == 0) red[warp] = top_s;
    __syncthreads();
    const float mn = max_nan(m, max_nan(max_nan(red[0], red[1]), max_nan(red[2], red[3])));
    const float f = m == kNegInf ? 0.f : expf(m - mn);
    p[d] = s == kNegInf ? 0.f : expf(s - mn);
    m = mn;
    l *= f;
    y *= f;
    __syncthreads();
    for (int k = 0; k < min(kD, n - i0); ++k) {
      const uint8_t* sb = sub_of[k];
      if (!sb) continue;
      const int i16 = i0 + k & 15;  // (a page's tokens keep their place in the list)
      const uint32_t w = *(const uint32_t*)(sb + 2048 + 4 * (2 * v.ng * i16 + v.ng + d / (kD / v.ng)));
      y += p[k] * fmaf((float)value_code(sb, i16, d), row_to_float((uint16_t)w, 1), row_to_float((uint16_t)(w >> 16), 1));
      l += p[k];
    }
  }
  bad = __syncthreads_or(bad);
  ys[d] = l != 0.f ? y / l : 0.f;
  __syncthreads();
  if (v.rotate && warp == 0) {
    float x[4];
    for (int e = 0; e < 4; ++e) x[e] = ys[4 * lane + e];
    wht_32x4(x, lane);
    for (int e = 0; e < 4; ++e) ys[4 * lane + e] = __uint_as_float(__float_as_uint(x[e] * 0.0625f) ^ sign_flip(v, 4 * lane + e));
  }
  __syncthreads();
  const float nan = __int_as_float(0x7fffffff);
  out[b * ob + t * ot + hq * oh + d] = float_to_row(bad ? nan : ys[d], v.half);
  if (lse && d == 0) lse[((int64_t)b * T + t) * Hq + hq] = bad ? nan : l == 0.f ? kNegInf : m + logf(l);
}

}  // namespace

size_t paged_attn_ws_bytes(const PagedView&, int32_t, int32_t) { return 256; }

int launch_paged_attn(const PagedView& v, const akv_rows& q, const akv_rows& out, float* lse, int32_t T, float sm_scale,
                      const akv_selection* sel, void*, void* stream) {
  const int64_t grid = (int64_t)v.rows * T * v.H * v.G;
  if (grid > INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  akv_paged_attn_kernel<<<(unsigned)grid, kD, 0, (cudaStream_t)stream>>>(
      v, (const uint16_t*)q.ptr, q.stride_b, q.stride_t, q.stride_h, (uint16_t*)out.ptr, out.stride_b, out.stride_t, out.stride_h,
      lse, T, sm_scale, sel ? sel->pages : nullptr, sel ? sel->count : nullptr, sel ? sel->top : 0);
  return (int)cudaGetLastError();
}

}  // namespace akv
