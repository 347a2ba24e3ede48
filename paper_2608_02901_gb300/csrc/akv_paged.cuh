// Device helpers of the paged 4-bit cache: addresses, types, the rotation.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "akv_internal.h"

namespace akv {
namespace {

// Every launch of these files is a programmatic dependent of what runs before it in its stream: its CTAs may be set up
// beside that, and wait for its end (and for its writes) before they touch memory.  Every CTA waits, so that whoever
// depends on the launch has waited for all before it as well.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <class... Params, class... Args>
int launch_after(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, void* stream, Args... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute pdl{};
  pdl.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  pdl.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = &pdl;
  cfg.numAttrs = 1;
  return (int)cudaLaunchKernelEx(&cfg, kernel, (Params)args...);
}

__device__ __forceinline__ float row_to_float(uint16_t x, int half) {
  return half ? __half2float(__ushort_as_half(x)) : __uint_as_float((uint32_t)x << 16);
}
__device__ __forceinline__ uint16_t float_to_row(float x, int half) {
  return half ? __half_as_ushort(__float2half_rn(x)) : __bfloat16_as_ushort(__float2bfloat16_rn(x));
}

// Tokens that request b holds, as every kernel reads them.
__device__ __forceinline__ int held_tokens(const PagedView& v, int b) {
  return min(max(v.lens[b], 0), v.max_pages << v.page_log);
}
// Page of table position j of request b, -1 where it is none of the pool's.
__device__ __forceinline__ int page_of(const PagedView& v, int b, int j) {
  const int page = v.table[(int64_t)b * v.table_stride + j];
  return (uint32_t)page < (uint32_t)v.n_pages ? page : -1;
}
__device__ __forceinline__ uint8_t* block_of(const PagedView& v, int page, int h) {
  return v.base + (uint64_t)page * v.page_bytes + (uint64_t)h * v.block_bytes;
}
// +0 or -0 pattern that flips the sign of dimension d where the rotation does.
__device__ __forceinline__ uint32_t sign_flip(const PagedView& v, int d) {
  return (uint32_t)((d < 64 ? v.sign_bits[0] : v.sign_bits[1]) >> (d & 63) & 1ull) << 31;
}

// Butterfly (stages 1, 2, 4, .., 64) of a row spread over a warp, four dimensions a lane (d = 4 lane + e).
__device__ __forceinline__ void wht_32x4(float (&x)[4], int lane) {
  float a = x[0] + x[1], b = x[0] - x[1], c = x[2] + x[3], d = x[2] - x[3];
  x[0] = a + c;
  x[1] = b + d;
  x[2] = a - c;
  x[3] = b - d;
#pragma unroll
  for (int h = 1; h < 32; h *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float o = __shfl_xor_sync(0xffffffffu, x[e], h);
      x[e] = lane & h ? o - x[e] : x[e] + o;
    }
}

__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

}  // namespace
}  // namespace akv
