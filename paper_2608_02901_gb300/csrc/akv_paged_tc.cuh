// Device helpers of the paged cache's kernels on the fifth-generation tensor cores: codes as fp16 operands, tensor memory, election.
//
// An operand of 128 of K (a row's dimensions) is two panels of 64 in the 128-byte swizzled layout, whose columns are dimension
// 32 j + 8 t + i at panel j / 2, 16-byte chunk 4 (j & 1) + t, place 2 (i & 3) + i / 4: the order in which a word of eight codes comes apart.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace akv {
namespace {

constexpr uint32_t kPanel = 128 * 128;  // bytes of 64 of an operand's K for 128 of its rows
constexpr uint32_t kExtra = 128 * 32;   // 16 of K

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }  // -126 .. 127
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t bits(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
__device__ __forceinline__ void sts128(uint32_t a, uint4 x) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
// Registers of a warpgroup's threads; a kernel's shares add up to no more than its launch has.
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// One lane of the warp, the same each time.
__device__ __forceinline__ bool elect_one() {
  uint32_t on;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(on));
  return on != 0;
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 32 columns of the thread's lane of tensor memory
__device__ __forceinline__ void tm_ld32(uint32_t at, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      " tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(at)
      : "memory");
}
// 16 columns of three places, waited for together.
__device__ __forceinline__ void tm_ld16x3(uint32_t at0, uint32_t at1, uint32_t at2, float (&u)[16], float (&v)[16], float (&w)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%48];\n"
      " tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%49];\n"
      " tcgen05.ld.sync.aligned.32x32b.x16.b32 {%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47}, [%50];\n"
      " tcgen05.wait::ld.sync.aligned;"
      : "=f"(u[0]), "=f"(u[1]), "=f"(u[2]), "=f"(u[3]), "=f"(u[4]), "=f"(u[5]), "=f"(u[6]), "=f"(u[7]), "=f"(u[8]), "=f"(u[9]), "=f"(u[10]), "=f"(u[11]), "=f"(u[12]), "=f"(u[13]), "=f"(u[14]), "=f"(u[15]),
        "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]), "=f"(w[4]), "=f"(w[5]), "=f"(w[6]), "=f"(w[7]), "=f"(w[8]), "=f"(w[9]), "=f"(w[10]), "=f"(w[11]), "=f"(w[12]), "=f"(w[13]), "=f"(w[14]), "=f"(w[15])
      : "r"(at0), "r"(at1), "r"(at2)
      : "memory");
}
// 32 columns at 0 and 64, or at 0, 32 and 64, waited for together.
__device__ __forceinline__ void tm_ld32xn(uint32_t at, float (&v)[2][32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%64];\n"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%65];\n"
      " tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0][0]), "=f"(v[0][1]), "=f"(v[0][2]), "=f"(v[0][3]), "=f"(v[0][4]), "=f"(v[0][5]), "=f"(v[0][6]), "=f"(v[0][7]), "=f"(v[0][8]), "=f"(v[0][9]), "=f"(v[0][10]), "=f"(v[0][11]), "=f"(v[0][12]), "=f"(v[0][13]), "=f"(v[0][14]), "=f"(v[0][15]), "=f"(v[0][16]), "=f"(v[0][17]), "=f"(v[0][18]), "=f"(v[0][19]), "=f"(v[0][20]), "=f"(v[0][21]), "=f"(v[0][22]), "=f"(v[0][23]), "=f"(v[0][24]), "=f"(v[0][25]), "=f"(v[0][26]), "=f"(v[0][27]), "=f"(v[0][28]), "=f"(v[0][29]), "=f"(v[0][30]), "=f"(v[0][31]),
        "=f"(v[1][0]), "=f"(v[1][1]), "=f"(v[1][2]), "=f"(v[1][3]), "=f"(v[1][4]), "=f"(v[1][5]), "=f"(v[1][6]), "=f"(v[1][7]), "=f"(v[1][8]), "=f"(v[1][9]), "=f"(v[1][10]), "=f"(v[1][11]), "=f"(v[1][12]), "=f"(v[1][13]), "=f"(v[1][14]), "=f"(v[1][15]), "=f"(v[1][16]), "=f"(v[1][17]), "=f"(v[1][18]), "=f"(v[1][19]), "=f"(v[1][20]), "=f"(v[1][21]), "=f"(v[1][22]), "=f"(v[1][23]), "=f"(v[1][24]), "=f"(v[1][25]), "=f"(v[1][26]), "=f"(v[1][27]), "=f"(v[1][28]), "=f"(v[1][29]), "=f"(v[1][30]), "=f"(v[1][31])
      : "r"(at), "r"(at + 64)
      : "memory");
}
__device__ __forceinline__ void tm_ld32xn(uint32_t at, float (&v)[3][32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%96];\n"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%97];\n"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%64, %65, %66, %67, %68, %69, %70, %71, %72, %73, %74, %75, %76, %77, %78, %79, %80, %81, %82, %83, %84, %85, %86, %87, %88, %89, %90, %91, %92, %93, %94, %95}, [%98];\n"
      " tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0][0]), "=f"(v[0][1]), "=f"(v[0][2]), "=f"(v[0][3]), "=f"(v[0][4]), "=f"(v[0][5]), "=f"(v[0][6]), "=f"(v[0][7]), "=f"(v[0][8]), "=f"(v[0][9]), "=f"(v[0][10]), "=f"(v[0][11]), "=f"(v[0][12]), "=f"(v[0][13]), "=f"(v[0][14]), "=f"(v[0][15]), "=f"(v[0][16]), "=f"(v[0][17]), "=f"(v[0][18]), "=f"(v[0][19]), "=f"(v[0][20]), "=f"(v[0][21]), "=f"(v[0][22]), "=f"(v[0][23]), "=f"(v[0][24]), "=f"(v[0][25]), "=f"(v[0][26]), "=f"(v[0][27]), "=f"(v[0][28]), "=f"(v[0][29]), "=f"(v[0][30]), "=f"(v[0][31]),
        "=f"(v[1][0]), "=f"(v[1][1]), "=f"(v[1][2]), "=f"(v[1][3]), "=f"(v[1][4]), "=f"(v[1][5]), "=f"(v[1][6]), "=f"(v[1][7]), "=f"(v[1][8]), "=f"(v[1][9]), "=f"(v[1][10]), "=f"(v[1][11]), "=f"(v[1][12]), "=f"(v[1][13]), "=f"(v[1][14]), "=f"(v[1][15]), "=f"(v[1][16]), "=f"(v[1][17]), "=f"(v[1][18]), "=f"(v[1][19]), "=f"(v[1][20]), "=f"(v[1][21]), "=f"(v[1][22]), "=f"(v[1][23]), "=f"(v[1][24]), "=f"(v[1][25]), "=f"(v[1][26]), "=f"(v[1][27]), "=f"(v[1][28]), "=f"(v[1][29]), "=f"(v[1][30]), "=f"(v[1][31]),
        "=f"(v[2][0]), "=f"(v[2][1]), "=f"(v[2][2]), "=f"(v[2][3]), "=f"(v[2][4]), "=f"(v[2][5]), "=f"(v[2][6]), "=f"(v[2][7]), "=f"(v[2][8]), "=f"(v[2][9]), "=f"(v[2][10]), "=f"(v[2][11]), "=f"(v[2][12]), "=f"(v[2][13]), "=f"(v[2][14]), "=f"(v[2][15]), "=f"(v[2][16]), "=f"(v[2][17]), "=f"(v[2][18]), "=f"(v[2][19]), "=f"(v[2][20]), "=f"(v[2][21]), "=f"(v[2][22]), "=f"(v[2][23]), "=f"(v[2][24]), "=f"(v[2][25]), "=f"(v[2][26]), "=f"(v[2][27]), "=f"(v[2][28]), "=f"(v[2][29]), "=f"(v[2][30]), "=f"(v[2][31])
      : "r"(at), "r"(at + 32), "r"(at + 64)
      : "memory");
}
__device__ __forceinline__ void tm_st32(uint32_t at, const float (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31])
      : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t at, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] B[smem]^T
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
      ::"r"(d), "r"(a), "l"(b_desc), "r"(idesc), "r"(acc)
      : "memory");
}
// A row's first eight of 16 K without swizzle; the second eight are 2048 bytes on.
__device__ __forceinline__ uint32_t extra_at(int row) { return (uint32_t)((row >> 3) * 128 + (row & 7) * 16); }
// Nibbles e and e + 4 of x (e = 0 .. 3) as two fp16 numbers c, y = x >> 8: 1024 + c less 1024, or (1024 + 16 c) / 16 less 64.
struct ValueCodes {
  __half2 even = __float2half2_rn(-1024.f), odd = __float2half2_rn(-64.f), sixteenth = __float2half2_rn(0.0625f);
  __device__ __forceinline__ __half2 operator()(uint32_t x, uint32_t y, int e) const {
    const uint32_t z = e < 2 ? x : y;
    return e & 1 ? __hfma2(as_half2((z & 0x00f000f0u) | 0x64006400u), sixteenth, odd) : __hadd2(as_half2((z & 0x000f000fu) | 0x64006400u), even);
  }
};
// The same as 2 c - 15, x2 = x << 1, y2 = x >> 7: 1024 + 2 c less 1039, or (1024 + 32 c) / 16 less 79.
struct KeyCodes {
  __half2 even = __float2half2_rn(-1039.f), odd = __float2half2_rn(-79.f), sixteenth = __float2half2_rn(0.0625f);
  __device__ __forceinline__ __half2 operator()(uint32_t x2, uint32_t y2, int e) const {
    const uint32_t z = e < 2 ? x2 : y2;
    return e & 1 ? __hfma2(as_half2((z & 0x01e001e0u) | 0x64006400u), sixteenth, odd) : __hadd2(as_half2((z & 0x001e001eu) | 0x64006400u), even);
  }
};
// A key times 2 is (2 c - 15) a + (2 m + 15 a): the first goes into the products as an fp16 number and the exact rest, the second with the
// queries' sums in 16 more dimensions.  (Sums of codes from 0 up are larger than what they leave in the end, and the tensor cores cut at
// their size.)  Keys too large for fp16 enter as 2^-5 of that.
constexpr float kLargeDown = 0.03125f;
// A word of eight key codes: its places in the operand's halves.
__device__ __forceinline__ void key_word(const KeyCodes& codes, uint32_t x, __half2 scale, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
  const uint32_t x2 = x << 1, y2 = x >> 7;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __half2 c = codes(x2, y2, e), z = __hmul2(c, scale);
    hi[e] = bits(z);
    lo[e] = bits(__hfma2(c, scale, __hneg2(z)));
  }
}
// The 16 more dimensions of a key: 2 m + 15 a of each group (times `down`, a power of two) as two halves h, l against the three
// parts p of the queries' sum: h p0 + h p1 + h p2 + l p0 + l p1.  `spoil`: a NaN in their place.  Dimensions 10 to 12 are `ones`, for what a
// query row adds to all its logits.
template <int NG>
__device__ __forceinline__ void key_extra(const uint32_t (&words)[NG], float down, bool spoil, float ones, uint4& first, uint4& second) {
  uint32_t h[2] = {0, 0}, l[2] = {0, 0};
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const float a = __half2float(__ushort_as_half((unsigned short)words[g])), m = __half2float(__ushort_as_half((unsigned short)(words[g] >> 16)));
    const float z = fmaf(a, 15.f, 2.f * m) * down;
    const __half hi = __float2half_rn(z);
    h[g] = __half_as_ushort(hi);
    l[g] = __half_as_ushort(__float2half_rn(z - __half2float(hi)));
  }
  if (spoil) h[0] = 0x7e00u;
  first = make_uint4(h[0] * 0x10001u, h[0] | l[0] << 16, l[0] | h[1] << 16, h[1] * 0x10001u);
  const uint32_t one = __half_as_ushort(__float2half_rn(ones));
  second = make_uint4(l[1] * 0x10001u, one * 0x10001u, one, 0);
}
// Butterfly of R rows side by side (a row by itself waits for each of its exchanges).
template <int R>
__device__ __forceinline__ void wht_rows(float (&x)[R][4], int lane) {
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float a = x[r][0] + x[r][1], b = x[r][0] - x[r][1], c = x[r][2] + x[r][3], d = x[r][2] - x[r][3];
    x[r][0] = a + c, x[r][1] = b + d, x[r][2] = a - c, x[r][3] = b - d;
  }
#pragma unroll
  for (int h = 1; h < 32; h *= 2)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float o = __shfl_xor_sync(0xffffffffu, x[r][e], h);
        x[r][e] = lane & h ? o - x[r][e] : x[r][e] + o;
      }
}
// R query rows of akv_paged_query.cu by a warp, 8 or 16: from their records (lane r has row r's; null: zeros) into operand panels (hi, with HILO low
// halves two panels on) and the 16 more dimensions; place(r, row, panels, extra).  All loads come first: each would wait for the store before it.
template <bool HILO, int R, class Place>
__device__ __forceinline__ void place_queries(int lane, const uint8_t* record, Place place) {
  auto from = [&](int r) { return (const uint8_t*)__shfl_sync(0xffffffffu, (unsigned long long)record, r); };
  uint4 x[R], y = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint8_t* at = from(r);
    x[r] = make_uint4(0, 0, 0, 0);
    if (at && (HILO || lane < 16)) x[r] = *(const uint4*)(at + 16 * lane);
  }
  const uint8_t* at = from(lane >> 1 & (R - 1));
  if (at) y = *(const uint4*)(at + 512 + 16 * (lane & 1));
  const int c = lane & 15;  // chunk 4 j + t: panel j / 2, chunk 4 (j & 1) + t of it
  int row;
  uint32_t panels, extra;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    place(r, row, panels, extra);
    if (HILO || lane < 16)
      sts128(panels + (uint32_t)(lane >> 4) * (2 * kPanel) + (uint32_t)(c >> 3) * kPanel + 128 * row + 16 * ((c & 7) ^ (row & 7)), x[r]);
  }
  place(lane >> 1 & (R - 1), row, panels, extra);
  if (lane < 2 * R) sts128(extra + extra_at(row) + 2048 * (lane & 1), y);
}
// Operand of 16 K without swizzle: [2][16][8 rows][16 bytes], 2048 bytes from one half of K to the other, 128 between groups of rows.
__device__ __forceinline__ uint64_t plain_desc(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(2048u >> 4) << 16) | ((uint64_t)(128u >> 4) << 32) | ((uint64_t)1u << 46);
}

}  // namespace
}  // namespace akv
