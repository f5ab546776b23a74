// Device helpers of the 8-bit context cache: e4m3 conversions and block exponents.
#pragma once

#include "cache.h"
#include "common.cuh"

namespace ravel {

// two floats -> two e4m3 (nearest, ties to even; finite inputs within 448), lo in the low byte
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// the low / high two e4m3 of a word -> f16x2 (exact; NaN stays NaN)
__device__ __forceinline__ uint32_t e4m3_lo(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t e4m3_hi(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, b;\n\t}" : "=r"(r) : "r"(w));
  return r;
}

__device__ __forceinline__ float f16lo(uint32_t h) {
  float r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, a;\n\t}" : "=f"(r) : "r"(h));
  return r;
}
__device__ __forceinline__ float f16hi(uint32_t h) {
  float r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, b;\n\t}" : "=f"(r) : "r"(h));
  return r;
}

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float exp2i(int e) { return __int_as_float((e + 127) << 23); }

// The smallest e >= kCacheExpMin with x * 2^up <= 448 * 2^e = 1.75 * 2^(e + 8), from the
// bits of a finite x >= 0: exact.
__device__ __forceinline__ int block_exponent(uint32_t bits, int up) {
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0) + up;
  return max(e, kCacheExpMin);
}

__device__ __forceinline__ void e4m3x16_to_f32(const uint4& w, float scale, float* x) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = e4m3_lo(u[i]), b = e4m3_hi(u[i]);
    x[4 * i] = f16lo(a) * scale;
    x[4 * i + 1] = f16hi(a) * scale;
    x[4 * i + 2] = f16lo(b) * scale;
    x[4 * i + 3] = f16hi(b) * scale;
  }
}

__device__ __forceinline__ uint4 f32_to_e4m3x16(const float* x, float scale) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    u[i] = to_e4m3x2(x[4 * i] * scale, x[4 * i + 1] * scale) |
           to_e4m3x2(x[4 * i + 2] * scale, x[4 * i + 3] * scale) << 16;
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// What the launch before wrote, or other CTAs of this one, is read by plain loads or by these:
// launches overlap, so that no tensor is read-only for as long as a kernel lives, and a load
// of the read-only path (or one that the compiler takes for a pure function) might be older
// than the wait in front of it (volatile statements stay in their order, the wait's among them).
// l2: past the L1; once: read only once; kept: read by many warps of a CTA
__device__ __forceinline__ float ld_l2(const float* p) {
  float v;
  asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float2 ld_l2(const float2* p) {
  float2 v;
  asm volatile("ld.global.cg.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_l2(const float4* p) {
  float4 v;
  asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float2 ld_once(const float2* p) {
  float2 v;
  asm volatile("ld.global.cs.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ float2 ld_kept(const float2* p) {
  float2 v;
  asm volatile("ld.global.L1::evict_last.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
  return v;
}

// 16 values of a row from dim d on (zeros from hd on; hd is a multiple of 8)
template <typename T>
__device__ __forceinline__ void load16(const T* row, int d, int hd, int vec, float* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int d8 = d + 8 * h;
    if (d8 >= hd) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[8 * h + i] = 0.f;
    } else if (vec) {
      constexpr int NV = 8 * sizeof(T) / 16;
      uint4 w[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) w[i] = *((const uint4*)(row + d8) + i);
      const T* p = (const T*)w;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[8 * h + i] = to_f32(p[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[8 * h + i] = to_f32(row[d8 + i]);
    }
  }
}

}  // namespace ravel
