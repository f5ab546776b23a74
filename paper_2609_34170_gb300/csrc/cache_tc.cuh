// What the tensor-core kernels of the 8-bit context cache share: operands in 8 bits,
// waits, and Q laid out in two pieces.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include "cache_attn.cuh"

namespace ravel {

constexpr int BM = 128, BT = 128;              // rows, tokens of a tile
constexpr uint32_t QB = BM * 64;               // bytes of a 64-dim block of a piece of Q
constexpr uint32_t KU = BT * 64;               // bytes of a K unit: 128 tokens x 64 dims
constexpr int kQExp = 7;                        // Q's largest magnitude per row is below 2^(kQExp + 1)

// Shared-memory descriptor of a K-major tile of 64-byte rows, 64-byte swizzled: 8-row
// groups 512 bytes apart.
__device__ __forceinline__ uint64_t sw64_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(512 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)4 << 61;
}

// D += A B of 8-bit operands (K = 32), issued by the elected lane of a converged warp
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t el) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(el));
}

// f16 A and B (kind::f16) or e4m3 ones (kind::f8f6f4, of which one may be e5m2), fp32 D
constexpr uint32_t kE5m2A = 1u << 7, kE5m2B = 1u << 10;
__device__ __forceinline__ uint32_t idesc_f16(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ void sts_u4(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds_u4(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ float4 lds_f4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts_u2(uint32_t a, uint32_t x, uint32_t y) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory");
}
// two f16 -> two e4m3 (nearest, ties to even; NaN stays NaN), low halves first
__device__ __forceinline__ uint32_t f16_to_e4m3(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
  return r;
}
// and two e5m2
__device__ __forceinline__ uint32_t f16_to_e5m2(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
  return r;
}
__device__ __forceinline__ uint32_t f16_sub(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Two fp32 operations an instruction, and the larger of three: the softmax is bound by the
// instructions that it issues.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Wait of a converged warp for a phase, bounded: 2^24 tries of 20 to 200 cycles each.  Four
// instructions a try: twenty warps whose waits read the global timer between tries, as those
// of kernels with fewer do, took over half of an SM's issue slots; tries with a time hint
// sleep past the arrival.
__device__ __forceinline__ bool wait_phase(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\t"
      "mov.u32 n, 0;\n\t"
      "TRY: mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra DONE;\n\t"
      "add.u32 n, n, 1;\n\t"
      "setp.lt.u32 q, n, 16777216;\n\t"
      "@q bra TRY;\n\t"
      "DONE: selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return __all_sync(0xffffffffu, ok != 0);
}

// The same for up to four phases, tried side by side (a try's latency is most of a wait's for
// what has arrived; one behind the other, four waits took 500 cycles).  All lanes wait for
// the same barriers.
__device__ __forceinline__ bool wait_phases(uint64_t* b0, uint32_t p0, uint64_t* b1, uint32_t p1, uint64_t* b2, uint32_t p2,
                                            uint64_t* b3, uint32_t p3) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p, q, r, s, t;\n\t.reg .u32 n;\n\t"
      "mov.u32 n, 0;\n\t"
      "TRY: mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 r, [%3], %4;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 s, [%5], %6;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 t, [%7], %8;\n\t"
      "and.pred p, p, r;\n\t"
      "and.pred s, s, t;\n\t"
      "and.pred p, p, s;\n\t"
      "@p bra DONE;\n\t"
      "add.u32 n, n, 1;\n\t"
      "setp.lt.u32 q, n, 16777216;\n\t"
      "@q bra TRY;\n\t"
      "DONE: selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(b0)), "r"(p0), "r"(smem_u32(b1)), "r"(p1), "r"(smem_u32(b2)), "r"(p2), "r"(smem_u32(b3)), "r"(p3)
      : "memory");
  return __all_sync(0xffffffffu, ok != 0);
}

// A warp's writes to shared memory become visible to the tensor core: one arrival per warp.
__device__ __forceinline__ void written(uint64_t* bar) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// One value of a converged warp, so that the compiler knows it: the operands of the
// asynchronous instructions then stay in uniform registers.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Q rows rb .. rb + 7 of the tile of rows from r0 on of robot b, KV head h (8 NB lanes
// with 8 dims each to a row), scaled by the row's power of two to a largest magnitude
// in [2^kQExp, 2^(kQExp + 1)), in two pieces: y rounded to e4m3, and what is left, in e5m2.
// Of a y from 2^-6 on (2^-13 of the row's largest) that is at most 8 units of bf16's last
// place, three bits: the pieces are y.  Below, what is left is rounded to e5m2 by at most
// 2^-14: an element is never off by more than 2^-21 of the row's largest magnitude.  (An e4m3
// rest would end at 2^-9, 2^-17 of the largest: small dims beside a large one that the keys do
// not use were lost.)  64-byte rows of 64 dims, 64-byte swizzled, blocks of QB bytes, the second piece NB blocks
// behind the first: into shared memory at q0 or, where `to` is given, there.  row_done:
// called by one lane with each row's place in the tile and its exponent bits.
template <int NB, typename F>
__device__ __forceinline__ void stage_q8(const CacheAttnArgs& a, const Sight& s, int b, int h, int r0, int rb, uint32_t q0,
                                         uint8_t* to, F row_done) {
  const int lane = threadIdx.x & 31;
  constexpr int LPR = 8 * NB, RPW = 32 / LPR, PASS = 8 / RPW;
  const int sub = lane / LPR < RPW ? lane / LPR : 0, dl = lane % LPR;
  const bool mine = lane / LPR < RPW, on = mine && 8 * dl < a.c.hd;
  // (a row that does not exist reads the robot's first: loads without branches, all on
  // their way together)
  const uint32_t end_row = (uint32_t)(s.count * a.G);
  const bf16* base = (const bf16*)a.q + (size_t)((long long)b * a.q_robot) + (size_t)h * a.G * a.c.hd + (on ? 8 * dl : 0);
  uint32_t r = (uint32_t)(r0 + rb + sub), i = a.by_G.of(r), g = r - i * (uint32_t)a.G, there = 0u;
  uint4 x[PASS];
  const bf16* at[PASS];
#pragma unroll
  for (int p = 0; p < PASS; ++p) {
    at[p] = base;
    if (r < end_row) {
      there |= on ? 1u << p : 0u;
      at[p] += (size_t)((long long)i * a.q_token) + (size_t)g * a.c.hd;
    }
    r += RPW;
    g += RPW;
    while (g >= (uint32_t)a.G) {
      g -= (uint32_t)a.G;
      ++i;
    }
  }
  if (a.vec) {
#pragma unroll
    for (int p = 0; p < PASS; ++p) x[p] = *(const uint4*)at[p];
  } else {
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      bf16 y[8];
#pragma unroll
      for (int z = 0; z < 8; ++z) y[z] = at[p][z];
      memcpy(&x[p], y, 16);
    }
  }
#pragma unroll
  for (int p = 0; p < PASS; ++p) {
    const bool t = there >> p & 1u;
    const uint32_t y[4] = {t ? x[p].x : 0u, t ? x[p].y : 0u, t ? x[p].z : 0u, t ? x[p].w : 0u};
    // the largest magnitude's bits: NaN counts as larger than all
    uint32_t top = __vmaxu2(__vmaxu2(y[0] & 0x7fff7fffu, y[1] & 0x7fff7fffu), __vmaxu2(y[2] & 0x7fff7fffu, y[3] & 0x7fff7fffu));
    top = max(top >> 16, top & 0xffffu);
    if (RPW == 1) {
      top = __reduce_max_sync(0xffffffffu, top);
    } else {
#pragma unroll
      for (int o = 1; o < LPR; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    const int e = (int)(top >> 7);
    const float f = e == 255 ? __int_as_float(0x7fffffff) : exp2i(min(kQExp + 127 - e, 126));
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const uint32_t h0 = pack_f16x2(__uint_as_float(y[2 * z] << 16) * f, __uint_as_float(y[2 * z] & 0xffff0000u) * f);
      const uint32_t h1 = pack_f16x2(__uint_as_float(y[2 * z + 1] << 16) * f, __uint_as_float(y[2 * z + 1] & 0xffff0000u) * f);
      hi[z] = f16_to_e4m3(h0) | f16_to_e4m3(h1) << 16;
      lo[z] = f16_to_e5m2(f16_sub(h0, e4m3_lo(hi[z]))) | f16_to_e5m2(f16_sub(h1, e4m3_hi(hi[z]))) << 16;
    }
    const int lr = rb + p * RPW + sub;
    if (mine) {
      const uint32_t off = (uint32_t)(dl >> 3) * QB + (uint32_t)lr * 64u +
                           (uint32_t)((((dl >> 1) & 3) ^ ((lr >> 1) & 3)) * 16 + (dl & 1) * 8);
      if (to) {
        *(uint2*)(to + off) = make_uint2(hi[0], hi[1]);
        *(uint2*)(to + off + NB * QB) = make_uint2(lo[0], lo[1]);
      } else {
        sts_u2(q0 + off, hi[0], hi[1]);
        sts_u2(q0 + off + NB * QB, lo[0], lo[1]);
      }
      if (dl == 0) row_done(lr, e);
    }
  }
}

// Softmax factor of a row whose largest |q| has exponent bits e.  (Rows below 2^-119
// keep fewer bits; -x >= -126.)
__device__ __forceinline__ float q_factor(int e, float scale_log2) {
  return exp2i(-min(kQExp + 127 - e, 126)) * scale_log2;
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void st_cluster_f4(uint32_t a, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster_f2(uint32_t a, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ float ld_cluster_f1(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a));
  return v;
}

// the encoder of tensor maps; a layer's codes [B Hkv T][hdp] in boxes of `in` dims x
// box_rows, swizzled over rows of `in` bytes or not
cudaError_t cache_tc_encoder();
cudaError_t encode_codes(CUtensorMap* m, const uint8_t* base, const CacheLayer& c, int batch, int in, int box_rows,
                         bool swizzle);

}  // namespace ravel
