// Device helpers of the products with 4-bit weights.
#pragma once

#include "common.cuh"
#include "decode.h"
#include "tc_common.cuh"

namespace ravel {

constexpr int kRanks = 8;    // CTAs that share the ks of their rows at most

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight values of a row from k on; what is not there is zero (a code past the end stands for
// weight 0, but 0 times a neighbour's NaN is not).
__device__ __forceinline__ uint4 load_x(const bf16* row, int k, int K, bool there, int vec) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  if (!there || k >= K) return r;
  if (vec && k + 8 <= K) return *(const uint4*)(row + k);
  uint16_t v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = k + i < K ? ((const uint16_t*)row)[k + i] : 0;
  memcpy(&r, v, 16);
  return r;
}

__device__ __forceinline__ float ld_cluster_f(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// One sum of all ranks, in their order (the loads on their way together).
__device__ __forceinline__ float over_ranks(const float* p, int ranks) {
  const uint32_t at = smem_u32(p);
  float x[kRanks];
#pragma unroll
  for (int i = 0; i < kRanks; ++i) x[i] = ld_cluster_f(mapa_shared(at, (uint32_t)min(i, ranks - 1)));
  float v = x[0];
#pragma unroll
  for (int i = 1; i < kRanks; ++i) v += i < ranks ? x[i] : 0.f;
  return v;
}

__device__ __forceinline__ void copy_async(void* to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

}  // namespace ravel
