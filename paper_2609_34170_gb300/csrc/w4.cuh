// Device helpers of the products with 4-bit weights.
#pragma once

#include "common.cuh"
#include "decode.h"
#include "tc_common.cuh"

namespace ravel {

constexpr int kRanks = 4;    // CTAs that share the ks of their rows at most

// CTAs (1, 2, 4) that share the ks of a unit of work: as many as there are SMs for and `blocks` of 64 ks for each.
inline int w4_ranks(long long units, int kblocks, int blocks, int most, int sms) {
  int ranks = 1;
  while (ranks < most && units * ranks * 2 <= sms && kblocks >= ranks * 2 * blocks) ranks *= 2;
  return ranks;
}
inline int w4_tc_tokens(int M) { return M <= 32 ? 32 : 64; }   // of a unit of the tcgen05 kernel
// How the tcgen05 kernel goes through a matrix: the units (128 rows of weights x 32 or 64 tokens) of the last round, if
// there are few, are shared (after full rounds, whose CTAs all have to be there at once, by 2 CTAs).  Clusters of 8 of CTAs
// that fill an SM start late: 64 rows x 2048 x 8192 16.7 us with them, 10.8 with 4.
struct W4TcPlan {
  int grid, ranks;
  long long pieces;   // of 128 ks, of the CTA that has most
  W4TcPlan(const W4Args& a, int tokens) {
    const int units = (a.w.tiles + 7) / 8 * ((a.M + tokens - 1) / tokens), sms = a.num_sms / 2 * 2, all = (a.w.kblocks + 1) / 2;
    const bool rounds = units >= a.num_sms;
    const int last = rounds ? units % sms : units;
    ranks = last > 0 ? w4_ranks(last, a.w.kblocks, 4, rounds ? 2 : kRanks, sms) : 1;
    grid = !rounds ? units * ranks : ranks > 1 ? sms : a.num_sms;
    pieces = (rounds ? (long long)(units / sms) * all : 0) + (last > 0 ? (all + ranks - 1) / ranks : 0);
  }
};

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight values of a row from k on; what is not there is zero (a code past the end stands for
// weight 0, but 0 times a neighbour's NaN is not).
__device__ __forceinline__ uint4 load_x(const bf16* row, int k, int K, bool there) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  if (!there || k >= K) return r;
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

__device__ __forceinline__ void copy_async(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

}  // namespace ravel
