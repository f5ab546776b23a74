// Products with 4-bit weights for more tokens than a warp's MMAs carry at the pace of memory: tcgen05, with
// the weights widened into shared memory.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "decode.h"
#include "launch.h"
#include "tc_common.cuh"
#include "w4.cuh"

namespace ravel {
namespace {

// A CTA takes 128 rows of weights, the MMAs' M, and NTOK tokens, their N.  Per block of 64 ks:
//   four of 12 warps widen: a thread takes a row's 64 codes out of a ring of its warp (asynchronous copies),
//     makes them c - z in bf16 and stores them as the row's 128 bytes of A, in a swizzled tile;
//   one warp loads the tokens' values by TMA into a swizzled tile, which is B;
//   one warp issues the MMAs.  A group's products are summed into an accumulator of their own, in turn;
//   eight warps take the accumulators, scale them by the group's scale and add them up in fp32 registers, half
//     of a row's tokens to a thread, and at the end of the ks store the outputs.
// So weights enter as whole numbers, as in the other kernels; no scaled weight is rounded.
//
// An MMA of 128 x NTOK x 16 occupies the tensor core for 71 cycles at any NTOK up to 128, a block of 128 x
// 64 weights (4 KB) for 284: 14 bytes a cycle, two thirds of what memory delivers.  MEASURED
constexpr int kSets = 3;        // of four warps that widen a block
constexpr int kSumWarp = 4 * kSets, kXWarp = kSumWarp + 8, kMmaWarp = kXWarp + 1;
constexpr int kTcThreads = 32 * (kMmaWarp + 1);
constexpr int kBlocks = 3;      // blocks of A
constexpr int kXBlocks = 6;     // blocks of B, most of them on their way (their latency is that of four blocks' MMAs)
constexpr int kCodeRing = 4;    // blocks of codes on their way to a warp
constexpr int kScaleHalf = 4;   // groups' scales that come to a thread together, while as many are used
constexpr uint32_t kTcCols = 256;
constexpr int kSumPitch = 132;  // floats of a token's 128 rows

template <int NTOK, int GS>
struct TcShared {
  static constexpr int kAccs = (int)kTcCols / NTOK;
  uint8_t a[kBlocks][128 * 128];                        // swizzled rows of 128 bytes, as x
  uint8_t x[kXBlocks][NTOK * 128];                      // swizzled rows of 128 bytes
  uint4 codes[4 * kSets][kCodeRing][2][32];
  uint2 sz[4 * kSets][kCodeRing][GS == 1 ? 2 : 1][2][8];
  uint32_t scale[2 * kScaleHalf][256];
  float sums[NTOK * kSumPitch];                         // GeGLU's up rows, or the sums for the other ranks
  uint64_t full[kBlocks], empty[kBlocks], x_full[kXBlocks], x_empty[kXBlocks], acc_full[kAccs], acc_empty[kAccs], up_full, up_free, ended;
  uint32_t tmem;
};

// x += a s, y += b s in one instruction
__device__ __forceinline__ void fma_pair(float& x, float& y, uint32_t a, uint32_t b, float s) {
  asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %4};\n\tmov.b64 r, {%0, %1};\n\t"
      "fma.rn.f32x2 r, p, q, r;\n\tmov.b64 {%0, %1}, r;\n\t}"
      : "+f"(x), "+f"(y)
      : "r"(a), "r"(b), "f"(s));
}

// A wait that tries some times before it looks at the clock.
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity) {
  for (int i = 0; i < 64; ++i)
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return mbar_wait_warp(bar, parity);
}

// GS: 32s of ks in a group
template <int NTOK, int GS>
__global__ void __launch_bounds__(kTcThreads, 1) w4_tc_kernel(const __grid_constant__ CUtensorMap x_map, W4Args a) {
  typedef TcShared<NTOK, GS> Shared;
  constexpr int kAccs = Shared::kAccs;
  extern __shared__ __align__(1024) unsigned char tc_smem[];
  Shared& s = *(Shared*)tc_smem;
  const W4Matrix& w = a.w;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (smem_u32(tc_smem) & 1023u) {   // (the swizzled layout counts on it)
    if (tid == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  const int ranks = (int)gridDim.z, rank = ranks > 1 ? (int)cluster_ctarank() : 0;
  const int row_tiles = (w.tiles + 7) / 8, units = row_tiles * ((a.M + NTOK - 1) / NTOK);
  // this rank's blocks, whole groups of them
  constexpr int kGran = GS == 4 ? 2 : 1;
  const int grains = (w.kblocks + kGran - 1) / kGran;
  const int k0 = min((int)((long long)grains * rank / ranks) * kGran, w.kblocks);
  const int k1 = min((int)((long long)grains * (rank + 1) / ranks) * kGran, w.kblocks);
  constexpr int per_group = GS == 4 ? 7 : GS == 2 ? 6 : 5;

  // codes of the sequence of blocks (unit by unit), every kSets-th of them, into the warp's ring
  const int blocks_here = k1 - k0, quarter = warp & 3;
  int next_unit = blockIdx.x, next_kb = k0, next_slot = 0;
  const uint4 *from0 = nullptr, *from1 = nullptr;   // this lane's pieces of the next block, by tile
  const uint2* from_sz = nullptr;                   // this lane's piece of the tile's scales
  const int sz_t = lane >> 2 & 1, sz_h = lane >> 3;
  auto skip = [&](int n) {   // n blocks on
    const int unit = next_unit;
    next_kb += n;
    while (next_kb >= k1 && next_unit < units) next_kb -= blocks_here, next_unit += gridDim.x;
    if (unit != next_unit || !from0) {
      const int tile0 = next_unit % row_tiles * 8 + 2 * quarter;   // (past the end: anything that is finite)
      const int t0 = min(tile0, w.tiles - 1), t1 = min(tile0 + 1, w.tiles - 1);
      from0 = w.codes + ((size_t)t0 * w.kblocks + next_kb) * 32 + lane;
      from1 = w.codes + ((size_t)t1 * w.kblocks + next_kb) * 32 + lane;
      from_sz = w.sz + (size_t)(sz_t ? t1 : t0) * w.groups * 8 + (lane & 3) * 2;
    } else {
      from0 += n * 32;
      from1 += n * 32;
    }
  };
  // pieces change places with the rows, so that eight lanes that read a piece of eight rows hit all banks
  const int put = (lane >> 2) * 4 + ((lane & 3) ^ (lane >> 3));
  auto fetch = [&] {
    if (next_unit < units) {
      copy_async(&s.codes[warp][next_slot][0][put], from0, true);
      copy_async(&s.codes[warp][next_slot][1][put], from1, true);
      if (sz_h < (GS == 1 ? 2 : 1)) {
        const int group = min((next_kb * 64 + sz_h * 32) >> per_group, w.groups - 1);
        copy_async(&s.sz[warp][next_slot][sz_h][sz_t][(lane & 3) * 2], from_sz + (size_t)group * 8, true);
      }
      if (++next_slot == kCodeRing) next_slot = 0;
      skip(kSets);
    }
    copies_commit();
  };
  // scales of the sequence of groups, a thread its row's
  const int srow = quarter * 32 + lane, sthread = (tid - 32 * kSumWarp) & 255;
  const int group0 = k0 * 2 / GS, groups_here = (blocks_here * 2 + GS - 1) / GS;
  int scale_unit = blockIdx.x, scale_at = 0;
  const uint32_t scale_to = smem_u32(&s.scale[0][sthread]);
  // half of the ring: the next kScaleHalf groups of the unit (past the last one there are no values, and its
  // scale will do: every unit takes whole halves)
  auto fetch_scales = [&](int half) {
    if (scale_unit < units) {
      const int tile = min(scale_unit % row_tiles * 8 + (srow >> 4), w.tiles - 1);
      const uint32_t* from = (const uint32_t*)w.sz + (((size_t)tile * w.groups + group0) * 8 + (srow & 7)) * 2 + (srow >> 3 & 1);
#pragma unroll
      for (int i = 0; i < kScaleHalf; ++i)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(scale_to + (half * kScaleHalf + i) * 1024),
                     "l"(from + 16 * (size_t)min(scale_at + i, w.groups - 1 - group0))
                     : "memory");
      scale_at += kScaleHalf;
      if (scale_at >= groups_here) scale_at = 0, scale_unit += gridDim.x;
    }
    copies_commit();
  };

  // loaded weights do not change: on their way before the launch before has ended
  if (warp < kSumWarp) {
    skip(warp / 4);
    for (int i = 0; i < kCodeRing - 1; ++i) fetch();
  } else if (warp < kXWarp) {
    fetch_scales(0);
    fetch_scales(1);
  }
  if (tid == 0) {
    for (int i = 0; i < kBlocks; ++i) {
      mbar_init(&s.full[i], 4);   // the warps that widen it
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < kXBlocks; ++i) {
      mbar_init(&s.x_full[i], 1);
      mbar_init(&s.x_empty[i], 1);
    }
    for (int i = 0; i < kAccs; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 8);
    }
    mbar_init(&s.up_full, 4);
    mbar_init(&s.up_free, 4);
    mbar_init(&s.ended, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_trigger();
  pdl_wait();   // (before any TMEM is taken: the launch before may still need it)
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "r"(kTcCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  const uint32_t tmem = s.tmem;
  bool ok = true;

  if (warp < kSumWarp) {
    const int t = lane >> 4, g = lane & 7, hi = lane >> 3 & 1;
    int slot = 0, block = warp / 4;   // the warp's first block of the sequence, in the ring of blocks
    uint32_t parity = 1u;             // of empty[block]
    if (block >= kBlocks) block -= kBlocks, parity ^= 1u;
    int unit = blockIdx.x, kb = k0;
    auto on = [&](int n) {
      kb += n;
      while (kb >= k1 && unit < units) kb -= blocks_here, unit += gridDim.x;
    };
    for (on(warp / 4); unit < units; on(kSets)) {
        copies_wait<kCodeRing - 2>();
        __syncwarp();
        fetch();   // (into the slot that was read last)
        uint32_t z[GS == 1 ? 2 : 1];
#pragma unroll
        for (int h = 0; h < (GS == 1 ? 2 : 1); ++h)
          z[h] = __byte_perm(((const uint32_t*)&s.sz[warp][slot][h][t][g])[hi], 0u, 0x1010);
        uint32_t out[2][16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 c4 = s.codes[warp][slot][t][g * 4 + (q ^ (g >> 1))];
          const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {   // word 2h + s: ks 32h + 8q + 4s ..
            const uint32_t v = c[i] >> 4 * hi, zz = z[GS == 1 ? i >> 1 : 0];
            out[i >> 1][q * 4 + (i & 1) * 2] = sub_bf16x2((v & 0x000f000fu) | 0x43004300u, zz);
            out[i >> 1][q * 4 + (i & 1) * 2 + 1] = sub_bf16x2((v >> 8 & 0x000f000fu) | 0x43004300u, zz);
          }
        }
        if (++slot == kCodeRing) slot = 0;
        ok = wait_for(&s.empty[block], parity);
        if (!ok) break;
        // pieces of 16 bytes change places with the rows
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t* v = &out[j >> 2][(j & 3) * 4];
          *(uint4*)(s.a[block] + srow * 128 + ((j ^ (srow & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.full[block]);
        block += kSets;
        if (block >= kBlocks) block -= kBlocks, parity ^= 1u;
    }
  } else if (warp < kXWarp) {
    constexpr int kTok = NTOK / 2;   // of a thread
    const int first = (warp - kSumWarp) / 4 * kTok;
    int acc_at = 0, half = 0;
    uint32_t parity = 0u, up_parity = 0u;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    for (int unit = blockIdx.x; unit < units && ok; unit += gridDim.x) {
      const int m0 = unit / row_tiles * NTOK, tile = unit % row_tiles, row = tile * 128 + srow, tokens = min(NTOK, a.M - m0);
      float sum[kTok];
#pragma unroll
      for (int i = 0; i < kTok; ++i) sum[i] = 0.f;
      for (int group = 0; group < groups_here; ++group) {
        if (group % kScaleHalf == 0) copies_wait<1>();
        const float scale = __uint_as_float(s.scale[half * kScaleHalf + group % kScaleHalf][sthread] & 0xffff0000u);
        if (group % kScaleHalf == kScaleHalf - 1 || group + 1 == groups_here) {   // (this half is read)
          fetch_scales(half);
          half ^= 1;
        }
        ok = wait_for(&s.acc_full[acc_at], parity);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[kTok / 16][16];
#pragma unroll
        for (int i = 0; i < kTok / 16; ++i) tmem_ld16_async(tmem + lanes + acc_at * NTOK + first + i * 16, v[i]);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < kTok / 16; ++i) tmem_reg_fence16(v[i]);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.acc_empty[acc_at]);
        if (++acc_at == kAccs) acc_at = 0, parity ^= 1u;
#pragma unroll
        for (int i = 0; i < kTok; i += 2) fma_pair(sum[i], sum[i + 1], v[i / 16][i % 16], v[i / 16][i % 16 + 1], scale);
      }
      if (!ok) break;
      if (ranks > 1) {   // (the only unit)
#pragma unroll
        for (int i = 0; i < kTok; ++i) s.sums[(first + i) * kSumPitch + srow] = sum[i];
        continue;
      }
      const float bias = a.bias && row < w.N ? a.bias[row] : 0.f;
      if (a.epi == EPI_GEGLU) {   // (bounded waits: a warp that gave up does not come)
        if (quarter >= 2) {
          ok = wait_for(&s.up_free, up_parity ^ 1u);
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < kTok; ++i) s.sums[(first + i) * kSumPitch + srow] = sum[i] + bias;
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.up_full);
        } else {
          ok = wait_for(&s.up_full, up_parity);
          if (!ok) break;
          bf16* out = (bf16*)a.out + (size_t)(m0 + first) * a.ldo + tile * 64 + srow;
#pragma unroll
          for (int i = 0; i < kTok; ++i)
            if (first + i < tokens) out[(size_t)i * a.ldo] = from_f32<bf16>(gelu_tanh_f(sum[i] + bias) * s.sums[(first + i) * kSumPitch + srow + 64]);
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.up_free);
        }
        up_parity ^= 1u;
      } else if (row < w.N) {
        const size_t at = (size_t)(m0 + first) * a.ldo + row;
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
          if (first + i >= tokens) break;
          const size_t to = at + (size_t)i * a.ldo;
          float v = sum[i] + bias;
          if (a.epi == EPI_STORE_SILU) v = silu_f(v);
          if (a.epi == EPI_ADD_F32) ((float*)a.out)[to] += v;
          else if (a.out_bf16) ((bf16*)a.out)[to] = from_f32<bf16>(v);
          else ((float*)a.out)[to] = v;
        }
      }
    }
  } else if (warp < kMmaWarp) {
    const uint32_t el = elect_one();
    uint64_t keep;   // (every CTA reads them)
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(keep));
    int block = 0, issued = 0;
    uint32_t parity = 1u;
    for (int unit = blockIdx.x; unit < units && ok; unit += gridDim.x) {
      const int m0 = unit / row_tiles * NTOK;
      for (int kb = k0; kb < k1; ++kb) {
        ok = wait_for(&s.x_empty[block], parity);
        if (!ok) break;
        mbar_expect_tx_el(&s.x_full[block], NTOK * 128, el);
        tma_load_2d_el(&x_map, smem_u32(&s.x_full[block]), smem_u32(s.x[block]), kb * 64, m0, keep, el);
        ++issued;
        if (++block == kXBlocks) block = 0, parity ^= 1u;
      }
    }
    // nobody leaves with loads in flight, not even where a wait ran out
    for (int n = max(0, issued - kXBlocks); n < issued; ++n) ok = wait_for(&s.x_full[n % kXBlocks], (n / kXBlocks) & 1u) && ok;
  } else {
    const uint32_t el = elect_one();
    const uint32_t idesc = idesc_bf16(128, NTOK);
    const uint64_t xd0 = sw128_desc(smem_u32(s.x[0])), ad0 = sw128_desc(smem_u32(s.a[0]));
    constexpr int kAccsOf = GS == 1 ? 2 : 1;   // accumulators that a block begins
    int block = 0, x_block = 0, acc_at = 0, in_unit = 0;
    uint32_t parity = 0u, x_parity = 0u, acc_parity = 1u;
    const int mine = blockIdx.x < units ? (units - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;
    for (long long left = (long long)mine * blocks_here; left > 0; --left) {
      // GS 4: a group is two blocks, or one at the end
      const bool first = GS < 4 || (in_unit & 1) == 0, last = GS < 4 || (in_unit & 1) || in_unit + 1 == blocks_here;
      ok = wait_for(&s.x_full[x_block], x_parity);
      if (!ok) break;
      ok = wait_for(&s.full[block], parity);
      if (!ok) break;
      if (first) {
        ok = wait_for(&s.acc_empty[acc_at], acc_parity);
        if (!ok) break;
        if (kAccsOf == 2) {   // (the accumulators are an even number)
          ok = wait_for(&s.acc_empty[acc_at + 1], acc_parity);
          if (!ok) break;
        }
      }
      tc_fence_after();
      const uint64_t ad = ad0 + (uint32_t)(block * (128 * 128 >> 4)), xd = xd0 + (uint32_t)(x_block * (NTOK * 128 >> 4));
      const uint32_t td = tmem + acc_at * NTOK, more = first ? 0u : 1u;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        umma_bf16(td + (kAccsOf == 2 ? (j >> 1) * NTOK : 0), ad + 2 * j, xd + 2 * j, idesc, j % (4 / kAccsOf) > 0 ? 1u : more, el);
      if (last) {
        umma_commit(&s.acc_full[acc_at], el);
        if (kAccsOf == 2) umma_commit(&s.acc_full[acc_at + 1], el);
        acc_at += kAccsOf;
        if (acc_at == kAccs) acc_at = 0, acc_parity ^= 1u;
      }
      umma_commit(&s.empty[block], el);
      umma_commit(&s.x_empty[x_block], el);
      if (++block == kBlocks) block = 0, parity ^= 1u;
      if (++x_block == kXBlocks) x_block = 0, x_parity ^= 1u;
      if (++in_unit == blocks_here) in_unit = 0;
    }
    umma_commit(&s.ended, el);   // nothing is in flight when the columns are given back
    ok = wait_for(&s.ended, 0u) && ok;
  }
  copies_wait<0>();
  if (!ok && lane == 0) raise_error(a.err, ERR_TIMEOUT);
  if (ranks > 1) {
    cluster_sync();
    const int unit = blockIdx.x, m0 = unit / row_tiles * NTOK, tile = unit % row_tiles, tokens = min(NTOK, a.M - m0);
    const bool glu = a.epi == EPI_GEGLU;
    const int shift = glu ? 6 : 7, all = tokens << shift, e0 = all * rank / ranks, e1 = all * (rank + 1) / ranks;
    for (int e = e0 + tid; e < e1; e += kTcThreads) {
      const int m = e >> shift, r = e & ((1 << shift) - 1), row = tile * 128 + r;
      auto value = [&](int r) {
        const int n = tile * 128 + r;
        return over_ranks(&s.sums[m * kSumPitch + r], ranks) + (a.bias && n < w.N ? a.bias[n] : 0.f);
      };
      float v = value(r);
      if (glu) {
        ((bf16*)a.out)[(size_t)(m0 + m) * a.ldo + tile * 64 + r] = from_f32<bf16>(gelu_tanh_f(v) * value(r + 64));
        continue;
      }
      if (row >= w.N) continue;
      const size_t to = (size_t)(m0 + m) * a.ldo + row;
      if (a.epi == EPI_STORE_SILU) v = silu_f(v);
      if (a.epi == EPI_ADD_F32) ((float*)a.out)[to] += v;
      else if (a.out_bf16) ((bf16*)a.out)[to] = from_f32<bf16>(v);
      else ((float*)a.out)[to] = v;
    }
    cluster_sync();   // nobody leaves while its sums are read
  }
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTcCols) : "memory");
}

// Shared memory, at least the columns' share of the SM's, so that CTAs that fit together in the one fit in
// the other (a cluster's CTAs wait for one another with their columns taken).
template <int NTOK, int GS>
constexpr size_t tc_smem_of() {
  constexpr size_t share = (size_t)kTcCols * (228 * 1024) / 512 - 1024;
  return sizeof(TcShared<NTOK, GS>) > share ? sizeof(TcShared<NTOK, GS>) : share;
}

template <int NTOK, int GS>
cudaError_t init_gs() {
  return cudaFuncSetAttribute(w4_tc_kernel<NTOK, GS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tc_smem_of<NTOK, GS>());
}

std::atomic<void*> g_encode{nullptr};

cudaError_t get_encoder() {
  if (g_encode.load()) return cudaSuccess;
  cudaDriverEntryPointQueryResult q;
  void* fn = nullptr;
  const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
  if (e != cudaSuccess) return e;
  if (q != cudaDriverEntryPointSuccess || !fn) return cudaErrorSymbolNotFound;
  g_encode.store(fn);
  return cudaSuccess;
}

template <int NTOK, int GS>
cudaError_t launch_gs(const W4Args& a, cudaStream_t st) {
  CUtensorMap map;   // boxes of NTOK tokens x 64 ks, zeros past the ends
  cuuint64_t dims[2] = {(cuuint64_t)a.w.K, (cuuint64_t)a.M};
  cuuint64_t strides[1] = {(cuuint64_t)a.lda * 2};
  cuuint32_t box[2] = {64, NTOK}, steps[2] = {1, 1};
  const auto encode = (PFN_cuTensorMapEncodeTiled_v12000)g_encode.load();
  if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.x), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  const int units = (a.w.tiles + 7) / 8 * ((a.M + NTOK - 1) / NTOK);
  // the ks of a unit over as many CTAs (1, 2, 4, 8) as there are SMs for and four blocks for each
  int ranks = 1;
  while (ranks < kRanks && units * ranks * 2 <= a.num_sms && a.w.kblocks >= ranks * 2 * 4) ranks *= 2;
  const Overlap overlap;
  return launch_kernel_cluster(w4_tc_kernel<NTOK, GS>, dim3(ranks > 1 ? units : std::min(units, a.num_sms), 1, ranks), dim3(kTcThreads),
                               tc_smem_of<NTOK, GS>(), st, dim3(1, 1, ranks), map, a);
}

template <int NTOK>
cudaError_t launch_ntok(const W4Args& a, cudaStream_t st) {
  return a.w.group == 128 ? launch_gs<NTOK, 4>(a, st) : a.w.group == 64 ? launch_gs<NTOK, 2>(a, st) : launch_gs<NTOK, 1>(a, st);
}

}  // namespace

cudaError_t init_w4_tc_kernels() {
  cudaError_t e = get_encoder();
  if (e == cudaSuccess) e = init_gs<32, 1>();
  if (e == cudaSuccess) e = init_gs<32, 2>();
  if (e == cudaSuccess) e = init_gs<32, 4>();
  if (e == cudaSuccess) e = init_gs<64, 1>();
  if (e == cudaSuccess) e = init_gs<64, 2>();
  if (e == cudaSuccess) e = init_gs<64, 4>();
  return e;
}

cudaError_t launch_w4_tc(const W4Args& a, cudaStream_t st) {
  return a.M <= 32 ? launch_ntok<32>(a, st) : launch_ntok<64>(a, st);
}

}  // namespace ravel
