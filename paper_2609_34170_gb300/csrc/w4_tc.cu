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

// A CTA takes 128 rows of weights, the MMAs' M, and NTOK tokens, their N.  Per piece of 128 ks:
//   four of the warps that widen do so: a thread takes half of the codes of two rows out of a ring of its warp
//     (asynchronous copies), makes them c - z in bf16 and stores them into A, two swizzled tiles of 64 ks;
//   one warp loads the tokens' values by TMA, two tiles of B;
//   one warp issues the MMAs.  A group's products are summed into an accumulator of their own, in turn;
//   eight warps take the accumulators, scale them by the group's scale and add them up in fp32 registers, half
//     of a row's tokens to a thread, and at the end of the ks store the outputs.
// So weights enter as whole numbers, as in the other kernels; no scaled weight is rounded.
//
// 64 rows x 65536 x 8192 with groups of 128 (268 MB of codes) 124 us: 2.4 TB/s, 0.55 PFLOP/s.  What bounds it is
// neither memory (44 us) nor the tensor core (an MMA of 128 x NTOK x 16 takes 71 cycles at any NTOK up to
// 128: 63 us) but the roles' own instructions: of the 1000 cycles a piece takes, the MMA warp spends 240 on its
// MMAs and the rest on waits that have mostly ended, commits and the loop, a warp that widens 2000 on every third
// piece, and a warp that sums 500 on scales and 250 on a piece's sums.  On the way here: tokens by asynchronous copies of
// four warps 225 (their addresses took longer than the MMAs), pieces of 64 ks 185, A in tensor memory the
// same as in shared memory, mma.sync with eight pairs of tiles sharing the tokens 267 (its MMAs alone are 113).
constexpr int kPieces = 3;      // pieces of A and B in the making
constexpr int kCodeRing = 2;    // pieces of codes on their way to a warp
constexpr int kScaleHalf = 4;   // groups' scales that come to a thread together, while as many are used
constexpr uint32_t kTcCols = 512;
constexpr int kSumPitch = 132;  // floats of a token's 128 rows
constexpr int kUpPitch = 68;    // of its 64 up rows
constexpr size_t kTcSmem = 227 * 1024;   // the SM's, as its tensor memory: CTAs of a cluster wait for one another with both taken

// GS: 32s of ks in a group
template <int NTOK, int GS>
struct TcShape {
  static constexpr int kSets = GS == 1 ? 2 : 3;          // of four warps that widen a piece (as many as have room for codes)
  static constexpr int kSumWarp = 4 * kSets, kXWarp = kSumWarp + 8, kMmaWarp = kXWarp + 1, kThreads = 32 * (kMmaWarp + 1);
  static constexpr int kGroups = 4 / GS;                 // of a piece
  // pieces whose accumulators there are; where they are as many as the pieces in the making, one barrier says of a
  // piece that its operands are free and its accumulators full (who waits for it is never a round behind: a piece is made,
  // and its accumulators written, only when both waits for the one three before have ended)
  static constexpr bool kOne = (int)kTcCols / NTOK / kGroups >= kPieces;
  static constexpr int kSlots = kOne ? kPieces : (int)kTcCols / NTOK / kGroups;
  struct Piece {
    uint8_t a[2][128 * 128], x[2][NTOK * 128];           // swizzled rows of 128 bytes
  };
  struct Codes {
    uint4 codes[2][2][32];                               // [64 ks][tile]
    uint2 sz[kGroups][2][8];
  };
  struct Shared {
    union {
      Piece pieces[kPieces];
      float sums[NTOK * kSumPitch];                      // for the other ranks, once every MMA is done
    };
    Codes ring[4 * kSets][kCodeRing];
    uint32_t scale[2][256][kScaleHalf];
    float up[NTOK * kUpPitch];                           // GeGLU's up rows
    uint64_t full[kPieces], empty[kPieces], acc_full[kSlots], acc_empty[kSlots], up_full, up_free, ended;
    uint32_t tmem;
  };
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

template <int NTOK, int GS>
__global__ void __launch_bounds__(TcShape<NTOK, GS>::kThreads, 1) w4_tc_kernel(const __grid_constant__ CUtensorMap x_map, W4Args a) {
  typedef TcShape<NTOK, GS> Shape;
  constexpr int kSets = Shape::kSets, kSumWarp = Shape::kSumWarp, kXWarp = Shape::kXWarp, kMmaWarp = Shape::kMmaWarp;
  constexpr int kGroups = Shape::kGroups, kSlots = Shape::kSlots;
  extern __shared__ __align__(1024) unsigned char tc_smem[];
  typename Shape::Shared& s = *(typename Shape::Shared*)tc_smem;
  const W4Matrix& w = a.w;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quarter = warp & 3;
  if (smem_u32(tc_smem) & 1023u) {   // (the swizzled layout counts on it)
    if (tid == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  const int ranks = (int)gridDim.z, rank = ranks > 1 ? (int)cluster_ctarank() : 0;
  const int row_tiles = (w.tiles + 7) / 8, units = row_tiles * ((a.M + NTOK - 1) / NTOK);
  // this rank's pieces
  const int pieces = (w.kblocks + 1) / 2;
  const int p0 = (int)((long long)pieces * rank / ranks), p1 = (int)((long long)pieces * (rank + 1) / ranks), pieces_here = p1 - p0;
  const int mine = (int)blockIdx.x < units ? (units - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;   // units

  // codes of the sequence of pieces (unit by unit), every kSets-th of them, into the warp's ring
  int next_unit = blockIdx.x, next_piece = p0, next_slot = 0;
  const uint4 *from0 = nullptr, *from1 = nullptr;   // this lane's part of a block of 64 ks, by tile
  const uint2* from_sz = nullptr;                   // this lane's part of a tile's scales
  const int sz_t = lane >> 2 & 1, sz_g = lane >> 3;
  auto skip = [&](int n) {   // n pieces on
    const int unit = next_unit;
    next_piece += n;
    while (next_piece >= p1 && next_unit < units) next_piece -= pieces_here, next_unit += gridDim.x;
    if (unit != next_unit || !from0) {
      const int tile0 = next_unit % row_tiles * 8 + 2 * quarter;   // (past the end: anything that is finite)
      const int t0 = min(tile0, w.tiles - 1), t1 = min(tile0 + 1, w.tiles - 1);
      from0 = w.codes + (size_t)t0 * w.kblocks * 32 + lane;
      from1 = w.codes + (size_t)t1 * w.kblocks * 32 + lane;
      from_sz = w.sz + (size_t)(sz_t ? t1 : t0) * w.groups * 8 + (lane & 3) * 2;
    }
  };
  // parts change places with the rows, so that eight lanes that read a part of eight rows hit all banks
  const int put = (lane >> 2) * 4 + ((lane & 3) ^ (lane >> 3));
  auto fetch = [&] {
    if (next_unit < units) {
      typename Shape::Codes& to = s.ring[warp][next_slot];
      // (past the last block there are no values, and its codes will do)
      const size_t b0 = (size_t)(2 * next_piece) * 32, b1 = (size_t)min(2 * next_piece + 1, w.kblocks - 1) * 32;
      copy_async(&to.codes[0][0][put], from0 + b0, true);
      copy_async(&to.codes[0][1][put], from1 + b0, true);
      copy_async(&to.codes[1][0][put], from0 + b1, true);
      copy_async(&to.codes[1][1][put], from1 + b1, true);
      if (sz_g < kGroups)
        copy_async(&to.sz[sz_g][sz_t][(lane & 3) * 2], from_sz + (size_t)min(next_piece * kGroups + sz_g, w.groups - 1) * 8, true);
      if (++next_slot == kCodeRing) next_slot = 0;
      skip(kSets);
    }
    copies_commit();
  };
  // scales of the sequence of groups, a thread its row's
  const int srow = quarter * 32 + lane, sthread = (tid - 32 * kSumWarp) & 255;
  const int group0 = p0 * kGroups, groups_here = pieces_here * kGroups;
  int scale_unit = blockIdx.x, scale_at = 0;
  const uint32_t scale_to = smem_u32(&s.scale[0][sthread][0]);
  const uint32_t* from_scale = nullptr;   // of the unit's first group
  // half of the ring: the next kScaleHalf groups of the unit (past the last one there are no values, and its
  // scale will do: every unit takes whole halves)
  auto fetch_scales = [&](int half) {
    if (scale_unit < units) {
      if (scale_at == 0) {
        const int tile = min(scale_unit % row_tiles * 8 + (srow >> 4), w.tiles - 1);
        from_scale = (const uint32_t*)w.sz + ((size_t)tile * w.groups * 8 + (srow & 7)) * 2 + (srow >> 3 & 1);
      }
      const int at = group0 + scale_at, most = w.groups - 1;
#pragma unroll
      for (int i = 0; i < kScaleHalf; ++i)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(scale_to + half * (256 * kScaleHalf * 4) + i * 4),
                     "l"(from_scale + 16 * (size_t)(uint32_t)min(at + i, most))
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
    for (int i = 0; i < kPieces; ++i) {
      mbar_init(&s.full[i], 5);   // four warps that widen, and the tokens' bytes
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < kSlots; ++i) {
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
    const int t = lane >> 4, g = lane & 7, hi = lane >> 3 & 1, set = warp / 4;
    int slot = 0, at = set % kPieces;                    // the warp's first piece of the sequence, in the ring of pieces
    uint32_t parity = 1u ^ (uint32_t)(set / kPieces);    // of empty[at]
    for (long long left = (long long)mine * pieces_here - set; left > 0; left -= kSets) {
      copies_wait<kCodeRing - 2>();
      __syncwarp();
      fetch();   // (into the slot that was read last)
      const typename Shape::Codes& from = s.ring[warp][slot];
      if (++slot == kCodeRing) slot = 0;
      typename Shape::Piece& to = s.pieces[at];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t z0[2], z8[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint2 sz = from.sz[(2 * half + h) / GS][t][g];
          z0[h] = __byte_perm(sz.x, 0u, 0x1010);
          z8[h] = __byte_perm(sz.y, 0u, 0x1010);
        }
        uint4 c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) c[i] = from.codes[half][t][g * 4 + ((2 * hi + i) ^ (g >> 1))];
        if (half == 0) {
          ok = wait_for(&s.empty[at], parity);
          if (!ok) break;
        }
        // word 2h + s of part q: ks 32h + 8q + 4s .., nibbles 0, 2 of row g and 1, 3 of row g + 8; a row's 16 bytes 4h + q
        // change places with the row (by the same for both)
        uint8_t* row = to.a[half] + (quarter * 32 + t * 16 + g) * 128;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t word[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r0[4], r8[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t v = word[2 * h + e];
              r0[2 * e] = sub_bf16x2((v & 0x000f000fu) | 0x43004300u, z0[h]);
              r8[2 * e] = sub_bf16x2((v >> 4 & 0x000f000fu) | 0x43004300u, z8[h]);
              r0[2 * e + 1] = sub_bf16x2((v >> 8 & 0x000f000fu) | 0x43004300u, z0[h]);
              r8[2 * e + 1] = sub_bf16x2((v >> 12 & 0x000f000fu) | 0x43004300u, z8[h]);
            }
            uint8_t* piece = row + (((4 * h + 2 * hi + i) ^ g) << 4);
            *(uint4*)piece = make_uint4(r0[0], r0[1], r0[2], r0[3]);
            *(uint4*)(piece + 8 * 128) = make_uint4(r8[0], r8[1], r8[2], r8[3]);
          }
        }
      }
      if (!ok) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.full[at]);
      at += kSets;
      if (at >= kPieces) at -= kPieces, parity ^= 1u;
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
      for (int piece = 0; piece < pieces_here; ++piece) {
        const int in_half = piece * kGroups % kScaleHalf;
        if (in_half == 0) copies_wait<1>();
        float scale[kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) scale[i] = __uint_as_float(s.scale[half][sthread][in_half + i] & 0xffff0000u);
        if (in_half + kGroups == kScaleHalf || piece + 1 == pieces_here) {   // (this half is read)
          fetch_scales(half);
          half ^= 1;
        }
        ok = wait_for(Shape::kOne ? &s.empty[acc_at] : &s.acc_full[acc_at], parity);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int group = 0; group < kGroups; ++group) {
          uint32_t v[kTok / 16][16];
#pragma unroll
          for (int i = 0; i < kTok / 16; ++i) tmem_ld16_async(tmem + lanes + (acc_at * kGroups + group) * NTOK + first + i * 16, v[i]);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < kTok / 16; ++i) tmem_reg_fence16(v[i]);
          if (group == kGroups - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.acc_empty[acc_at]);
          }
#pragma unroll
          for (int i = 0; i < kTok; i += 2) fma_pair(sum[i], sum[i + 1], v[i / 16][i % 16], v[i / 16][i % 16 + 1], scale[group]);
        }
        if (++acc_at == kSlots) acc_at = 0, parity ^= 1u;
      }
      if (!ok) break;
      if (ranks > 1) {   // (the only unit, and its last MMA is done: the pieces are free)
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
          for (int i = 0; i < kTok; ++i) s.up[(first + i) * kUpPitch + srow - 64] = sum[i] + bias;
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.up_full);
        } else {
          ok = wait_for(&s.up_full, up_parity);
          if (!ok) break;
          bf16* out = (bf16*)a.out + (size_t)(m0 + first) * a.ldo + tile * 64 + srow;
#pragma unroll
          for (int i = 0; i < kTok; ++i)
            if (first + i < tokens) out[(size_t)i * a.ldo] = from_f32<bf16>(gelu_tanh_f(sum[i] + bias) * s.up[(first + i) * kUpPitch + srow]);
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
    int at = 0;
    uint32_t parity = 1u;
    long long issued = 0;
    for (int unit = blockIdx.x; unit < units && ok; unit += gridDim.x) {
      const int m0 = unit / row_tiles * NTOK;
      for (int piece = p0; piece < p1; ++piece) {
        ok = wait_for(&s.empty[at], parity);
        if (!ok) break;
        mbar_expect_tx_el(&s.full[at], 2 * NTOK * 128, el);
        tma_load_2d_el(&x_map, smem_u32(&s.full[at]), smem_u32(s.pieces[at].x[0]), piece * 128, m0, keep, el);
        tma_load_2d_el(&x_map, smem_u32(&s.full[at]), smem_u32(s.pieces[at].x[1]), piece * 128 + 64, m0, keep, el);
        ++issued;
        if (++at == kPieces) at = 0, parity ^= 1u;
      }
    }
    // nobody leaves with loads in flight, not even where a wait ran out
    for (long long n = issued > kPieces ? issued - kPieces : 0; n < issued; ++n)
      ok = wait_for(&s.full[n % kPieces], (uint32_t)(n / kPieces) & 1u) && ok;
  } else {
    const uint32_t el = elect_one();
    const uint32_t idesc = idesc_bf16(128, NTOK);
    const uint64_t ad0 = sw128_desc(smem_u32(s.pieces[0].a[0])), xd0 = sw128_desc(smem_u32(s.pieces[0].x[0]));
    int at = 0, acc_at = 0;
    uint32_t parity = 0u, acc_parity = 1u;
    for (long long left = (long long)mine * pieces_here; left > 0; --left) {
      ok = wait_for(&s.full[at], parity);
      if (!ok) break;
      ok = wait_for(&s.acc_empty[acc_at], acc_parity);
      if (!ok) break;
      tc_fence_after();
      const uint32_t ahead = (uint32_t)(at * (sizeof(typename Shape::Piece) >> 4));
      const uint64_t ad = ad0 + ahead, xd = xd0 + ahead;
      const uint32_t td = tmem + acc_at * kGroups * NTOK;
#pragma unroll
      for (int j = 0; j < 8; ++j) {   // 16 ks each
        const int group = j / (2 * GS);
        umma_bf16(td + group * NTOK, ad + (j / 4) * (128 * 128 >> 4) + 2 * (j % 4), xd + (j / 4) * (NTOK * 128 >> 4) + 2 * (j % 4), idesc,
                  j % (2 * GS) > 0 ? 1u : 0u, el);
      }
      if (!Shape::kOne) umma_commit(&s.acc_full[acc_at], el);
      umma_commit(&s.empty[at], el);
      if (++acc_at == kSlots) acc_at = 0, acc_parity ^= 1u;
      if (++at == kPieces) at = 0, parity ^= 1u;
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
    for (int e = e0 + tid; e < e1; e += Shape::kThreads) {
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

template <int NTOK, int GS>
cudaError_t init_gs() {
  static_assert(sizeof(typename TcShape<NTOK, GS>::Shared) <= kTcSmem, "shared memory");
  static_assert(sizeof(typename TcShape<NTOK, GS>::Piece) % 1024 == 0, "swizzled tiles");
  return cudaFuncSetAttribute(w4_tc_kernel<NTOK, GS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kTcSmem);
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
  // the ks of a unit over as many CTAs (1, 2, 4, 8) as there are SMs for and two pieces for each
  int ranks = 1;
  while (ranks < kRanks && units * ranks * 2 <= a.num_sms && a.w.kblocks >= ranks * 2 * 4) ranks *= 2;
  const Overlap overlap;
  return launch_kernel_cluster(w4_tc_kernel<NTOK, GS>, dim3(ranks > 1 ? units : std::min(units, a.num_sms), 1, ranks),
                               dim3(TcShape<NTOK, GS>::kThreads), kTcSmem, st, dim3(1, 1, ranks), map, a);
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
