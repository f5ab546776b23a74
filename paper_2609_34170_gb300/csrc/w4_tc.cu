// Products with 4-bit weights for more tokens than a warp's MMAs carry at the pace of memory: tcgen05, with
// the weights widened into tensor memory.
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
//   four of the warps that widen do so: a thread takes the codes of two rows out of a ring of its warp (asynchronous
//     copies), makes them c - z in bf16 and stores them into A, in tensor memory, as the fragments that they are;
//   one warp loads the tokens' values by TMA, two swizzled tiles of B, and every eight groups the rows' scales;
//   one warp issues the MMAs.  A group's products are summed into an accumulator of their own, in turn;
//   eight warps take the accumulators, scale them by the group's scale and add them up in fp32 registers, half
//     of a row's tokens to a thread, and at the end of the ks store the outputs.
// So weights enter as whole numbers, as in the other kernels; no scaled weight is rounded.
//
// 64 rows x 65536 x 8192 with groups of 128 (268 MB of codes) 93 us: 3.0 TB/s, 0.74 PFLOP/s.  What bounds it is
// neither memory (44 us) nor the tensor pipe (busy for 30 % of an SM's active cycles) but the roles' own instructions, some ten
// cycles each with 22 warps on four schedulers (which issue in 66 % of the cycles, the integer pipe busy for 65 %): of
// the 830 cycles that a piece takes at the 1.93 GHz seen, the warps that sum need all for some 100 of them, a warp that widens
// 1800 on every third piece, and the MMA warp 700 for its wait, a commit and eight MMAs, each of which (128 x NTOK x 16) keeps it for
// 71 at any NTOK up to 128: 568 cycles of a piece, 63 us in all.  Measured on the way here (same product, us): mma.sync with eight
// pairs of tiles sharing the tokens 267; tokens by asynchronous copies of four warps 225; pieces of 64 ks 185; A in shared
// memory, three pieces in the making, scales by copies of each thread 124; A in tensor memory and scales by bulk copies
// 111; the last of 3.4 rounds shared by pairs of CTAs and outputs without a branch each 98; units joined a token to a
// warp 93.  Warps that sum in turn, all of a row's tokens to a thread that has more registers, are no
// faster.
constexpr int kSets = 3;        // of four warps that widen a piece
constexpr int kScaleBatch = kPadGroups, kScaleBufs = 3;   // groups of a unit whose scales come together; batches there is room for
constexpr int kScalePitch = kScaleBatch * 64 + 64;         // bytes of a tile's: rows of two tiles in different banks
constexpr uint32_t kTcCols = 512;
constexpr int kSumPitch = 132;  // floats of a token's 128 rows
constexpr int kUpPitch = 68;    // of its 64 up rows
constexpr size_t kTcSmem = 227 * 1024;   // the SM's, as its tensor memory: CTAs of a cluster wait for one another with both taken
constexpr int kSumWarp = 4 * kSets, kXWarp = kSumWarp + 8, kMmaWarp = kXWarp + 1, kTcThreads = 32 * (kMmaWarp + 1);

// GS: 32s of ks in a group
template <int NTOK, int GS>
struct TcShape {
  static constexpr int kBlocks = 2;                      // of 64 ks in a piece
  static constexpr int kGroups = 2 * kBlocks / GS;       // of a piece
  static constexpr int kColsA = 32 * kBlocks, kColsAcc = kGroups * NTOK;   // of tensor memory
  // pieces in the making, and pieces whose accumulators there are; where they are as many, one barrier says of a
  // piece that its operands are free and its accumulators full, and one that its operands are there and its accumulators
  // free (who waits for them is never a round behind: a piece is made, and its accumulators written, only when both
  // waits for the one before it in its place have ended)
  static constexpr int kFit = (int)kTcCols / (kColsA + kColsAcc);
  static constexpr bool kOne = kFit >= 3;
  static constexpr int kPieces = kOne ? (kFit < 4 ? kFit : 4) : 3;
  static constexpr int kSlots = kOne ? kPieces : ((int)kTcCols - kPieces * kColsA) / kColsAcc;
  static constexpr int kCodeRing = 4;                     // pieces of codes on their way to a warp
  struct Piece {
    uint8_t x[kBlocks][NTOK * 128];                      // swizzled rows of 128 bytes
  };
  struct Codes {
    uint4 codes[kBlocks][2][32];                         // [64 ks][tile]
    uint2 sz[kGroups][2][8];
  };
  struct Shared {
    union {
      Piece pieces[kPieces];
      float sums[NTOK * kSumPitch];                      // for the other ranks, once every MMA is done
    };
    Codes ring[4 * kSets][kCodeRing];
    float up[NTOK * kUpPitch];                           // GeGLU's up rows
    alignas(16) uint8_t scales[kScaleBufs][8][kScalePitch];
    uint64_t scale_full[kScaleBufs], scale_empty[kScaleBufs], full[kPieces], empty[kPieces], acc_full[kSlots], acc_empty[kSlots], up_full, up_free, ended;
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

// 16 rows x 64 ks of A (lanes from those of at on): lane 4g + q's columns 2q, 2q + 1 of each 8 of rows g and g + 8.
__device__ __forceinline__ void store_a(uint32_t at, const uint32_t (&v)[4][4]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at),
      "r"(v[0][0]), "r"(v[0][1]), "r"(v[0][2]), "r"(v[0][3]), "r"(v[1][0]), "r"(v[1][1]), "r"(v[1][2]), "r"(v[1][3]), "r"(v[2][0]),
      "r"(v[2][1]), "r"(v[2][2]), "r"(v[2][3]), "r"(v[3][0]), "r"(v[3][1]), "r"(v[3][2]), "r"(v[3][3])
      : "memory");
}

// A wait that tries some times before it looks at the clock.
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity) {
  for (int i = 0; i < 64; ++i)
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return mbar_wait_warp(bar, parity);
}

template <int NTOK, int GS>
__global__ void __launch_bounds__(kTcThreads, 1) w4_tc_kernel(const __grid_constant__ CUtensorMap x_map, W4Args a, int ranks) {
  typedef TcShape<NTOK, GS> Shape;
  constexpr int kPieces = Shape::kPieces, kSlots = Shape::kSlots, kBlocks = Shape::kBlocks, kGroups = Shape::kGroups;
  constexpr int kCodeRing = Shape::kCodeRing;
  extern __shared__ __align__(1024) unsigned char tc_smem[];
  typename Shape::Shared& s = *(typename Shape::Shared*)tc_smem;
  const W4Matrix& w = a.w;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quarter = warp & 3;
  if (smem_u32(tc_smem) & 1023u) {   // (the swizzled layout counts on it)
    if (tid == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  const int rank = ranks > 1 ? (int)cluster_ctarank() : 0;
  const int row_tiles = (w.tiles + 7) / 8, units = row_tiles * ((a.M + NTOK - 1) / NTOK);
  const int pieces = (w.kblocks + kBlocks - 1) / kBlocks;
  // Units go round the CTAs.  With ranks > 1 the units of the round that is not full go to a cluster each, whose CTAs share
  // its pieces.
  const int full = ranks > 1 ? units / (int)gridDim.x : (int)blockIdx.x < units ? (units - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;
  const int last_unit = full * (int)gridDim.x + (int)blockIdx.x / ranks;
  const bool joint = ranks > 1 && last_unit < units;
  const int rounds = full + joint, p0 = (int)((long long)pieces * rank / ranks), p1 = (int)((long long)pieces * (rank + 1) / ranks);
  auto unit_of = [&](int round) { return round < full ? (int)blockIdx.x + round * (int)gridDim.x : last_unit; };
  auto first_of = [&](int round) { return round < full ? 0 : p0; };
  auto end_of = [&](int round) { return round < full ? pieces : p1; };

  // codes of the sequence of pieces (unit by unit), every kSets-th of them, into the warp's ring
  int next_round = 0, next_piece = first_of(0), next_end = end_of(0), next_slot = 0;
  const uint4 *from0 = nullptr, *from1 = nullptr;   // this lane's part of a block of 64 ks, by tile
  const uint2* from_sz = nullptr;                   // this lane's part of a tile's scales
  const int sz_t = lane >> 2 & 1, sz_g = lane >> 3;
  auto skip = [&](int n) {   // n pieces on
    next_piece += n;
    if (next_piece >= next_end || !from0) {
      while (next_round < rounds && next_piece >= next_end) {
        next_piece += first_of(++next_round) - next_end;
        next_end = end_of(next_round);
      }
      const int tile0 = unit_of(next_round) % row_tiles * 8 + 2 * quarter;   // (past the end: anything that is finite)
      const int t0 = min(tile0, w.tiles - 1), t1 = min(tile0 + 1, w.tiles - 1);
      from0 = w.codes + (size_t)t0 * w.kblocks * 32 + lane;
      from1 = w.codes + (size_t)t1 * w.kblocks * 32 + lane;
      from_sz = w.sz + (size_t)(sz_t ? t1 : t0) * w.groups * 8 + (lane & 3) * 2;
    }
  };
  // parts change places with the rows, so that four rows' halves of parts hit all banks
  const int put = lane ^ (lane >> 2 & 2);
  auto fetch = [&] {
    if (next_round < rounds) {
      typename Shape::Codes& to = s.ring[warp][next_slot];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {   // (past the last block there are no values, and its codes will do)
        const size_t at = (size_t)min(kBlocks * next_piece + b, w.kblocks - 1) * 32;
        copy_async(&to.codes[b][0][put], from0 + at);
        copy_async(&to.codes[b][1][put], from1 + at);
      }
      if (sz_g < kGroups)
        copy_async(&to.sz[sz_g][sz_t][(lane & 3) * 2], from_sz + (size_t)min(next_piece * kGroups + sz_g, w.groups - 1) * 8);
      if (++next_slot == kCodeRing) next_slot = 0;
      skip(kSets);
    }
    copies_commit();
  };
  if (tid == 32 * kXWarp) asm volatile("prefetch.tensormap [%0];" ::"l"(&x_map) : "memory");
  // loaded weights do not change: on their way before the launch before has ended
  if (warp < kSumWarp) {
    skip(warp / 4);
    for (int i = 0; i < kCodeRing - 1; ++i) fetch();
  }
  if (tid == 0) {
    for (int i = 0; i < kPieces; ++i) {
      mbar_init(&s.full[i], Shape::kOne ? 13 : 5);   // four warps that widen, the tokens' bytes and, kOne, eight warps that sum
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 8);
    }
    for (int i = 0; i < kScaleBufs; ++i) {
      mbar_init(&s.scale_full[i], 1);
      mbar_init(&s.scale_empty[i], 8);
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
    const int g = lane >> 2, q = lane & 3, set = warp / 4;
    int slot = 0, at = set % kPieces;                    // the warp's first piece of the sequence, in the ring of pieces
    uint32_t parity = 1u ^ (uint32_t)(set / kPieces);    // of empty[at]
    const uint32_t a_at = tmem + Shape::kSlots * Shape::kColsAcc + ((uint32_t)(quarter * 32) << 16);
    for (long long left = (long long)full * pieces + (joint ? p1 - p0 : 0) - set; left > 0; left -= kSets) {
      copies_wait<kCodeRing - 2>();
      __syncwarp();
      fetch();   // (into the slot that was read last)
      const typename Shape::Codes& from = s.ring[warp][slot];
      if (++slot == kCodeRing) slot = 0;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // what rows g and g + 8 of a tile give to an MMA's columns 2q and 2q + 1 of A: ks 4q .. 4q + 3 of 16
          uint32_t made[4][4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint2 c = *((const uint2*)&from.codes[b][t][g * 4 + ((2 * e + (q >> 1)) ^ (g & 2))] + (q & 1));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint2 sz = from.sz[(2 * b + h) / GS][t][g];
              const uint32_t z0 = __byte_perm(sz.x, 0u, 0x1010), z8 = __byte_perm(sz.y, 0u, 0x1010), v = h ? c.y : c.x;
              made[2 * h + e][0] = sub_bf16x2((v & 0x000f000fu) | 0x43004300u, z0);
              made[2 * h + e][1] = sub_bf16x2((v >> 8 & 0x000f000fu) | 0x43004300u, z0);
              made[2 * h + e][2] = sub_bf16x2((v >> 4 & 0x000f000fu) | 0x43004300u, z8);
              made[2 * h + e][3] = sub_bf16x2((v >> 12 & 0x000f000fu) | 0x43004300u, z8);
            }
          }
          if (b == 0 && t == 0) {   // (the piece's place is taken only once there is something to store)
            ok = wait_for(&s.empty[at], parity);
            if (!ok) goto widened;
            tc_fence_after();
          }
          store_a(a_at + at * Shape::kColsA + b * 32 + ((uint32_t)(t * 16) << 16), made);
        }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.full[at]);
      at += kSets;
      if (at >= kPieces) at -= kPieces, parity ^= 1u;
    }
  widened:;
  } else if (warp < kXWarp) {
    constexpr int kTok = NTOK / 2;   // of a thread
    const int first = (warp - kSumWarp) / 4 * kTok;
    int at = 0, scale_at = 0;
    const int srow = quarter * 32 + lane;
    uint32_t parity = 0u, up_parity = 0u, scale_parity = 0u;
    // this row's scale of the next group (sz: row g's and row g + 8's side by side)
    const uint32_t my_scales = smem_u32(&s.scales[0][srow >> 4][(srow & 7) * 8 + (srow >> 1 & 4)]);
    uint32_t from_scale = my_scales;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    if (Shape::kOne && lane == 0)
      for (int i = 0; i < kPieces; ++i) mbar_arrive(&s.full[i]);   // (no accumulator holds anything yet)
    for (int round = 0; round < rounds && ok; ++round) {
      const int unit = unit_of(round), pieces_here = end_of(round) - first_of(round);
      float sum[kTok];
#pragma unroll
      for (int i = 0; i < kTok; ++i) sum[i] = 0.f;
      for (int piece = 0; piece < pieces_here; ++piece) {
        if (piece % (kScaleBatch / kGroups) == 0) {
          ok = wait_for(&s.scale_full[scale_at], scale_parity);
          if (!ok) break;
        }
        uint32_t scale[kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(scale[i]) : "r"(from_scale + i * 64));
        from_scale += kGroups * 64;
        const bool batch_read = (piece + 1) % (kScaleBatch / kGroups) == 0 || piece + 1 == pieces_here;
        ok = wait_for(Shape::kOne ? &s.empty[at] : &s.acc_full[at], parity);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int group = 0; group < kGroups; ++group) {
#pragma unroll
          for (int i = 0; i < kTok; i += 16) {
            uint32_t v[16];
            tmem_ld16_async(tmem + lanes + (at * kGroups + group) * NTOK + first + i, v);
            tmem_wait_ld();
            tmem_reg_fence16(v);
            if (group == kGroups - 1 && i + 16 == kTok) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(Shape::kOne ? &s.full[at] : &s.acc_empty[at]);
              if (lane == 0 && batch_read) mbar_arrive(&s.scale_empty[scale_at]);
            }
#pragma unroll
            for (int j = 0; j < 16; j += 2) fma_pair(sum[i + j], sum[i + j + 1], v[j], v[j + 1], __uint_as_float(scale[group] & 0xffff0000u));
          }
        }
        if (++at == kSlots) at = 0, parity ^= 1u;
        if (batch_read) {
          if (++scale_at == kScaleBufs) scale_at = 0, scale_parity ^= 1u;
          from_scale = my_scales + scale_at * (8 * kScalePitch);
        }
      }
      if (!ok) break;
      if (round == full) {   // (joint: the last unit, and its last MMA is done, the pieces are free)
#pragma unroll
        for (int i = 0; i < kTok; ++i) s.sums[(first + i) * kSumPitch + srow] = sum[i];
        continue;
      }
      const int m0 = unit / row_tiles * NTOK, tile = unit % row_tiles, row = tile * 128 + srow;
      const int here = min(kTok, a.M - m0 - first);   // tokens that there are
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
          for (int i = 0; i < kTok; ++i, out += a.ldo)
            if (i < here) *out = from_f32<bf16>(gelu_tanh_f(sum[i] + bias) * s.up[(first + i) * kUpPitch + srow]);
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.up_free);
        }
        up_parity ^= 1u;
      } else if (row < w.N) {
        const size_t at = (size_t)(m0 + first) * a.ldo + row;
#pragma unroll
        for (int i = 0; i < kTok; ++i) sum[i] += bias;
        if (a.epi == EPI_STORE_SILU) {
#pragma unroll
          for (int i = 0; i < kTok; ++i) sum[i] = silu_f(sum[i]);
        }
        if (a.out_bf16) {
          bf16* to = (bf16*)a.out + at;
#pragma unroll
          for (int i = 0; i < kTok; ++i, to += a.ldo)
            if (i < here) *to = from_f32<bf16>(sum[i]);
        } else if (a.epi == EPI_ADD_F32) {
          float* to = (float*)a.out + at;
#pragma unroll
          for (int i0 = 0; i0 < kTok; i0 += 4, to += (size_t)4 * a.ldo) {   // (four loads on their way at a time)
            float was[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) was[i] = i0 + i < here ? to[(size_t)i * a.ldo] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (i0 + i < here) to[(size_t)i * a.ldo] = was[i] + sum[i0 + i];
          }
        } else {
          float* to = (float*)a.out + at;
#pragma unroll
          for (int i = 0; i < kTok; ++i, to += a.ldo)
            if (i < here) *to = sum[i];
        }
      }
    }
  } else {
    if (warp == kXWarp) {
    const uint32_t el = elect_one();
    uint64_t keep;   // (every CTA reads them)
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(keep));
    int at = 0, scale_at = 0;
    uint32_t parity = 1u, scale_parity = 1u;
    long long issued = 0, batches = 0;
    for (int round = a.withhold ? rounds : 0; round < rounds && ok; ++round) {
      const int unit = unit_of(round), m0 = unit / row_tiles * NTOK, first = first_of(round), end = end_of(round);
      // (past the last tile: any that is finite; past the last group of a tile: the next one's, or zeros)
      const uint2* sz = w.sz + ((size_t)min(unit % row_tiles * 8 + (lane & 7), w.tiles - 1) * w.groups + first * kGroups) * 8;
      for (int piece = first; piece < end; ++piece) {
        const int group = (piece - first) * kGroups;
        if (group % kScaleBatch == 0) {
          ok = wait_for(&s.scale_empty[scale_at], scale_parity);
          if (!ok) break;
          mbar_expect_tx_el(&s.scale_full[scale_at], 8 * kScaleBatch * 64, el);
          __syncwarp();
          if (lane < 8)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                             smem_u32(s.scales[scale_at][lane])),
                         "l"(sz + (size_t)group * 8), "r"(kScaleBatch * 64), "r"(smem_u32(&s.scale_full[scale_at]))
                         : "memory");
          __syncwarp();
          ++batches;
          if (++scale_at == kScaleBufs) scale_at = 0, scale_parity ^= 1u;
        }
        ok = wait_for(&s.empty[at], parity);
        if (!ok) break;
        mbar_expect_tx_el(&s.full[at], kBlocks * NTOK * 128, el);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
          tma_load_2d_el(&x_map, smem_u32(&s.full[at]), smem_u32(s.pieces[at].x[b]), (piece * kBlocks + b) * 64, m0, keep, el);
        ++issued;
        if (++at == kPieces) at = 0, parity ^= 1u;
      }
    }
    // nobody leaves with loads in flight, not even where a wait ran out
    for (long long n = issued > kPieces ? issued - kPieces : 0; n < issued; ++n)
      ok = wait_for(&s.full[n % kPieces], (uint32_t)(n / kPieces) & 1u) && ok;
    for (long long n = batches > kScaleBufs ? batches - kScaleBufs : 0; n < batches; ++n)
      ok = wait_for(&s.scale_full[n % kScaleBufs], (uint32_t)(n / kScaleBufs) & 1u) && ok;
    } else if (warp == kMmaWarp) {
    const uint32_t el = elect_one();
    const uint32_t idesc = idesc_bf16(128, NTOK);
    const uint64_t xd0 = sw128_desc(smem_u32(s.pieces[0].x[0]));
    int at = 0, acc_at = 0;
    uint32_t parity = 0u, acc_parity = 1u;
    for (int round = 0; round < rounds && ok; ++round) {
      for (int left = end_of(round) - first_of(round); left > 0; --left) {
        ok = wait_for(&s.full[at], parity);
        if (!ok) break;
        if (!Shape::kOne) {
          ok = wait_for(&s.acc_empty[acc_at], acc_parity);
          if (!ok) break;
        }
        tc_fence_after();
        const uint64_t xd = xd0 + (uint32_t)(at * (sizeof(typename Shape::Piece) >> 4));
        const uint32_t td = tmem + acc_at * Shape::kColsAcc, ta = tmem + kSlots * Shape::kColsAcc + at * Shape::kColsA;
#pragma unroll
        for (int j = 0; j < 4 * kBlocks; ++j)   // 16 ks each
          umma_bf16_ts(td + j / (2 * GS) * NTOK, ta + 8 * j, xd + (j / 4) * (NTOK * 128 >> 4) + 2 * (j % 4), idesc, j % (2 * GS) > 0 ? 1u : 0u, el);
        if (!Shape::kOne) umma_commit(&s.acc_full[acc_at], el);
        umma_commit(&s.empty[at], el);
        if (++acc_at == kSlots) acc_at = 0, acc_parity ^= 1u;
        if (++at == kPieces) at = 0, parity ^= 1u;
      }
    }
    umma_commit(&s.ended, el);   // nothing is in flight when the columns are given back
    ok = wait_for(&s.ended, 0u) && ok;
  }
  }
  copies_wait<0>();
  if (!ok && lane == 0) raise_error(a.err, ERR_TIMEOUT);
  if (joint) {
    cluster_sync();
    const int m0 = last_unit / row_tiles * NTOK, tile = last_unit % row_tiles, tokens = min(NTOK, a.M - m0);
    // a warp per token: four of its rows' sums to a lane, of all ranks in their order (the loads on their way together)
    for (int m = tokens * rank / ranks + warp; m < tokens * (rank + 1) / ranks; m += kTcThreads / 32) {
      float x[kRanks][4], v[4];
#pragma unroll
      for (int i = 0; i < kRanks; ++i)
        if (i < ranks) {
          const uint32_t from = mapa_shared(smem_u32(&s.sums[m * kSumPitch + lane]), (uint32_t)i);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = ld_cluster_f(from + 128 * j);
        }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = x[0][j];
#pragma unroll
        for (int i = 1; i < kRanks; ++i)
          if (i < ranks) v[j] += x[i][j];
        const int n = tile * 128 + lane + 32 * j;
        if (a.bias && n < w.N) v[j] += a.bias[n];
      }
      if (a.epi == EPI_GEGLU) {
        bf16* to = (bf16*)a.out + (size_t)(m0 + m) * a.ldo + tile * 64 + lane;
        to[0] = from_f32<bf16>(gelu_tanh_f(v[0]) * v[2]);
        to[32] = from_f32<bf16>(gelu_tanh_f(v[1]) * v[3]);
        continue;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = tile * 128 + lane + 32 * j;
        if (row >= w.N) continue;
        const size_t to = (size_t)(m0 + m) * a.ldo + row;
        if (a.epi == EPI_STORE_SILU) v[j] = silu_f(v[j]);
        if (a.epi == EPI_ADD_F32) ((float*)a.out)[to] += v[j];
        else if (a.out_bf16) ((bf16*)a.out)[to] = from_f32<bf16>(v[j]);
        else ((float*)a.out)[to] = v[j];
      }
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
  // (a set's last wait was kSets pieces ago; the round before the one that it waits for now has to have ended by then, for a
  // barrier's parity does not tell a round from the second next one)
  static_assert(TcShape<NTOK, GS>::kPieces >= kSets, "places");
  static_assert(TcShape<NTOK, GS>::kPieces * TcShape<NTOK, GS>::kColsA + TcShape<NTOK, GS>::kSlots * TcShape<NTOK, GS>::kColsAcc <= (int)kTcCols, "tensor memory");
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
  const W4TcPlan plan(a, NTOK);
  const Overlap overlap;
  return launch_kernel_cluster(w4_tc_kernel<NTOK, GS>, dim3(plan.grid), dim3(kTcThreads), kTcSmem, st, dim3(plan.ranks, 1, 1), map, a, plan.ranks);
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
  W4Args b = a;
  b.withhold = w4_withheld() > 0 && w4_withheld()-- > 0;
  return w4_tc_tokens(a.M) == 32 ? launch_ntok<32>(b, st) : launch_ntok<64>(b, st);
}

}  // namespace ravel
