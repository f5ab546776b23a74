// Attention over the 8-bit context cache for many query rows (an expert's slots,
// prompts), bf16, on the 5th-generation tensor cores.
//
// An item is 128 rows (row r = query * G + head of the group) of one (robot, KV
// head) and a share (split) of the 128-token tiles that they see; CTAs, one per SM,
// walk the items of their launch:
//   S = Q K^T        tcgen05.mma kind::f8f6f4, M = 128, N = 128, into TMEM: the codes
//                    of K as they are, Q in two 8-bit pieces
//   P = 2^(S - m)    softmax warps: TMEM -> registers -> f16 P over S in TMEM
//   O += P V         tcgen05.mma kind::f16, M = 128, N = head dim, 16 tokens at a time
// Warp roles (640 threads): warps 0-7 softmax and output (see TcShape::own); warps
// 8-11 lay out the next item's Q, warps 12-15 widen V; warp 16 TMEM and MMAs; warps 17, 18 load the
// codes of K and V (19 idle, so that registers move between whole warpgroups).
// Every role walks the items on its own, so that one item's output lies beside the
// next one's Q, K and first scores.
//
// What bounds it at head dim 256 is shared memory: per tile (2048 cycles of MMA) its
// 128 bytes a cycle carry 192 KB of MMA operands, and every code that is widened to
// f16 costs 4 bytes more of TMA, reading and writing.  So K is not widened: bf16's 8
// significant bits are 4 in e4m3 and the rest in e5m2 (see stage_q8: exactly, down to
// 2^-13 of the row's largest, and within 2^-21 of it below), whose two MMAs at twice the
// rate cost what one in f16 does.  V is: 2^-9 is the least P that e4m3 holds, and a long flat tail
// of smaller ones carries weight.  The codes of V come by TMA and are widened in
// shared memory to f16 (exact), into the 128-byte swizzled layout of a TMA load of
// f16 rows.  (Widening K as well, in units of 64 head dims, 448 KB a tile, took 3600
// to 4400 cycles; with the codes loaded to registers by the widening warps a step
// took a load's latency, as the proxy fence that ends it waits for the loads in
// flight.)
//
// Numbers as in the kernel for few rows: a power of two per row of Q, block exponents
// of K on the scores, those of V on P.  P is at most 2^7 of the reference, 2^15 while
// a grown one waits for its rescaling of O (only growth by more than 2^8 rescales);
// what contributes less than 2^-31 of the row's largest is dropped.
//
// Measured: 16 prompts of 816 tokens (8 heads of 256, one KV head) 88.5 us, 985 TFLOP/s
// (causal 71); 2 of 8191 with a window of 1024 (16 heads of 64) 193 us, without the window
// 425; 50 slots of 16 robots over 816 tokens, 20 us.  A tile of 128 x 128 takes 1570 cycles at head dim 64, 1940
// at 128, 2190 at 192 and 2550 at 256 (MMAs alone: 512, 1024, 1536, 2048), an item's begin and
// end 7500 to 12000 more.  Up to 128 the softmax bounds it; of a tile that two threads a row
// share, one after the other: scores in 130, maxima 250, their exchange 250, exponentials 700,
// P out, the wait for the next scores; at 256 that chain beside the widening's share of
// shared memory (without MMAs and widening 2220).
#include <algorithm>

#include "cache_index.h"
#include "cache_tc.cuh"
#include "launch.h"

namespace ravel {
namespace {

constexpr int TCT = 640;
constexpr uint32_t CB = 64 * 64;               // bytes of a slot of V's codes: 64 tokens x 64 dims
constexpr uint32_t VB = 64 * 128;              // bytes of a 64-dim block of a V half
constexpr float kTcShift = 7.f;                // P's largest value is 2^kTcShift (times 2^8 while lazy)
constexpr int kTcCluster = 8;                  // splits that are a cluster

template <int NB> struct TcShape {
  // shared memory at NB blocks of 64 head dims: Q's pieces, the rings of K units, of widened
  // V halves and of V's codes, barriers and row data
  static constexpr int KS = NB == 4 ? 4 : 8;
  static constexpr int VS = NB >= 3 ? 3 : (NB == 2 ? 4 : 8);
  // a multiple of the 4 warps that widen them: each slot is then waited for by one warp, in
  // order.  (Loads may complete out of order; a warp that waits for a slot's next phase while
  // another's load into it is still on its way would take the phase before for it.)
  static constexpr int CV = 8;
  static_assert(CV % 4 == 0, "widening warps");
  // (a half's slot is waited for by whichever warp comes to it: one that has codes for it knows
  // that the slot's half before has begun, which was past that wait)
  static_assert(CV <= VS * NB, "widening ahead");
  static constexpr uint32_t q_bytes = 2 * NB * QB;
  static constexpr uint32_t ring = KS * KU + VS * NB * VB + CV * CB;
  // Up to head dim 64 TMEM holds three tiles of scores and two outputs: each softmax
  // warpgroup takes every second tile, a thread a row, with references and an output of its
  // own, joined at the item's end, so that one's waits lie beside the other's work: 1570
  // cycles a tile instead of 1780 (2 causal prompts of 8191: 424 us instead of 479; with a
  // window of 1024, of whose ten tiles three are masked, twice then, 193 instead of 199).  Beyond,
  // both share a tile, two threads to a row: with the two buffers of scores that fit at 128,
  // a P's way to the scores of the tile after next, 1450 cycles, ate the gain.
  static constexpr bool own = NB == 1;
  static constexpr int SB = own ? 3 : 2;   // buffers of scores
  // places for the halves' maxima: in turn where there is room, which saves a barrier a tile
  static constexpr int XM = NB == 4 ? 1 : 2;
  static constexpr uint32_t bars = own ? 640 : 512;   // bytes of barriers and flags
  static constexpr uint32_t bytes = q_bytes + ring + bars + 512 + XM * 2048;
  static_assert(bytes <= 227 * 1024, "shared memory");
  // a row of the fp32 output that splits exchange (over the rings): 16 bytes more than
  // the dims, so that rows written by neighbouring lanes fall on different banks
  static constexpr uint32_t xrow = NB * 64 * 4 + 16;
  static_assert(BM * xrow <= ring && BM * 4 * 256 <= ring && BM * 4 * 8 <= q_bytes, "exchange");
};

struct TcMaps {
  CUtensorMap k, v;   // a layer's codes [B Hkv T][hdp]: boxes of 64 dims x 128 rows (swizzled), x 64 rows
};

// 16 codes -> two 16-byte pieces of f16
__device__ __forceinline__ void widen(uint4 w, uint32_t lo, uint32_t hi) {
  sts_u4(lo, make_uint4(e4m3_lo(w.x), e4m3_hi(w.x), e4m3_lo(w.y), e4m3_hi(w.y)));
  sts_u4(hi, make_uint4(e4m3_lo(w.z), e4m3_hi(w.z), e4m3_lo(w.w), e4m3_hi(w.w)));
}

__device__ __forceinline__ void store_bf16x8(bf16* dst, uint4 w, bool wide) {
  if (wide) {
    *(uint4*)dst = w;
  } else {
    bf16 y[8];
    memcpy(y, &w, 16);
#pragma unroll
    for (int z = 0; z < 8; ++z) dst[z] = y[z];
  }
}

// Registers of a warpgroup: launched with 96 each (640 x 96 = 61440); softmax
// 2 x 128 x 136, Q and widening 2 x 128 x 80, the rest 128 x 48: 61440.
template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Item w of a launch: its (robot, KV head), row tile, split, and the tiles of tokens
// that it walks.
struct Item {
  int head, b, h, tile, split;
  Sight s;
  bool ok, live;     // the robot's numbers are in range; some row sees something
  int t0, n;         // tiles t0 .. t0 + n - 1 of the sight's units
  int hi;            // tokens from here on are nobody's
  __device__ __forceinline__ int token(int i) const {
    return unit_place(t0 + i, s.sink_units, s.from) * BT;
  }
  // tokens of tile i that exist for these rows, in groups of 16
  __device__ __forceinline__ int groups(int i) const { return (min(BT, hi - token(i)) + 15) >> 4; }
  __device__ __forceinline__ int halves() const { return n == 0 ? 0 : 2 * n - (groups(n - 1) > 4 ? 0 : 1); }
};

// Items are ordered by groups of a.group (robot, KV head) pairs whose caches stay in L2
// together, within a group by row tile from the last one on (causal: the longest first,
// so that the CTAs' shares even out), then by split.
__device__ __forceinline__ Item item_of(const CacheAttnArgs& a, int w) {
  Item it;
  const uint32_t x = a.by_splits.of((uint32_t)w);
  it.split = w - (int)x * a.splits;
  const uint32_t gi = a.by_group.of(x), rem = x - gi * a.by_group.d;
  const bool whole = ((int)gi + 1) * a.group <= a.batch * a.c.Hkv;
  const uint32_t pairs = whole ? a.by_pairs.d : a.by_last.d, row = whole ? a.by_pairs.of(rem) : a.by_last.of(rem);
  it.tile = a.row_tiles - 1 - (int)row;
  it.head = (int)(gi * a.group + rem - row * pairs);
  it.b = (int)a.by_heads.of((uint32_t)it.head);
  it.h = it.head - it.b * a.c.Hkv;
  it.ok = robot_sight(a, it.b, it.s);
  it.live = it.tile * BM < it.s.count * a.G && it.s.len > 0;
  it.t0 = it.n = it.hi = 0;
  if (it.live) {
    tile_sight(a, it.s, it.tile * BM, it.tile * BM + BM - 1, BT);
    it.hi = row_mask(a, it.s, min(it.tile * BM + BM, it.s.count * a.G) - 1).hi;
    // units * split / splits, and the same of the next split
    const uint32_t each = a.by_splits.of((uint32_t)it.s.units), more = (uint32_t)it.s.units - each * a.by_splits.d;
    it.t0 = (int)(each * it.split + a.by_splits.of(more * it.split));
    it.n = (int)(each * (it.split + 1) + a.by_splits.of(more * (it.split + 1))) - it.t0;
  }
  return it;
}

template <int NB>
__global__ void __launch_bounds__(TCT, 1) cache_tc_kernel(const __grid_constant__ TcMaps maps, CacheAttnArgs a) {
  using Shape = TcShape<NB>;
  constexpr int HDP = 64 * NB, KS = Shape::KS, VS = Shape::VS, CV = Shape::CV, SB = Shape::SB;
  constexpr uint32_t VH = NB * VB;   // bytes of a V half
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t q0 = smem_u32(smem), k0 = q0 + Shape::q_bytes, v0 = k0 + KS * KU, cv0 = v0 + VS * VH;
  uint8_t* tail = smem + Shape::q_bytes + Shape::ring;
  uint64_t* k_full = (uint64_t*)tail;
  uint64_t* k_empty = k_full + KS;
  uint64_t* v_full = k_empty + KS;
  uint64_t* v_empty = v_full + VS;
  uint64_t* cv_full = v_empty + VS;
  uint64_t* cv_empty = cv_full + CV;
  uint64_t* s_full = cv_empty + CV;   // [SB]
  uint64_t* p_full = s_full + SB;     // [SB]
  uint64_t* pv_done = p_full + SB;    // [SB]
  uint64_t* q_full = pv_done + SB;    // an item's Q is laid out ...
  uint64_t* q_empty = q_full + 1;     // ... and its last S has completed
  uint64_t* o_free = q_empty + 1;     // an item's output has been read
  uint64_t* q_laid = o_free + 1;      // an item's Q is laid out in L2
  uint64_t* ended = q_laid + 1;
  uint32_t* tmem_slot = (uint32_t*)(ended + 1);
  int* abort_flag = (int*)(tmem_slot + 1);
  int* last_flag = abort_flag + 1;
  int* issued_flag = last_flag + 1;               // [3] loads of K, V and Q issued
  // exponent bits of the rows' largest |q|, [4][128], by item: S runs up to two tiles, so up
  // to two items, ahead of the softmax, and Q one more
  uint8_t* row_exp = tail + Shape::bars;
  float2* xm = (float2*)(row_exp + 512);   // [XM][2][128] row maxima, then sums, of the two halves
  static_assert((2 * KS + 2 * VS + 2 * CV + 3 * SB + 5) * 8 + 24 <= Shape::bars, "barriers");

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const CacheLayer& L = a.c;
  const int items = a.row_tiles * a.splits * L.Hkv * a.batch;
  pdl_wait();   // (before any TMEM is taken: the launch before may still need it)
  if (q0 & 1023u) {   // (the swizzled layouts count on it)
    if (threadIdx.x == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < KS; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < VS; ++i) {
      mbar_init(&v_full[i], NB);   // the steps of a half
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < CV; ++i) {
      mbar_init(&cv_full[i], 1);
      mbar_init(&cv_empty[i], 1);
    }
    issued_flag[0] = issued_flag[1] = 0;
    for (int i = 0; i < SB; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], Shape::own ? 128 : 256);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    mbar_init(q_laid, 4);
    issued_flag[2] = 0;
    mbar_init(o_free, 8);
    mbar_init(ended, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  pdl_trigger();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t o_col = SB * BT;
  static_assert(o_col + (Shape::own ? 2 : 1) * HDP <= 512, "TMEM");

  auto stage = [&](const Item& it, int rb, int qi, uint8_t* to) {
    stage_q8<NB>(a, it.s, it.b, it.h, it.tile * BM, rb, q0, to, [&](int lr, int e) { row_exp[(qi & 3) * BM + lr] = (uint8_t)e; });
  };
  // the first item's Q, by all warps that have nothing else to do yet
  if (warp < 16) {
    for (int w = blockIdx.x; w < items; w += gridDim.x) {
      const Item it = item_of(a, w);
      if (it.n == 0) continue;
      stage(it, 8 * warp, 0, nullptr);
      break;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("bar.arrive 6, 544;" ::: "memory");   // (with warp 16)
  }

  if (warp >= 8 && warp < 12) {
    regs_down<80>();
    // ---- Q of the items after the first: into the CTA's place in L2 while the item before is
    // at work, from there into shared memory in one copy as soon as its last S has completed.
    // (Into shared memory directly, at that time, the rows' 100 instructions each left the
    // tensor core without Q for 15000 cycles an item.)
    uint8_t* place = a.q_ws + (size_t)blockIdx.x * Shape::q_bytes;
    int qi = 0;   // items so far
    bool ok = true;
    for (int w = blockIdx.x; ok && w < items; w += gridDim.x) {
      const Item it = item_of(a, w);
      if (it.n == 0) continue;
      if (qi > 0) {
        if (qi > 1) ok = wait_phase(q_full, (uint32_t)qi & 1u);   // the item before's copy has been read
        if (!ok) break;
#pragma unroll 1
        for (int rb = 0; rb < 32; rb += 8) stage(it, (warp - 8) * 32 + rb, qi, place);
        __threadfence();
        asm volatile("fence.proxy.async;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(q_laid);
        if (warp == 8) {
          ok = wait_phase(q_laid, (uint32_t)(qi - 1) & 1u) && wait_phase(q_empty, (uint32_t)(qi - 1) & 1u);
          if (ok && lane == 0) {
            mbar_expect_tx(q_full, Shape::q_bytes);
            asm volatile(
                "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(q0),
                "l"(place), "r"(Shape::q_bytes), "r"(smem_u32(q_full))
                : "memory");
            issued_flag[2] = qi;
          }
          __syncwarp();
        }
      }
      ++qi;
    }
    if (!ok && lane == 0) *abort_flag = 1;
  } else if (warp >= 12 && warp < 16) {
    regs_down<80>();
    // ---- widening of V: halves of 64 tokens, in steps of 64 tokens x 64 dims.  A warp takes every fourth step
    // as a whole, so that the waits, the proxy fence and the shared-memory latency of one lie
    // beside the work on the others.  Lane: 16 codes at dim 16 (lane % 4) of rows lane / 4,
    // lane / 4 + 8, ...
    const uint32_t sw = (uint32_t)(lane >> 2), row = (uint32_t)(lane >> 2) * 128u;
    const uint32_t lo = row + ((((uint32_t)lane & 3u) * 2u) ^ sw) * 16u, hi = row + ((((uint32_t)lane & 3u) * 2u + 1u) ^ sw) * 16u;
    int u = warp - 12, end = 0;   // this warp's next step, the steps so far
    bool ok = true;
    for (int w = blockIdx.x; ok && w < items; w += gridDim.x) {
      end += item_of(a, w).halves() * NB;
      for (; u < end; u += 4) {
        const int cs = u % CV, part = u / NB, slot = part % VS;
        ok = wait_phase(&cv_full[cs], (uint32_t)(u / CV) & 1u);
        if (!ok) break;
        uint4 x[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) x[y] = lds_u4(cv0 + (uint32_t)cs * CB + 16u * lane + 512u * y);
        ok = wait_phase(&v_empty[slot], ((uint32_t)(part / VS) & 1u) ^ 1u);
        if (!ok) break;
        const uint32_t to = v0 + (uint32_t)slot * VH + (uint32_t)(u % NB) * VB;
#pragma unroll
        for (int y = 0; y < 8; ++y) widen(x[y], to + lo + 1024u * y, to + hi + 1024u * y);
        written(&v_full[slot]);
        // the codes' slot is free only here, with their use: an arrival right behind the loads is
        // seen before the loads are done when copies fill shared memory (the next item's Q)
        if (lane == 0) mbar_arrive(&cv_empty[cs]);
      }
    }
    if (!ok && lane == 0) *abort_flag = 1;
  } else if (warp >= 16) {
    regs_down<48>();
    if (warp == 16) {
      // ---- MMAs, in the order S 0, S 1, P V 0, S 2, P V 1, S 3, ...: two tiles of scores in
      // flight, into the next item where this one ends
      const uint32_t el = elect_one();
      const uint32_t idesc_s = idesc_f16(BM, BT), idesc_o = idesc_f16(BM, HDP) | (1u << 16);
      const uint64_t qd0 = sw64_desc(q0), kd0 = sw64_desc(k0), vd0 = sw128_mn_desc(v0, VB);
      // the items with tiles, in order: tiles and the last one's groups of 16 tokens, 0 behind the
      // last item.  The next one is looked up while there is nothing to issue; lane q % 32 keeps
      // item q's for P V, up to two items behind S.
      int ws = blockIdx.x, ahead = 0, kept = 0;
      bool looked = false;
      auto look = [&]() {
        ahead = 0;
        looked = true;
        for (; ws < items && ahead == 0; ws += gridDim.x) {
          const Item it = item_of(a, ws);
          const int n = uniform(it.n);
          if (n > 0) ahead = n << 4 | uniform(it.groups(n - 1));
        }
      };
      int sn = 0, pn = 0, last = 0;                   // tiles of S's and P V's items
      int si = 0, pi = 0, sq = 0, pq = 0;             // tiles done of them; items begun
      int gs = 0, gp = 0;                             // tiles in all
      int sk = 0, sv = 0, bs = 0, bp = 0;             // slots; buffers of scores
      uint32_t phk = 0, phv = 0, php = 0;
      bool ok = true;
      asm volatile("bar.sync 6, 544;" ::: "memory");
      look();
      looked = false;
      kept = ahead;
      sn = pn = ahead >> 4;
      last = ahead & 15;
      while (pn > 0) {
        while (sn > 0 && gs < gp + SB) {
          if (si == 0) {
            // an item's last P V goes first: its output is what the softmax does next
            if (gs > gp) break;
            if (sq > 0) ok = wait_phase(q_full, (uint32_t)(sq - 1) & 1u);   // (the first item's came through barrier 6)
          }
          if (ok) {   // the tile's K units
            auto unit = [&](int x) { return sk + x < KS ? sk + x : sk + x - KS; };
            auto par = [&](int x) { return sk + x < KS ? phk : phk ^ 1u; };
            constexpr int u1 = NB > 1 ? 1 : 0, u2 = NB > 2 ? 2 : 0, u3 = NB > 3 ? 3 : 0;
            ok = NB == 1 ? wait_phase(&k_full[sk], phk)
                         : wait_phases(&k_full[sk], phk, &k_full[unit(u1)], par(u1), &k_full[unit(u2)], par(u2), &k_full[unit(u3)],
                                       par(u3));
          }
          if (!ok) break;
          tc_fence_after();
          const uint32_t sd = tmem + (uint32_t)bs * BT;
          uint64_t ad = qd0;
#pragma unroll 1
          for (int blk = 0; blk < NB; ++blk, ad += QB >> 4) {
            const uint64_t bd = kd0 + (uint32_t)sk * (KU >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)   // both pieces of Q
              umma_f8(sd, ad + (k >> 1) * (NB * QB >> 4) + 2 * (k & 1), bd + 2 * (k & 1), k < 2 ? idesc_s : idesc_s | kE5m2A, (blk > 0 || k > 0) ? 1u : 0u, el);
            umma_commit(&k_empty[sk], el);
            if (++sk == KS) {
              sk = 0;
              phk ^= 1u;
            }
          }
          umma_commit(&s_full[bs], el);
          ++gs;
          if (++bs == SB) bs = 0;
          if (++si == sn) {
            umma_commit(q_empty, el);
            si = 0;
            ++sq;
            if (!looked) look();
            looked = false;
            sn = ahead >> 4;
            if (lane == (sq & 31)) kept = ahead;
          }
        }
        if (!looked && pi == 0) look();   // (the softmax is at the output of the item before)
        const uint32_t pa = tmem + (uint32_t)bp * BT, od = tmem + o_col + (Shape::own ? (uint32_t)(gp & 1) * HDP : 0u);
        const int groups = pi + 1 < pn ? BT / 16 : last;
        if (ok) {   // P, the first half of V (both, where several tiles' lie in the ring), a free O
          const bool two = NB <= 2 && groups > 4, first = pi == 0 && pq > 0;
          const int s = two ? (sv + 1 < VS ? sv + 1 : 0) : sv;
          ok = wait_phases(&p_full[bp], php, &v_full[sv], phv, &v_full[s], s < sv ? phv ^ 1u : phv,
                           first ? o_free : &v_full[sv], first ? (uint32_t)(pq - 1) & 1u : phv);
        }
        if (!ok) break;
        tc_fence_after();
#pragma unroll 1
        for (int hv = 0; 4 * hv < groups; ++hv) {
          if (NB > 2 && hv > 0) {
            ok = wait_phase(&v_full[sv], phv);
            if (!ok) break;
            tc_fence_after();
          }
          const uint64_t bd = vd0 + (uint32_t)sv * (VH >> 4);
          const uint32_t ph = pa + 32 * hv, more = hv > 0 || pi > (Shape::own ? 1 : 0) ? 1u : 0u;
          if (groups >= 4 * hv + 4) {   // (a comparison and a branch per MMA take longer than the MMA)
#pragma unroll
            for (int k = 0; k < 4; ++k) umma_bf16_ts(od, ph + 8 * k, bd + 128 * k, idesc_o, k > 0 ? 1u : more, el);
          } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
              if (4 * hv + k < groups) umma_bf16_ts(od, ph + 8 * k, bd + 128 * k, idesc_o, k > 0 ? 1u : more, el);
          }
          umma_commit(&v_empty[sv], el);
          if (++sv == VS) {
            sv = 0;
            phv ^= 1u;
          }
        }
        if (!ok) break;
        umma_commit(&pv_done[bp], el);
        ++gp;
        if (++bp == SB) {
          bp = 0;
          php ^= 1u;
        }
        if (++pi == pn) {
          pi = 0;
          ++pq;
          const int x = __shfl_sync(0xffffffffu, kept, pq & 31);   // (S has come to it)
          pn = x >> 4;
          last = x & 15;
        }
      }
      if (!ok) {   // what was issued ends before the TMEM goes away
        umma_commit(ended, el);
        wait_phase(ended, 0);
        if (lane == 0) *abort_flag = 1;
      }
      __syncwarp();
    } else if (warp < 19) {
      // ---- the codes' loads
      const uint32_t el = elect_one();
      const bool is_k = warp == 17;
      const int ring = is_k ? KS : CV;
      uint64_t *full = is_k ? k_full : cv_full, *empty = is_k ? k_empty : cv_empty;
      uint64_t pol;
      asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
      int slot = 0, issued = 0;
      uint32_t ph = 1;
      bool ok = true;
      for (int w = blockIdx.x; ok && w < items; w += gridDim.x) {
        const Item it = item_of(a, w);
        const int y0 = it.head * L.T, n = uniform(it.n);
        // a (robot, KV head)'s codes come to L2 as its first items begin, up to 256 KB of them
        // (its row tiles ask for the same lines at the same time); of a window behind sinks the
        // longer of the two, as a rule the window
        if (it.n > 0 && (it.tile & 7) == 0 && el) {
          const UnitRun run = longest_run(it.t0, it.n, it.s.sink_units, it.s.from);
          const size_t from = ((size_t)y0 + (size_t)run.at * BT) * HDP;
          prefetch_l2_bulk((is_k ? L.k : L.v) + from, (uint32_t)min((size_t)run.units * BT * HDP, (size_t)(256 << 10)));
        }
        // K: a tile's units of 64 dims; V: its halves of 64 tokens, each NB blocks of 64 dims
        const int halves = uniform(it.halves());
        for (int i = 0; ok && i < n; ++i) {
          const int j0 = uniform(y0 + it.token(i)), steps = NB * (is_k ? 1 : min(2, halves - 2 * i));
          for (int q = 0; q < steps; ++q) {
            ok = wait_phase(&empty[slot], ph);
            if (!ok) break;
            if (is_k) {
              mbar_expect_tx_el(&full[slot], KU, el);
              tma_load_2d_el(&maps.k, smem_u32(&full[slot]), k0 + (uint32_t)slot * KU, 64 * q, j0, pol, el);
            } else {
              mbar_expect_tx_el(&full[slot], CB, el);
              tma_load_2d_el(&maps.v, smem_u32(&full[slot]), cv0 + (uint32_t)slot * CB, 64 * (q % NB), j0 + 64 * (q / NB), pol, el);
            }
            ++issued;
            if (++slot == ring) {
              slot = 0;
              ph ^= 1u;
            }
          }
        }
      }
      if (lane == 0) {
        issued_flag[is_k ? 0 : 1] = issued;
        if (!ok) *abort_flag = 1;
      }
      __syncwarp();
    }
  } else {
    regs_up<136>();
    // ---- softmax and output: row r (TMEM lane r), tokens 64 hf .. of each tile
    const int q4 = warp & 3, hf = warp >> 2, r = q4 * 32 + lane;
    auto pair_bar = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + q4) : "memory"); };   // warps w and w + 4
    const uint32_t lane_base = tmem + ((uint32_t)(q4 * 32) << 16);
    const uintptr_t places = (uintptr_t)a.out | (uintptr_t)(a.out_robot * 2) | (uintptr_t)(a.out_token * 2);
    const bool wide = places % 16 == 0;
    bool ok = true;   // (after a wait that ran out the loops go on without waiting, so that pairs meet at every barrier)
    int gt = 0, qi = 0;   // tiles and items with Q so far
    Item coming = item_of(a, blockIdx.x);
    for (int w = blockIdx.x; w < items; w += gridDim.x) {
      const Item it = coming;
      const int after = min(w + (int)gridDim.x, items - 1);   // (looked up where the tensor core is waited for)
      const int r0 = it.tile * BM, rows = min(BM, a.n * a.G - r0), n = it.n;
      const size_t head = it.head;
      bf16* out0 = (bf16*)a.out + (size_t)((long long)it.b * a.out_robot) + (size_t)it.h * a.G * L.hd;
      auto out_row = [&](int lr) {
        const uint32_t x = (uint32_t)(r0 + lr), i = a.by_G.of(x);
        return out0 + (size_t)((long long)i * a.out_token) + (size_t)(x - i * (uint32_t)a.G) * L.hd;
      };
      if (!it.ok && it.tile == 0 && it.h == 0 && it.split == 0 && threadIdx.x == 0) raise_error(a.err, ERR_SHAPE);
      if (!it.live) {   // nothing to see: zeros
        if (it.split == 0) {
          for (int x = threadIdx.x; x < rows * L.hd; x += 256) out_row(x / L.hd)[x % L.hd] = __float2bfloat16_rn(0.f);
          if (a.mass && (int)threadIdx.x < rows) a.row_ml[head * a.n * a.G + r0 + threadIdx.x] = make_float2(0.f, 0.f);
        }
        coming = item_of(a, after);
        continue;
      }
      const RowMask mk = row_mask(a, it.s, r0 + r);
      const RowMask firstm = row_mask(a, it.s, r0), lastm = row_mask(a, it.s, min(r0 + BM, it.s.count * a.G) - 1);
      float rf = 0.f;
      const int8_t *KE = L.ke + head * (L.T / 16), *VE = L.ve + head * (L.T / 16);
      // references in the log2 domain, integral: m of the row's sum, W of O (largest score + value exponent)
      float m = -INFINITY, W = -INFINITY, l = 0.f;
      // 64 of a tile's scores from the row's column `at` on, token j the first; hidden ones -inf
      auto scores = [&](uint32_t at, int j, bool full, float (&sc)[64]) {
        uint32_t raw[64];
#pragma unroll
        for (int q = 0; q < 64; q += 16) tmem_ld16_async(at + q, raw + q);
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < 64; q += 16) tmem_reg_fence16(raw + q);
#pragma unroll
        for (int k = 0; k < 64; ++k) sc[k] = __uint_as_float(raw[k]);
        if (!full) {
#pragma unroll
          for (int k2 = 0; k2 < 64; k2 += 32) {
            const uint32_t see = mk.bits(j + k2);
#pragma unroll
            for (int k = 0; k < 32; ++k) sc[k2 + k] = see >> k & 1u ? sc[k2 + k] : -INFINITY;
          }
        }
      };
      // a block's factor (not 0, which times a hidden score's -inf would not be a number)
      auto factor = [&](uint32_t kes, int t) { return fmaxf(rf * exp2i((int)(int8_t)(kes >> (8 * t))), 1e-37f); };
      // their largest score and largest score + value exponent
      auto maxima = [&](const float (&sc)[64], uint32_t kes, uint32_t ves, float& mx, float& wx) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float m5[5];
#pragma unroll
          for (int e = 0; e < 5; ++e) m5[e] = max3(sc[16 * t + 3 * e], sc[16 * t + 3 * e + 1], sc[16 * t + 3 * e + 2]);
          const float x = fmaxf(max3(m5[0], m5[1], m5[2]), max3(m5[3], m5[4], sc[16 * t + 15])) * factor(kes, t);
          mx = fmaxf(mx, x);
          wx = fmaxf(wx, x + (float)(int8_t)(ves >> (8 * t)));
        }
      };
      // their weights into P at `to`, and into the row's sum
      auto weights = [&](const float (&sc)[64], uint32_t kes, uint32_t ves, float mu, float wu, uint32_t to) {
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
          uint32_t wd[16];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int blk = 2 * h2 + t;
            // the value exponent goes into that of P and out of the block's sum again
            const float vf = fmaxf((float)(int8_t)(ves >> (8 * blk)), wu - mu - kVeBelow), nbt = kTcShift + vf - wu;
            const float f = factor(kes, blk);
            float2 e[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              e[q] = fma2(make_float2(sc[16 * blk + 2 * q], sc[16 * blk + 2 * q + 1]), make_float2(f, f), make_float2(nbt, nbt));
              e[q] = make_float2(fast_exp2(e[q].x), fast_exp2(e[q].y));
              wd[8 * t + q] = pack_f16x2(e[q].x, e[q].y);
            }
            const float2 s = add2(add2(add2(e[0], e[1]), add2(e[2], e[3])), add2(add2(e[4], e[5]), add2(e[6], e[7])));
            l = fmaf(s.x + s.y, pow2f(wu - mu - vf), l);
          }
          tmem_st16u(to + 16 * h2, wd);
        }
      };
      // new references; where W rises by much, O, which holds P V of the earlier tiles (or every
      // second one) once that of tile g has completed, is rescaled
      auto refer = [&](float mx, float wx, bool any, int g, float& mu, float& wu) {
        const float mn = fmaxf(m, ceilf(mx)), wn = fmaxf(W, ceilf(wx));
        mu = mn == -INFINITY ? 0.f : mn;
        l *= pow2f_down(m - mu);
        m = mn;
        const bool need = wn > W + 8.f;
        if (any && __any_sync(0xffffffffu, need)) {
          if (ok) ok = wait_phase(&pv_done[g % SB], (uint32_t)(g / SB) & 1u);
          tc_fence_after();
          const float alpha = need ? pow2f_down(W - wn) : 1.f;
          constexpr int NC = Shape::own ? 64 : 16;   // columns at a time (a shared tile's scores are held meanwhile)
#pragma unroll 1
          for (int cb = Shape::own ? hf * HDP : 16 * hf; cb < (Shape::own ? (hf + 1) * HDP : HDP); cb += Shape::own ? NC : 32) {
            uint32_t o[NC];
#pragma unroll
            for (int q = 0; q < NC; q += 16) tmem_ld16_async(lane_base + o_col + cb + q, o + q);
            tmem_wait_ld();
#pragma unroll
            for (int q = 0; q < NC; q += 16) {
              tmem_reg_fence16(o + q);
#pragma unroll
              for (int x = 0; x < 16; ++x) o[q + x] = __float_as_uint(__uint_as_float(o[q + x]) * alpha);
              tmem_st16u(lane_base + o_col + cb + q, o + q);
            }
          }
          tmem_wait_st();
        }
        if (need) W = wn;
        wu = W == -INFINITY ? 0.f : W;
      };
      if constexpr (Shape::own) {
        const int i0 = (gt ^ hf) & 1;   // this warpgroup's first tile
#pragma unroll 1
        for (int i = i0; i < n; i += 2) {
          const int j0 = it.token(i), g = gt + i, bs = g % SB;
          const uint2 ke = *(const uint2*)(KE + j0 / 16), ve = *(const uint2*)(VE + j0 / 16);   // exponents of its blocks
          const bool full = j0 + BT <= firstm.hi && (j0 >= lastm.lo || j0 + BT <= a.sinks);
          if (ok) ok = wait_phase(&s_full[bs], (uint32_t)(g / SB) & 1u);
          tc_fence_after();
          if (i == i0) rf = q_factor(row_exp[(qi & 3) * BM + r], a.scale_log2);   // (S needed Q: it is there)
          const uint32_t srow = lane_base + (uint32_t)bs * BT;
          float mx = -INFINITY, wx = -INFINITY, mu, wu;
#pragma unroll 1
          for (int c = 0; c < BT; c += 64) {
            float sc[64];
            scores(srow + c, j0 + c, full, sc);
            maxima(sc, c ? ke.y : ke.x, c ? ve.y : ve.x, mx, wx);
          }
          refer(mx, wx, i >= 2, g - 2, mu, wu);
          // (P goes over scores that have been read again by then)
#pragma unroll 1
          for (int c = 0; c < BT; c += 64) {
            float sc[64];
            scores(srow + c, j0 + c, full, sc);
            weights(sc, c ? ke.y : ke.x, c ? ve.y : ve.x, mu, wu, srow + c / 2);
          }
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(&p_full[bs]);
        }
        gt += n;
      } else {
        for (int i = 0; i < n; ++i, ++gt) {
          const int j0 = it.token(i);
          // exponents of this half's four blocks
          const uint32_t kes = *(const uint32_t*)(KE + j0 / 16 + 4 * hf), ves = *(const uint32_t*)(VE + j0 / 16 + 4 * hf);
          const bool full = j0 + BT <= firstm.hi && (j0 >= lastm.lo || j0 + BT <= a.sinks);
          if (ok) ok = wait_phase(&s_full[gt & 1], (uint32_t)(gt >> 1) & 1u);
          tc_fence_after();
          if (i == 0) rf = q_factor(row_exp[(qi & 3) * BM + r], a.scale_log2);   // (S needed Q: it is there)
          const uint32_t srow = lane_base + (uint32_t)(gt & 1) * BT;
          float sc[64], mx = -INFINITY, wx = -INFINITY, mu, wu;
          scores(srow + 64 * hf, j0 + 64 * hf, full, sc);
          maxima(sc, kes, ves, mx, wx);
          // (past the barrier both halves have read their scores, past a second or the next tile's
          // the maxima)
          float2* xt = xm + (Shape::XM > 1 ? (gt & 1) * 256 : 0);
          xt[hf * 128 + r] = make_float2(mx, wx);
          pair_bar();
          const float2 x0 = xt[r], x1 = xt[128 + r];
          if (Shape::XM == 1) pair_bar();
          refer(fmaxf(x0.x, x1.x), fmaxf(x0.y, x1.y), i > 0, gt - 1, mu, wu);
          weights(sc, kes, ves, mu, wu, srow + 32 * hf);
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(&p_full[gt & 1]);
        }
      }
      if (n > 0) ++qi;
      coming = item_of(a, after);
      if (ok && n > 0) {
        ok = wait_phase(&pv_done[(gt - 1) % SB], (uint32_t)((gt - 1) / SB) & 1u);
        tc_fence_after();
      }
      float of[2] = {1.f, 0.f};   // what the warpgroups' outputs are scaled by
      if constexpr (Shape::own) {
        float* xw = (float*)(xm + 256);
        xm[hf * 128 + r] = make_float2(m, l);
        xw[hf * 128 + r] = W;
        pair_bar();
        const float2 x0 = xm[r], x1 = xm[128 + r];
        const float w0 = xw[r], w1 = xw[128 + r];
        m = fmaxf(x0.x, x1.x);
        W = fmaxf(w0, w1);
        const float mu = m == -INFINITY ? 0.f : m, wu = W == -INFINITY ? 0.f : W;
        // (exact steps of powers of two, as between a row's references)
        l = fmaf(x0.y, pow2f_down(x0.x - mu), x1.y * pow2f_down(x1.x - mu));
        of[0] = pow2f_down(w0 - wu);
        of[1] = pow2f_down(w1 - wu);
      } else {
        pair_bar();   // (the last tile's maxima are read)
        xm[hf * 128 + r].x = l;
        pair_bar();
        l = xm[r].x + xm[128 + r].x;
      }
      pair_bar();
      const bool real = mk.hi > 0 && n > 0 && !(l <= 0.f);   // (a sum that is not a number stays one)
      const float inv = real ? pow2f(W - m) / l : 0.f;
      // 32 of the row's outputs, normalised (not numbers to go by where the row is not real)
      auto output = [&](int cb, uint32_t (&raw)[32]) {
        auto times = [](uint32_t& a, uint32_t& b, float f) {
          const float2 x = fma2(make_float2(__uint_as_float(a), __uint_as_float(b)), make_float2(f, f), make_float2(-0.f, -0.f));
          a = __float_as_uint(x.x);
          b = __float_as_uint(x.y);
        };
        if constexpr (!Shape::own) {
          tmem_ld32_async(lane_base + o_col + cb, raw);
          tmem_wait_ld();
          tmem_reg_fence16(raw);
          tmem_reg_fence16(raw + 16);
#pragma unroll
          for (int q = 0; q < 32; q += 2) times(raw[q], raw[q + 1], inv);
        } else {
          // (of a single tile, one output has nothing of this item)
          const int only = n == 1 ? (gt - 1) & 1 : 0;
          const float f0 = n > 1 ? of[0] * inv : inv, f1 = of[1] * inv;
#pragma unroll
          for (int q16 = 0; q16 < 32; q16 += 16) {
            uint32_t* x = raw + q16;
            uint32_t y[16] = {};
            tmem_ld16_async(lane_base + o_col + only * HDP + cb + q16, x);
            if (n > 1) tmem_ld16_async(lane_base + o_col + HDP + cb + q16, y);
            tmem_wait_ld();
            tmem_reg_fence16(x);
            tmem_reg_fence16(y);
#pragma unroll
            for (int q = 0; q < 16; q += 2) {
              times(x[q], x[q + 1], f0);
              if (n > 1) {
                const float2 z = fma2(make_float2(__uint_as_float(y[q]), __uint_as_float(y[q + 1])), make_float2(f1, f1),
                                      make_float2(__uint_as_float(x[q]), __uint_as_float(x[q + 1])));
                x[q] = __float_as_uint(z.x);
                x[q + 1] = __float_as_uint(z.y);
              }
            }
          }
        }
      };
      const float m_out = real ? m : -INFINITY, l_out = real ? l : 0.f;
      if (a.splits == 1) {
        if (a.mass && hf == 0 && r < rows) a.row_ml[head * a.n * a.G + r0 + r] = row_weight(m_out, l_out, kTcShift);
        // O / l as bf16, each thread's columns of its row
        bf16 *own = out_row(min(r, rows - 1)), *dst[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) dst[k] = out_row(min(q4 * 32 + (lane & ~3) + k, rows - 1)) + 8 * (lane & 3);
#pragma unroll 1
        for (int cb = 32 * hf; cb < HDP; cb += 64) {   // (the warpgroups take alternate columns)
          uint32_t raw[32];
          output(cb, raw);
          if (cb + 64 >= HDP) {   // the last of O: the next item's may begin
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
          }
          uint32_t wd[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) wd[q] = real ? pack_bf16x2(__uint_as_float(raw[2 * q]), __uint_as_float(raw[2 * q + 1])) : 0u;
          if (wide) {
            // four lanes' rows turned into four pieces of a row each: stores of 8 rows x 64 bytes
            auto turn = [&](uint32_t& a, uint32_t& b, int bit) {
              const uint32_t got = __shfl_xor_sync(0xffffffffu, lane & bit ? a : b, bit);
              (lane & bit ? a : b) = got;
            };
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              turn(wd[q], wd[4 + q], 1);
              turn(wd[8 + q], wd[12 + q], 1);
              turn(wd[q], wd[8 + q], 2);
              turn(wd[4 + q], wd[12 + q], 2);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (q4 * 32 + (lane & ~3) + k < rows && cb + 8 * (lane & 3) < L.hd)
                *(uint4*)(dst[k] + cb) = make_uint4(wd[4 * k], wd[4 * k + 1], wd[4 * k + 2], wd[4 * k + 3]);
          } else if (r < rows) {
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (cb + q < L.hd) own[cb + q] = __ushort_as_bfloat16((unsigned short)(wd[q / 2] >> (16 * (q & 1))));
          }
        }
        continue;
      }
      // splits (one item per CTA): normalised partials, joined in the splits' order: up to 8
      // splits are a cluster, whose CTAs read a share of the rows each from one another's
      // shared memory; of more, which store to L2, the last to arrive joins all rows
      const bool cluster = a.splits <= kTcCluster;
      const size_t unit = head * a.row_tiles + it.tile;
      constexpr uint32_t XR = Shape::xrow;
#pragma unroll 1
      for (int cb = 32 * hf; cb < HDP; cb += 64) {
        uint32_t raw[32];
        output(cb, raw);
#pragma unroll
        for (int q = 0; q < 32; ++q) raw[q] = real ? raw[q] : 0u;
        if (cluster) {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            sts_u4(k0 + (uint32_t)r * XR + 4u * (cb + 4 * q), make_uint4(raw[4 * q], raw[4 * q + 1], raw[4 * q + 2], raw[4 * q + 3]));
        } else if (r < rows) {
          uint4* part = (uint4*)(a.part + ((unit * a.splits + it.split) * BM + r) * HDP + cb);
#pragma unroll
          for (int q = 0; q < 8; ++q) __stcg(part + q, make_uint4(raw[4 * q], raw[4 * q + 1], raw[4 * q + 2], raw[4 * q + 3]));
        }
      }
      int ra = 0, rb = rows;
      if (cluster) {
        if (hf == 0) {
          xm[r] = make_float2(m_out, l_out);
        }
        cluster_sync();   // (the other roles arrive below)
        const int share = (rows + a.splits - 1) / a.splits;
        ra = it.split * share;
        rb = min(rows, ra + share);
      } else {
        if (hf == 0) __stcg(a.part_ml + (unit * a.splits + it.split) * BM + r, make_float2(m_out, l_out));
        __threadfence();
        asm volatile("bar.sync 5, 256;" ::: "memory");
        if (threadIdx.x == 0) *last_flag = atomicInc(a.arrived + unit, (unsigned)a.splits - 1u) == (unsigned)a.splits - 1u;
        asm volatile("bar.sync 5, 256;" ::: "memory");
        if (!*last_flag) rb = 0;
        __threadfence();
      }
      // the splits' weights per row, [splits][128], into Q's place (every S has completed)
      // or, where they may be many, the rings' ...
      float* wts = (float*)(smem + (cluster ? 0 : Shape::q_bytes));
      for (int rr = ra + threadIdx.x; rr < rb; rr += 256) {
        const float2* ml = a.part_ml + unit * a.splits * BM + rr;
        const uint32_t xml = smem_u32(xm) + 8u * rr;
        auto split_ml = [&](int q) {
          if (!cluster) return ld_l2(ml + q * BM);
          const uint32_t at = mapa_shared(xml, (uint32_t)q);
          return make_float2(ld_cluster_f1(at), ld_cluster_f1(at + 4));
        };
        float M = -INFINITY, S = 0.f;
        for (int q = 0; q < a.splits; ++q) M = fmaxf(M, split_ml(q).x);
        for (int q = 0; q < a.splits; ++q) {
          const float2 x = split_ml(q);
          const float wt = x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y);
          wts[q * BM + rr] = wt;
          S += wt;
        }
        const float sv = !(S <= 0.f) ? 1.f / S : 0.f;
        for (int q = 0; q < a.splits; ++q) wts[q * BM + rr] *= sv;
        if (a.mass) a.row_ml[head * a.n * a.G + r0 + rr] = row_weight(M, S, kTcShift);
      }
      asm volatile("bar.sync 5, 256;" ::: "memory");
      // ... then a warp per row
      if (8 * lane < L.hd) {
#pragma unroll 2
        for (int rr = ra + warp; rr < rb; rr += 8) {
          const float* p0 = a.part + (unit * a.splits * BM + rr) * HDP + 8 * lane;
          float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
          for (int q = 0; q < a.splits; ++q) {
            const float wt = wts[q * BM + rr];
            float4 y0, y1;
            if (cluster) {
              const uint32_t at = mapa_shared(k0 + (uint32_t)rr * XR + 32u * lane, (uint32_t)q);
              y0 = ld_cluster_f4(at);
              y1 = ld_cluster_f4(at + 16);
            } else {
              const float4* y = (const float4*)(p0 + (size_t)q * BM * HDP);
              y0 = ld_l2(y);
              y1 = ld_l2(y + 1);
            }
            acc[0] = fmaf(wt, y0.x, acc[0]);
            acc[1] = fmaf(wt, y0.y, acc[1]);
            acc[2] = fmaf(wt, y0.z, acc[2]);
            acc[3] = fmaf(wt, y0.w, acc[3]);
            acc[4] = fmaf(wt, y1.x, acc[4]);
            acc[5] = fmaf(wt, y1.y, acc[5]);
            acc[6] = fmaf(wt, y1.z, acc[6]);
            acc[7] = fmaf(wt, y1.w, acc[7]);
          }
          store_bf16x8(out_row(rr) + 8 * lane,
                       make_uint4(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]), pack_bf16x2(acc[4], acc[5]),
                                  pack_bf16x2(acc[6], acc[7])),
                       wide);
        }
      }
      if (cluster) cluster_sync();   // nobody leaves while its rows are read
    }
    if (!ok && lane == 0) *abort_flag = 1;
  }
  if (warp >= 8 && a.splits > 1 && a.splits <= kTcCluster && item_of(a, blockIdx.x).live) {
    cluster_sync();
    cluster_sync();
  }
  tc_fence_before();
  cta_sync();
  if (*abort_flag && threadIdx.x == 0) {
    // loads still on their way, at most a ring of them, land before the shared memory goes away
    for (int i = max(0, issued_flag[0] - KS); i < issued_flag[0]; ++i) mbar_wait(&k_full[i % KS], (uint32_t)(i / KS) & 1u);
    if (issued_flag[2] > 0) mbar_wait(q_full, (uint32_t)(issued_flag[2] - 1) & 1u);
    for (int i = max(0, issued_flag[1] - CV); i < issued_flag[1]; ++i) mbar_wait(&cv_full[i % CV], (uint32_t)(i / CV) & 1u);
    raise_error(a.err, ERR_TIMEOUT);
  }
  if (warp == 16)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int NB>
cudaError_t launch_nb(CacheAttnArgs a, cudaStream_t st) {
  a.row_tiles = (a.n * a.G + BM - 1) / BM;
  const long long tiles = (long long)a.row_tiles * a.c.Hkv * a.batch;
  long long seen = a.max_length;
  if (a.window > 0) seen = std::min(seen, (long long)a.window + a.sinks + BM / a.G + 1 + 2 * BT);
  const int units = (int)((seen + BT - 1) / BT);
  // As many splits as the SMs hold, as a cluster if that many clusters fit on the
  // device at once, and no more than shorten the longest one.
  int splits = (int)std::max(1ll, std::min(std::min((long long)a.num_sms / tiles, (long long)units), 256ll));
  if (splits <= kTcCluster)
    while (splits > 1 && a.clusters[splits] < tiles) --splits;
  if (splits > 1) splits = (units + (units + splits - 1) / splits - 1) / ((units + splits - 1) / splits);
  a.splits = splits;
  a.by_splits = LaunchDiv(splits);
  const TcMaps maps{a.maps->k_tc, a.maps->v_tc};
  // causal prompts: pairs whose caches take 48 MB together (beside the queries, in an L2 of 129)
  const long long pairs = (long long)a.c.Hkv * a.batch;
  a.group = 1;
  if (a.causal && !a.window) a.group = (int)std::min(pairs, std::max(1ll, (48ll << 20) / (2ll * a.max_length * a.c.hdp + 1)));
  if (tiles * a.splits > 0x7fff0000ll) return cudaErrorInvalidValue;
  a.by_group = LaunchDiv(a.group * a.row_tiles);
  a.by_pairs = LaunchDiv(a.group);
  a.by_last = LaunchDiv((int)std::max(1ll, pairs % a.group));
  const unsigned grid = a.splits == 1 ? (unsigned)std::min(tiles, (long long)a.num_sms) : (unsigned)(tiles * a.splits);
  const Overlap overlap;
  return launch_kernel_cluster(cache_tc_kernel<NB>, dim3(grid), dim3(TCT), TcShape<NB>::bytes, st,
                               dim3(a.splits <= kTcCluster ? a.splits : 1, 1, 1), maps, a);
}

template <int NB>
cudaError_t init_nb(int* clusters) {
  cudaError_t e = cudaFuncSetAttribute(cache_tc_kernel<NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<NB>::bytes);
  for (int s = 2; s <= kTcCluster && e == cudaSuccess; ++s) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    cfg.gridDim = dim3(s);
    cfg.blockDim = dim3(TCT);
    cfg.dynamicSmemBytes = TcShape<NB>::bytes;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = s;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&clusters[s], cache_tc_kernel<NB>, &cfg);
  }
  return e;
}

}  // namespace

static PFN_cuTensorMapEncodeTiled_v12000 g_enc = nullptr;

cudaError_t encode_codes(CUtensorMap* m, const uint8_t* base, const CacheLayer& c, int batch, int in, int box_rows,
                         bool swizzle) {
  cuuint64_t dims[2] = {(cuuint64_t)c.hdp, (cuuint64_t)batch * c.Hkv * c.T};
  cuuint64_t strides[1] = {(cuuint64_t)c.hdp};
  cuuint32_t box[2] = {(cuuint32_t)in, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  const CUresult r = g_enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, !swizzle ? CU_TENSOR_MAP_SWIZZLE_NONE : (in == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B), CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t cache_tc_encoder() {
  if (!g_enc) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
    if (e != cudaSuccess) return e;
    if (q != cudaDriverEntryPointSuccess || !fn) return cudaErrorSymbolNotFound;
    g_enc = (PFN_cuTensorMapEncodeTiled_v12000)fn;
  }
  return cudaSuccess;
}

cudaError_t launch_cache_attend_tc(const CacheAttnArgs& a, cudaStream_t st) {
  switch (a.c.hdp) {
    case 64: return launch_nb<1>(a, st);
    case 128: return launch_nb<2>(a, st);
    case 192: return launch_nb<3>(a, st);
    default: return launch_nb<4>(a, st);
  }
}

cudaError_t init_cache_tc_kernels(int hdp, int* clusters) {
  switch (hdp) {
    case 64: return init_nb<1>(clusters);
    case 128: return init_nb<2>(clusters);
    case 192: return init_nb<3>(clusters);
    default: return init_nb<4>(clusters);
  }
}

}  // namespace ravel
