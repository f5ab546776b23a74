// Attention over the 8-bit context cache for many query rows (an expert's slots,
// prompts), bf16, on the 5th-generation tensor cores.
//
// A CTA owns 128 rows (row r = query * G + head of the group) of one (robot, KV
// head) and a share (split) of the 128-token tiles that they see:
//   S = Q K^T        tcgen05.mma kind::f16, M = 128, N = 128, into TMEM
//   P = 2^(S - m)    softmax warps: TMEM -> registers -> f16 P over S in TMEM
//   O += P V         tcgen05.mma, M = 128, N = head dim, 16 tokens at a time
// Warp roles (640 threads): warps 0-7 Q, softmax and epilogue, two threads per row;
// warps 8-11 widen K, warps 12-15 widen V; warp 16 TMEM and MMAs; warps 17, 18 load
// the codes of K and V (19 idle, so that registers move between whole warpgroups).
//
// The codes come by TMA and are widened in shared memory to f16 (e4m3 -> f16 is
// exact), into the 128-byte swizzled layout that a TMA load of f16 rows would
// leave: K in units of 64 head dims (16 KB), V in halves of 64 tokens, each in
// rings of its own with its own warps, so that neither waits for the other's
// slots.  (With the codes loaded to registers by the widening warps themselves a
// unit took a load's latency, 900 cycles of the 512 that the MMAs of four units
// leave each: the proxy fence that ends a unit waits for the loads in flight.)
// Feeding the codes as kind::f8f6f4
// operands instead would need Q and P in 8 bits too: two pieces of each keep
// bf16's precision and cost what one f16 MMA does, but 2^-9 is the least P that
// e4m3 holds, and a long flat tail of smaller ones carries weight.
//
// Numbers as in the kernel for few rows: q in f16 under a power of two per row
// (exact for bf16), block exponents of K on the scores, those of V on P.  P is at
// most 2^7 of the reference, 2^15 while a grown one waits for its rescaling of O
// (only growth by more than 2^8 rescales); what contributes less than 2^-31 of the
// row's largest is dropped.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>

#include "cache_attn.cuh"
#include "launch.h"

namespace ravel {
namespace {

constexpr int TCT = 640;
constexpr int BM = 128, BT = 128;              // rows, tokens of a tile
constexpr uint32_t QB = BM * 128;              // bytes of a 64-dim block of Q
constexpr uint32_t KU = BT * 128;              // bytes of a K unit: 128 tokens x 64 dims
constexpr uint32_t CB = 64 * 64;                // bytes of a slot of codes: 64 tokens x 64 dims
constexpr uint32_t VB = 64 * 128;              // bytes of a 64-dim block of a V half
constexpr float kTcShift = 7.f;                // P's largest value is 2^kTcShift (times 2^8 while lazy)
constexpr int kTcCluster = 8;                  // splits that are a cluster
constexpr uint32_t kPolls = 1u << 25;          // polls without progress: seconds

template <int NB> struct TcShape {
  // shared memory at NB blocks of 64 head dims: Q, the rings of widened K units and V
  // halves, the rings of codes, barriers and row data
  static constexpr int KS = 4;
  static constexpr int VS = NB >= 3 ? 2 : 4;
  // a multiple of the 4 warps that widen them: each slot is then waited for by one warp, in
  // order.  (Loads may complete out of order; a warp that waits for a slot's next phase while
  // another's load into it is still on its way would take the phase before for it.)
  static constexpr int CS = NB == 4 ? 4 : 8;
  static_assert(CS % 4 == 0, "widening warps");
  static constexpr uint32_t ring = KS * KU + VS * NB * VB + 2 * CS * CB;
  static constexpr uint32_t bytes = NB * QB + ring + 3072;
  static_assert(bytes <= 227 * 1024, "shared memory");
  // a row of the fp32 output that splits exchange (over the rings): 16 bytes more than
  // the dims, so that rows written by neighbouring lanes fall on different banks
  static constexpr uint32_t xrow = NB * 64 * 4 + 16;
  static_assert(BM * xrow <= ring && BM * 4 * 256 <= ring && BM * 4 * 8 <= NB * QB, "exchange");
};

struct TcMaps {
  CUtensorMap k, v;   // a layer's codes [B Hkv T][hdp] in boxes of 64 dims x 64 rows
};

// f16 A and B, fp32 D
__device__ __forceinline__ uint32_t idesc_f16(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ void sts_u4(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// 16 codes -> two 16-byte pieces of f16
__device__ __forceinline__ void widen(uint4 w, uint32_t lo, uint32_t hi) {
  sts_u4(lo, make_uint4(e4m3_lo(w.x), e4m3_hi(w.x), e4m3_lo(w.y), e4m3_hi(w.y)));
  sts_u4(hi, make_uint4(e4m3_lo(w.z), e4m3_hi(w.z), e4m3_lo(w.w), e4m3_hi(w.w)));
}

// Registers of a warpgroup: launched with 96 each (640 x 96 = 61440); softmax
// 2 x 128 x 144, widening 2 x 128 x 80, the rest 128 x 24: 60416.
template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

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

// eight bf16 at any alignment
__device__ __noinline__ uint4 ldg_bf16x8(const bf16* p) {
  bf16 y[8];
#pragma unroll
  for (int z = 0; z < 8; ++z) y[z] = p[z];
  uint4 w;
  memcpy(&w, y, 16);
  return w;
}

__device__ __forceinline__ uint4 lds_codes(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ float2 ld_cluster_f2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a));
  return v;
}

// A warp's writes to shared memory become visible to the tensor core: one arrival per warp.
__device__ __forceinline__ void written(uint64_t* bar) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

template <int NB>
__global__ void __launch_bounds__(TCT, 1) cache_tc_kernel(const __grid_constant__ TcMaps maps, CacheAttnArgs a) {
  constexpr int HDP = 64 * NB, KS = TcShape<NB>::KS, VS = TcShape<NB>::VS, CS = TcShape<NB>::CS;
  constexpr uint32_t VH = NB * VB;   // bytes of a V half
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t q0 = smem_u32(smem), k0 = q0 + NB * QB, v0 = k0 + KS * KU, ck0 = v0 + VS * VH, cv0 = ck0 + CS * CB;
  uint8_t* tail = smem + NB * QB + TcShape<NB>::ring;
  uint64_t* k_full = (uint64_t*)tail;
  uint64_t* k_empty = k_full + KS;
  uint64_t* v_full = k_empty + KS;
  uint64_t* v_empty = v_full + VS;
  uint64_t* c_full = v_empty + VS;   // [2 CS] codes of K, then of V
  uint64_t* c_empty = c_full + 2 * CS;
  uint64_t* s_full = c_empty + 2 * CS;   // [2]
  uint64_t* p_full = s_full + 2;     // [2]
  uint64_t* pv_done = p_full + 2;    // [2]
  uint64_t* q_full = pv_done + 2;
  uint64_t* ended = q_full + 1;
  uint32_t* tmem_slot = (uint32_t*)(ended + 1);
  int* abort_flag = (int*)(tmem_slot + 1);
  int* last_flag = abort_flag + 1;
  int* c_issued = last_flag + 1;     // [2] loads of codes issued, K and V
  uint32_t* row_top = (uint32_t*)(tail + 512);    // [128] bits of the rows' largest |q|
  float2* xm = (float2*)(tail + 1024);            // [2][128] row maxima, then sums, of the two halves
  static_assert((2 * KS + 2 * VS + 4 * CS + 8) * 8 + 20 <= 512, "barriers");

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int b = blockIdx.z, h = blockIdx.y, split = blockIdx.x % a.splits;
  const int tile = a.row_tiles - 1 - (int)blockIdx.x / a.splits;   // (causal: the longest first)
  const CacheLayer& L = a.c;
  const int r0 = tile * BM, rows = min(BM, a.n * a.G - r0);
  const size_t head = (size_t)b * L.Hkv + h;
  Sight s;
  if (q0 & 1023u) {   // (the swizzled layouts count on it)
    if (threadIdx.x == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  if (!robot_sight(a, b, s) && threadIdx.x == 0 && blockIdx.x == 0 && h == 0) raise_error(a.err, ERR_SHAPE);
  bf16* out0 = (bf16*)a.out + (size_t)((long long)b * a.out_robot) + (size_t)h * a.G * L.hd;
  auto out_row = [&](int r) {
    const uint32_t i = (uint32_t)r / (uint32_t)a.G;
    return out0 + (size_t)((long long)i * a.out_token) + (size_t)((uint32_t)r - i * (uint32_t)a.G) * L.hd;
  };
  if (r0 >= s.count * a.G || s.len == 0) {   // nothing to see: zeros
    if (split == 0)
      for (int w = threadIdx.x; w < rows * L.hd; w += TCT) out_row(r0 + w / L.hd)[w % L.hd] = __float2bfloat16_rn(0.f);
    if (split == 0 && a.mass && threadIdx.x < rows)
      a.row_ml[head * a.n * a.G + r0 + threadIdx.x] = make_float2(0.f, 0.f);
    return;
  }
  tile_sight(a, s, r0, r0 + BM - 1, BT);
  const int t0 = (int)((long long)s.units * split / a.splits), t1 = (int)((long long)s.units * (split + 1) / a.splits);
  const int n = t1 - t0;
  const RowMask firstm = row_mask(a, s, r0), lastm = row_mask(a, s, min(r0 + BM, s.count * a.G) - 1);
  // first token of tile t, and how many of its tokens exist for these rows
  auto tile_token = [&](int t) { return (t < s.sink_units ? t : t - s.sink_units + s.from) * BT; };
  auto keys_of = [&](int j0) { return min(BT, lastm.hi - j0); };

  if (threadIdx.x == 0) {
    for (int i = 0; i < KS; ++i) {
      mbar_init(&k_full[i], 2);   // its steps
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < VS; ++i) {
      mbar_init(&v_full[i], NB);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2 * CS; ++i) {
      mbar_init(&c_full[i], 1);
      mbar_init(&c_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      c_issued[i] = 0;
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 256);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(q_full, 8);
    mbar_init(ended, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // Q: rows of 8 NB lanes with 8 dims each, 16 rows per softmax warp; on their way while
  // TMEM and barriers are set up
  constexpr int LPR = 8 * NB, RPW = 32 / LPR, PASS = 16 / RPW;
  const int q_sub = lane / LPR, q_dl = lane % LPR;
  uint4 qx[PASS];
  if (warp < 8) {
    const bool on = q_sub < RPW && 8 * q_dl < L.hd;
    const bf16* base = (const bf16*)a.q + (size_t)((long long)b * a.q_robot) + (size_t)h * a.G * L.hd + 8 * q_dl;
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const uint32_t r = (uint32_t)(r0 + warp * 16 + p * RPW + q_sub), i = r / (uint32_t)a.G;
      const bf16* at = base + (size_t)((long long)i * a.q_token) + (size_t)(r - i * a.G) * L.hd;
      qx[p] = make_uint4(0u, 0u, 0u, 0u);
      if (on && (int)i < s.count) qx[p] = a.vec ? __ldg((const uint4*)at) : ldg_bf16x8(at);
    }
  }
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t o_col = 2 * BT;

  if (warp >= 8 && warp < 16) {
    regs_down<80>();
    // ---- widening: K in units of 64 dims (warps 8-11), V in halves of 64 tokens (12-15), in
    // steps of 64 tokens x 64 dims.  A warp takes every fourth step as a whole, so that the
    // waits, the proxy fence and the shared-memory latency of one lie beside the work on the
    // others (a unit by four warps together took 750 cycles, little of it work).
    const bool is_k = warp < 12;
    // lane: 16 codes at dim 16 (lane % 4) of rows lane / 4, lane / 4 + 8, ...
    const uint32_t sw = (uint32_t)(lane >> 2), row = (uint32_t)(lane >> 2) * 128u;
    const uint32_t lo = row + ((((uint32_t)lane & 3u) * 2u) ^ sw) * 16u, hi = row + ((((uint32_t)lane & 3u) * 2u + 1u) ^ sw) * 16u;
    const uint32_t codes = (is_k ? ck0 : cv0) + 16u * lane;
    uint64_t *cf = c_full + (is_k ? 0 : CS), *ce = c_empty + (is_k ? 0 : CS);
    // a unit of K takes 2 steps, a half of V NB; every tile but the last has two halves
    const int per = is_k ? 2 : NB, ring = is_k ? KS : VS;
    const int steps = is_k ? n * NB * 2 : (n > 0 ? (2 * n - (keys_of(tile_token(t1 - 1)) > 64 ? 0 : 1)) * NB : 0);
    const uint32_t to0 = (is_k ? k0 : v0), slot_bytes = is_k ? KU : VH;
    uint64_t *full = is_k ? k_full : v_full, *empty = is_k ? k_empty : v_empty;
    bool ok = true;
    for (int u = warp & 3; u < steps; u += 4) {
      const int cs = u % CS, item = u / per, slot = item % ring;
      ok = mbar_wait_warp(&cf[cs], (uint32_t)(u / CS) & 1u);
      if (!ok) break;
      uint4 x[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) x[y] = lds_codes(codes + (uint32_t)cs * CB + 512u * y);
      ok = mbar_wait_warp(&empty[slot], ((uint32_t)(item / ring) & 1u) ^ 1u);
      if (!ok) break;
      __syncwarp();   // every lane has its codes
      if (lane == 0) mbar_arrive(&ce[cs]);
      const uint32_t to = to0 + (uint32_t)slot * slot_bytes + (uint32_t)(u % per) * VB;
#pragma unroll
      for (int y = 0; y < 8; ++y) widen(x[y], to + lo + 1024u * y, to + hi + 1024u * y);
      written(&full[slot]);
    }
    if (!ok && lane == 0) *abort_flag = 1;
  } else if (warp >= 16) {
    regs_down<24>();
    if (warp == 16) {
    // ---- MMAs: S of the next tile as soon as its K is there, P V of the oldest whose P is
    const uint32_t el = elect_one();
    const uint32_t idesc_s = idesc_f16(BM, BT), idesc_o = idesc_f16(BM, HDP) | (1u << 16);
    const uint64_t qd0 = sw128_desc(q0), kd0 = sw128_desc(k0), vd0 = sw128_mn_desc(v0, VB);
    int ns = 0, i = 0, sk = 0, sv = 0;
    uint32_t phk = 0, phv = 0, spins = 0;
    bool ok = mbar_wait_warp(q_full, 0);
    while (ok && i < n) {
      bool progress = false;
      if (ns < n && ns <= i + 1 && mbar_test_warp(&k_full[sk], phk)) {
        const uint32_t sd = tmem + (uint32_t)(ns & 1) * BT;
        uint64_t ad = qd0;
#pragma unroll 1
        for (int blk = 0; blk < NB; ++blk, ad += QB >> 4) {
          if (blk) ok = mbar_wait_warp(&k_full[sk], phk);
          if (!ok) break;
          tc_fence_after();
          const uint64_t bd = kd0 + (uint32_t)sk * (KU >> 4);
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_bf16(sd, ad + 2 * k, bd + 2 * k, idesc_s, (blk > 0 || k > 0) ? 1u : 0u, el);
          umma_commit(&k_empty[sk], el);
          if (++sk == KS) {
            sk = 0;
            phk ^= 1u;
          }
        }
        if (!ok) break;
        umma_commit(&s_full[ns & 1], el);
        ++ns;
        progress = true;
      }
      if (i < ns && mbar_test_warp(&p_full[i & 1], (uint32_t)(i >> 1) & 1u) && mbar_test_warp(&v_full[sv], phv)) {
        const uint32_t pa = tmem + (uint32_t)(i & 1) * BT;
        const int groups = (keys_of(tile_token(t0 + i)) + 15) >> 4;
#pragma unroll 1
        for (int hv = 0; 4 * hv < groups; ++hv) {
          if (hv) ok = mbar_wait_warp(&v_full[sv], phv);
          if (!ok) break;
          tc_fence_after();
          const uint64_t bd = vd0 + (uint32_t)sv * (VH >> 4);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (4 * hv + k < groups)
              umma_bf16_ts(tmem + o_col, pa + 8 * (4 * hv + k), bd + 128 * k, idesc_o, (i + hv + k > 0) ? 1u : 0u, el);
          umma_commit(&v_empty[sv], el);
          if (++sv == VS) {
            sv = 0;
            phv ^= 1u;
          }
        }
        if (!ok) break;
        umma_commit(&pv_done[i & 1], el);
        ++i;
        progress = true;
      }
      spins = progress ? 0u : spins + 1u;
      if (spins > kPolls) ok = false;
    }
    if (!ok) {   // what was issued ends before the TMEM goes away
      umma_commit(ended, el);
      mbar_wait_warp(ended, 0);
      if (lane == 0) *abort_flag = 1;
    }
    __syncwarp();
    } else if (warp < 19) {
      // ---- the codes' loads
      const uint32_t el = elect_one();
      const bool is_k = warp == 17;
      const uint32_t to = is_k ? ck0 : cv0;
      uint64_t *cf = c_full + (is_k ? 0 : CS), *ce = c_empty + (is_k ? 0 : CS);
      uint64_t pol;
      asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
      const int y0 = (int)(head * L.T);
      int slot = 0, issued = 0;
      uint32_t ph = 1;
      bool ok = true;
      for (int t = t0; ok && t < t1; ++t) {
        const int j0 = tile_token(t), steps = NB * (is_k || keys_of(j0) > 64 ? 2 : 1);
        for (int q = 0; q < steps; ++q) {
          ok = mbar_wait_warp(&ce[slot], ph);
          if (!ok) break;
          // K: the unit's two halves of 64 tokens; V: the half's blocks of 64 dims
          const int half = is_k ? q & 1 : q / NB, blk = is_k ? q >> 1 : q % NB;
          mbar_expect_tx_el(&cf[slot], CB, el);
          tma_load_2d_el(is_k ? &maps.k : &maps.v, smem_u32(&cf[slot]), to + (uint32_t)slot * CB, 64 * blk, y0 + j0 + 64 * half,
                         pol, el);
          ++issued;
          if (++slot == CS) {
            slot = 0;
            ph ^= 1u;
          }
        }
      }
      if (lane == 0) {
        c_issued[is_k ? 0 : 1] = issued;
        if (!ok) *abort_flag = 1;
      }
      __syncwarp();
    }
  } else {
    regs_up<144>();
    // ---- Q, scaled by the rows' powers of two
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const uint32_t u[4] = {qx[p].x, qx[p].y, qx[p].z, qx[p].w};
      uint32_t top = 0u;   // bits of the largest magnitude: NaN counts as larger than all
#pragma unroll
      for (int z = 0; z < 4; ++z) top = max(top, max((u[z] & 0x7fffu) << 16, u[z] & 0x7fff0000u));
      if (RPW == 1) {
        top = __reduce_max_sync(0xffffffffu, top);
      } else {
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      }
      const float f = top >= 0x7f800000u ? __int_as_float(0x7fffffff) : exp2i(min(14 - ((int)(top >> 23) - 127), 126));
      uint32_t w[4];
#pragma unroll
      for (int z = 0; z < 4; ++z) w[z] = pack_f16x2(__uint_as_float(u[z] << 16) * f, __uint_as_float(u[z] & 0xffff0000u) * f);
      const int lr = warp * 16 + p * RPW + q_sub;
      if (q_sub < RPW) {
        sts_u4(q0 + (uint32_t)(q_dl >> 3) * QB + (uint32_t)lr * 128u + (uint32_t)(((q_dl & 7) ^ (lr & 7)) * 16),
               make_uint4(w[0], w[1], w[2], w[3]));
        if (q_dl == 0) row_top[lr] = top;
      }
    }
    written(q_full);
    asm volatile("bar.sync 5, 256;" ::: "memory");   // row_top
    // ---- softmax and epilogue: row r (TMEM lane r), tokens 64 hf .. of each tile
    const int q4 = warp & 3, hf = warp >> 2, r = q4 * 32 + lane;
    auto pair_bar = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + q4) : "memory"); };   // warps w and w + 4
    const uint32_t lane_base = tmem + ((uint32_t)(q4 * 32) << 16);
    const RowMask mk = row_mask(a, s, r0 + r);
    // (rows whose largest |q| is below 2^-112 keep fewer bits; -e >= -126)
    const float rf = exp2i(-min(14 - ((int)(row_top[r] >> 23) - 127), 126)) * a.scale_log2;
    const int8_t *KE = L.ke + head * (L.T / 16), *VE = L.ve + head * (L.T / 16);
    // references in the log2 domain, integral: m of the row's sum, W of O (largest score + value exponent)
    float m = -INFINITY, W = -INFINITY, l = 0.f;
    bool ok = true;
    for (int i = 0; i < n; ++i) {
      const int j0 = tile_token(t0 + i);
      // exponents of this half's four blocks
      const uint32_t kes = *(const uint32_t*)(KE + j0 / 16 + 4 * hf), ves = *(const uint32_t*)(VE + j0 / 16 + 4 * hf);
      const bool full = j0 + BT <= firstm.hi && (j0 >= lastm.lo || j0 + BT <= a.sinks);
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&s_full[i & 1], (uint32_t)(i >> 1) & 1u));
      tc_fence_after();
      float sc[64];
      {
        uint32_t raw[64];
        const uint32_t srow = lane_base + (uint32_t)(i & 1) * BT + 64 * hf;
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld16_async(srow + 16 * q, raw + 16 * q);
        tmem_wait_ld();
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_reg_fence16(raw + 16 * q);
#pragma unroll
        for (int k = 0; k < 64; ++k) sc[k] = __uint_as_float(raw[k]);
      }
      if (!full) {
        const int jh = j0 + 64 * hf;
#pragma unroll
        for (int k = 0; k < 64; ++k) sc[k] = mk.sees(jh + k) ? sc[k] : -INFINITY;
      }
      float f[4], mx = -INFINITY, wx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        // (not 0, which times a hidden score's -inf would not be a number)
        f[t] = fmaxf(rf * exp2i((int)(int8_t)(kes >> (8 * t))), 1e-37f);
        float m4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          m4[e] = fmaxf(fmaxf(sc[16 * t + 4 * e], sc[16 * t + 4 * e + 1]), fmaxf(sc[16 * t + 4 * e + 2], sc[16 * t + 4 * e + 3]));
        const float x = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * f[t];
        mx = fmaxf(mx, x);
        wx = fmaxf(wx, x + (float)(int8_t)(ves >> (8 * t)));
      }
      // (past the first barrier both halves have read their scores, past the second the maxima)
      xm[hf * 128 + r] = make_float2(mx, wx);
      pair_bar();
      const float2 x0 = xm[r], x1 = xm[128 + r];
      pair_bar();
      const float mn = fmaxf(m, ceilf(fmaxf(x0.x, x1.x))), wn = fmaxf(W, ceilf(fmaxf(x0.y, x1.y)));
      const float mu = mn == -INFINITY ? 0.f : mn;
      l *= pow2f_down(m - mu);
      m = mn;
      const bool need = wn > W + 8.f;
      if (i > 0 && __any_sync(0xffffffffu, need)) {
        // O holds P V of every earlier tile before it is rescaled
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[(i - 1) & 1], (uint32_t)((i - 1) >> 1) & 1u));
        tc_fence_after();
        const float alpha = need ? pow2f_down(W - wn) : 1.f;
        for (int cb = 16 * hf; cb < HDP; cb += 32) {
          float o[16];
          tmem_ld16(lane_base + o_col + cb, o);
#pragma unroll
          for (int q = 0; q < 16; ++q) o[q] *= alpha;
          tmem_st16(lane_base + o_col + cb, o);
        }
        tmem_wait_st();
      }
      if (need) W = wn;
      const float wu = W == -INFINITY ? 0.f : W;
      const uint32_t prow = lane_base + (uint32_t)(i & 1) * BT + 32 * hf;
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        uint32_t w[16];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int blk = 2 * h2 + t;
          const float vf = fmaxf((float)(int8_t)(ves >> (8 * blk)), wu - mu - kVeBelow), nbt = kTcShift + vf - wu;
          float e[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) e[q] = fast_exp2(fmaf(sc[16 * blk + q], f[blk], nbt));
          float s4[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) s4[q] = (e[4 * q] + e[4 * q + 1]) + (e[4 * q + 2] + e[4 * q + 3]);
          l = fmaf((s4[0] + s4[1]) + (s4[2] + s4[3]), pow2f(wu - mu - vf), l);
#pragma unroll
          for (int q = 0; q < 8; ++q) w[8 * t + q] = pack_f16x2(e[2 * q], e[2 * q + 1]);
        }
        tmem_st16u(prow + 16 * h2, w);
      }
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&p_full[i & 1]);
    }
    if (ok && n > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[(n - 1) & 1], (uint32_t)((n - 1) >> 1) & 1u));
      tc_fence_after();
    }
    if (!ok && lane == 0) *abort_flag = 1;
    xm[hf * 128 + r].x = l;
    pair_bar();
    l = xm[r].x + xm[128 + r].x;
    const bool real = mk.hi > 0 && n > 0 && !(l <= 0.f);   // (a sum that is not a number stays one)
    const float inv = real ? pow2f(W - m) / l : 0.f;
    const float m_out = real ? m : -INFINITY, l_out = real ? l : 0.f;
    if (a.splits == 1) {
      if (a.mass && hf == 0 && r < rows) a.row_ml[head * a.n * a.G + r0 + r] = row_weight(m_out, l_out, kTcShift);
      // O / l as bf16 into Q's place (every S has completed), from where whole rows go out
      for (int cb = 32 * hf; cb < HDP; cb += 64) {
        uint32_t raw[32];
        tmem_ld32_async(lane_base + o_col + cb, raw);
        tmem_wait_ld();
        tmem_reg_fence16(raw);
        tmem_reg_fence16(raw + 16);
        const uint32_t at = q0 + (uint32_t)(cb >> 6) * QB + (uint32_t)r * 128u;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t w[4];
#pragma unroll
          for (int z = 0; z < 4; ++z)
            w[z] = real ? pack_bf16x2(__uint_as_float(raw[8 * q + 2 * z]) * inv, __uint_as_float(raw[8 * q + 2 * z + 1]) * inv) : 0u;
          sts_u4(at + (uint32_t)(((((cb & 32) >> 3) + q) ^ (r & 7)) * 16), make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
      asm volatile("bar.sync 5, 256;" ::: "memory");
      // a warp per row: 16-byte pieces
      const bool wide = ((uintptr_t)a.out | (uintptr_t)(a.out_robot * 2) | (uintptr_t)(a.out_token * 2)) % 16 == 0;
#pragma unroll 4
      for (int rr = warp; rr < rows; rr += 8) {
        bf16* dst = out_row(r0 + rr) + 8 * lane;
        if (8 * lane < L.hd) store_bf16x8(dst, lds_codes(q0 + (uint32_t)(lane >> 3) * QB + (uint32_t)rr * 128u + (uint32_t)(((lane & 7) ^ (rr & 7)) * 16)), wide);
      }
    } else {
      // normalised partials, joined in the splits' order: up to 8 splits are a cluster, whose
      // CTAs read a share of the rows each from one another's shared memory; of more, which
      // store to L2, the last to arrive joins all rows
      const bool cluster = a.splits <= kTcCluster;
      const size_t unit = head * a.row_tiles + tile;
      constexpr uint32_t XR = TcShape<NB>::xrow;
      for (int cb = 32 * hf; cb < HDP; cb += 64) {
        uint32_t raw[32];
        tmem_ld32_async(lane_base + o_col + cb, raw);
        tmem_wait_ld();
        tmem_reg_fence16(raw);
        tmem_reg_fence16(raw + 16);
#pragma unroll
        for (int q = 0; q < 32; ++q) raw[q] = real ? __float_as_uint(__uint_as_float(raw[q]) * inv) : 0u;
        if (cluster) {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            sts_u4(k0 + (uint32_t)r * XR + 4u * (cb + 4 * q), make_uint4(raw[4 * q], raw[4 * q + 1], raw[4 * q + 2], raw[4 * q + 3]));
        } else if (r < rows) {
          uint4* part = (uint4*)(a.part + ((unit * a.splits + split) * BM + r) * HDP + cb);
#pragma unroll
          for (int q = 0; q < 8; ++q) __stcg(part + q, make_uint4(raw[4 * q], raw[4 * q + 1], raw[4 * q + 2], raw[4 * q + 3]));
        }
      }
      int ra = 0, rb = rows;
      if (cluster) {
        pair_bar();   // (both halves have read the sums)
        if (hf == 0) xm[r] = make_float2(m_out, l_out);
        cluster_sync();   // (the other roles arrive below)
        const int share = (rows + a.splits - 1) / a.splits;
        ra = split * share;
        rb = min(rows, ra + share);
      } else {
        if (hf == 0) __stcg(a.part_ml + (unit * a.splits + split) * BM + r, make_float2(m_out, l_out));
        __threadfence();
        asm volatile("bar.sync 5, 256;" ::: "memory");
        if (threadIdx.x == 0) *last_flag = atomicInc(a.arrived + unit, (unsigned)a.splits - 1u) == (unsigned)a.splits - 1u;
        asm volatile("bar.sync 5, 256;" ::: "memory");
        if (!*last_flag) rb = 0;
        __threadfence();
      }
      const bool wide = ((uintptr_t)a.out | (uintptr_t)(a.out_robot * 2) | (uintptr_t)(a.out_token * 2)) % 16 == 0;
      // the splits' weights per row, [splits][128], into Q's place (every S has completed)
      // or, where they may be many, the rings' ...
      float* wts = (float*)(smem + (cluster ? 0 : NB * QB));
      for (int rr = ra + threadIdx.x; rr < rb; rr += 256) {
        const uint32_t xml = smem_u32(xm) + 8u * rr;
        const float2* ml = a.part_ml + unit * a.splits * BM + rr;
        float M = -INFINITY, S = 0.f;
        for (int q = 0; q < a.splits; ++q)
          M = fmaxf(M, cluster ? ld_cluster_f2(mapa_shared(xml, (uint32_t)q)).x : __ldcg(ml + q * BM).x);
        for (int q = 0; q < a.splits; ++q) {
          const float2 x = cluster ? ld_cluster_f2(mapa_shared(xml, (uint32_t)q)) : __ldcg(ml + q * BM);
          const float wt = x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y);
          wts[q * BM + rr] = wt;
          S += wt;
        }
        const float si = !(S <= 0.f) ? 1.f / S : 0.f;
        for (int q = 0; q < a.splits; ++q) wts[q * BM + rr] *= si;
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
              y0 = __ldcg(y);
              y1 = __ldcg(y + 1);
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
          store_bf16x8(out_row(r0 + rr) + 8 * lane,
                       make_uint4(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]), pack_bf16x2(acc[4], acc[5]),
                                  pack_bf16x2(acc[6], acc[7])),
                       wide);
        }
      }
      if (cluster) cluster_sync();   // nobody leaves while its rows are read
    }
  }
  if (warp >= 8 && a.splits > 1 && a.splits <= kTcCluster) {
    cluster_sync();
    cluster_sync();
  }
  tc_fence_before();
  cta_sync();
  if (*abort_flag && threadIdx.x == 0) {
    // loads still on their way, at most the last CS, land before the shared memory goes away
    for (int q = 0; q < 2; ++q)
      for (int i = max(0, c_issued[q] - CS); i < c_issued[q]; ++i) mbar_wait(&c_full[q * CS + i % CS], (uint32_t)(i / CS) & 1u);
    raise_error(a.err, ERR_TIMEOUT);
  }
  if (warp == 16)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

PFN_cuTensorMapEncodeTiled_v12000 g_enc = nullptr;

cudaError_t encode_codes(CUtensorMap* m, const uint8_t* base, const CacheLayer& c, int batch) {
  cuuint64_t dims[2] = {(cuuint64_t)c.hdp, (cuuint64_t)batch * c.Hkv * c.T};
  cuuint64_t strides[1] = {(cuuint64_t)c.hdp};
  cuuint32_t box[2] = {64u, 64u}, estr[2] = {1, 1};
  const CUresult r = g_enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
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
  TcMaps maps;
  cudaError_t e = encode_codes(&maps.k, a.c.k, a.c, a.batch);
  if (e == cudaSuccess) e = encode_codes(&maps.v, a.c.v, a.c, a.batch);
  if (e != cudaSuccess) return e;
  return launch_kernel_cluster(cache_tc_kernel<NB>, dim3(a.row_tiles * a.splits, a.c.Hkv, a.batch), dim3(TCT),
                               TcShape<NB>::bytes, st, dim3(a.splits <= kTcCluster ? a.splits : 1, 1, 1), maps, a);
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

cudaError_t launch_cache_attend_tc(const CacheAttnArgs& a, cudaStream_t st) {
  switch (a.c.hdp) {
    case 64: return launch_nb<1>(a, st);
    case 128: return launch_nb<2>(a, st);
    case 192: return launch_nb<3>(a, st);
    default: return launch_nb<4>(a, st);
  }
}

cudaError_t init_cache_tc_kernels(int hdp, int* clusters) {
  if (!g_enc) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
    if (e != cudaSuccess) return e;
    if (q != cudaDriverEntryPointSuccess || !fn) return cudaErrorSymbolNotFound;
    g_enc = (PFN_cuTensorMapEncodeTiled_v12000)fn;
  }
  switch (hdp) {
    case 64: return init_nb<1>(clusters);
    case 128: return init_nb<2>(clusters);
    case 192: return init_nb<3>(clusters);
    default: return init_nb<4>(clusters);
  }
}

}  // namespace ravel
