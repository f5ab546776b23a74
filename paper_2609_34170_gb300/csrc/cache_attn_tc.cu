// Attention over the 8-bit context cache for many query rows (an expert's slots,
// prompts), bf16, on the 5th-generation tensor cores.
//
// A CTA owns 128 rows (row r = query * G + head of the group) of one (robot, KV
// head) and a share (split) of the 128-token tiles that they see:
//   S = Q K^T        tcgen05.mma kind::f16, M = 128, N = 128, into TMEM
//   P = 2^(S - m)    softmax warps: TMEM -> registers -> f16 P over S in TMEM
//   O += P V         tcgen05.mma, M = 128, N = head dim, 16 tokens at a time
// Warp roles (640 threads): warps 0-7 Q, softmax and epilogue, two threads per row;
// warps 8-11 widen K, warps 12-15 widen V; warp 16 TMEM and MMAs (17-19 idle, so
// that registers can be moved between whole warpgroups).
//
// The codes go from global memory through the widening warps' registers into
// shared memory as f16 (e4m3 -> f16 is exact), in the 128-byte swizzled layout
// that a TMA load of f16 rows would leave: K in units of 64 head dims (16 KB),
// V in halves of 64 tokens, each in a ring of its own with its own producers, so
// that neither waits for the other's slots.  Feeding the codes as kind::f8f6f4
// operands instead would need Q and P in 8 bits too: two pieces of each keep
// bf16's precision and cost what one f16 MMA does, but 2^-9 is the least P that
// e4m3 holds, and a long flat tail of smaller ones carries weight.
//
// Numbers as in the kernel for few rows: q in f16 under a power of two per row
// (exact for bf16), block exponents of K on the scores, those of V on P.  P is at
// most 2^7 of the reference, 2^15 while a grown one waits for its rescaling of O
// (only growth by more than 2^8 rescales); what contributes less than 2^-31 of the
// row's largest is dropped.
#include <algorithm>

#include "cache_attn.cuh"
#include "launch.h"

namespace ravel {
namespace {

constexpr int TCT = 640;
constexpr int BM = 128, BT = 128;              // rows, tokens of a tile
constexpr uint32_t QB = BM * 128;              // bytes of a 64-dim block of Q
constexpr uint32_t KU = BT * 128;              // bytes of a K unit: 128 tokens x 64 dims
constexpr uint32_t VB = 64 * 128;              // bytes of a 64-dim block of a V half
constexpr float kTcShift = 7.f;                // P's largest value is 2^kTcShift (times 2^8 while lazy)
constexpr int kTcCluster = 8;                  // splits that are a cluster
constexpr uint32_t kPolls = 1u << 25;          // polls without progress: seconds

template <int NB> struct TcShape {
  // shared memory at NB blocks of 64 head dims: Q NB x 16 KB, then the rings
  static constexpr int KS = NB == 4 ? 4 : (NB == 3 ? 5 : 2 * NB);
  static constexpr int VS = NB == 4 ? 3 : 4;
  static constexpr uint32_t bytes = NB * QB + KS * KU + VS * NB * VB + 3072;
};
static_assert(TcShape<4>::bytes <= 227 * 1024 && TcShape<3>::bytes <= 227 * 1024, "shared memory");

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

// codes: read once by this CTA, by others of the same (robot, KV head) from L2
__device__ __forceinline__ uint4 ldg_codes(const uint8_t* p) { return __ldg((const uint4*)p); }

// A warp's writes to shared memory become visible to the tensor core: one arrival per warp.
__device__ __forceinline__ void written(uint64_t* bar) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

template <int NB>
__global__ void __launch_bounds__(TCT, 1) cache_tc_kernel(CacheAttnArgs a) {
  constexpr int HDP = 64 * NB, KS = TcShape<NB>::KS, VS = TcShape<NB>::VS;
  constexpr uint32_t VH = NB * VB;   // bytes of a V half
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t q0 = smem_u32(smem), k0 = q0 + NB * QB, v0 = k0 + KS * KU;
  uint8_t* tail = smem + NB * QB + KS * KU + VS * VH;
  uint64_t* k_full = (uint64_t*)tail;
  uint64_t* k_empty = k_full + KS;
  uint64_t* v_full = k_empty + KS;
  uint64_t* v_empty = v_full + VS;
  uint64_t* s_full = v_empty + VS;   // [2]
  uint64_t* p_full = s_full + 2;     // [2]
  uint64_t* pv_done = p_full + 2;    // [2]
  uint64_t* q_full = pv_done + 2;
  uint64_t* ended = q_full + 1;
  uint32_t* tmem_slot = (uint32_t*)(ended + 1);
  int* abort_flag = (int*)(tmem_slot + 1);
  int* last_flag = abort_flag + 1;
  uint32_t* row_top = (uint32_t*)(tail + 512);    // [128] bits of the rows' largest |q|
  float2* xm = (float2*)(tail + 1024);            // [2][128] row maxima, then sums, of the two halves
  static_assert((2 * 8 + 2 * 4 + 8) * 8 + 12 <= 512, "barriers");

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
  auto out_row = [&](int r) { return out0 + (size_t)((long long)(r / a.G) * a.out_token) + (size_t)(r % a.G) * L.hd; };
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
      mbar_init(&k_full[i], 4);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < VS; ++i) {
      mbar_init(&v_full[i], 4);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
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
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t o_col = 2 * BT;

  if (warp >= 8 && warp < 16) {
    regs_down<80>();
    // ---- widening: K in units of 64 dims (warps 8-11), V in halves of 64 tokens (12-15),
    // thread ct: 16 codes at dim 16 (ct % 4) of rows ct / 4, ct / 4 + 32, ...; the codes of
    // the next two steps are in flight (a step's latency is several times its work)
    const bool is_k = warp < 12;
    const int ct = (threadIdx.x - 256) & 127;
    const uint8_t* src = (is_k ? L.k : L.v) + head * L.T * HDP + (size_t)(ct >> 2) * HDP + 16 * (ct & 3);
    const uint32_t sw = (uint32_t)(ct >> 2) & 7u, row = (uint32_t)(ct >> 2) * 128u;
    const uint32_t lo = row + ((((uint32_t)ct & 3u) * 2u) ^ sw) * 16u, hi = row + ((((uint32_t)ct & 3u) * 2u + 1u) ^ sw) * 16u;
    int slot = 0;
    uint32_t ph = 1;
    bool ok = true;
    if (is_k) {
      uint4 x0[4], x1[4], x2[4];
      int t = t0, blk = 0;   // the unit to load next
      auto load = [&](uint4(&x)[4]) {
        if (t >= t1) return;
        const uint8_t* at = src + (size_t)tile_token(t) * HDP + 64 * blk;
#pragma unroll
        for (int y = 0; y < 4; ++y) x[y] = ldg_codes(at + (size_t)(32 * y) * HDP);
        if (++blk == NB) {
          blk = 0;
          ++t;
        }
      };
      auto put = [&](const uint4(&x)[4]) {
        ok = mbar_wait_warp(&k_empty[slot], ph);
        const uint32_t to = k0 + (uint32_t)slot * KU;
#pragma unroll
        for (int y = 0; y < 4; ++y) widen(x[y], to + lo + 4096u * y, to + hi + 4096u * y);
        written(&k_full[slot]);
        if (++slot == KS) {
          slot = 0;
          ph ^= 1u;
        }
      };
      load(x0);
      load(x1);
      int left = n * NB;
      while (left > 0) {
        load(x2);
        put(x0);
        if (!ok || --left == 0) break;
        load(x0);
        put(x1);
        if (!ok || --left == 0) break;
        load(x1);
        put(x2);
        if (!ok) break;
        --left;
      }
    } else {
      // a step: two blocks of 64 dims of a half (one, where their number is odd)
      constexpr int SB = NB % 2 ? 1 : 2, STEPS = NB / SB;
      uint4 x0[2 * SB], x1[2 * SB], x2[2 * SB];
      int t = t0, half = 0, step = 0;   // the step to load next
      auto load = [&](uint4(&x)[2 * SB]) {
        if (t >= t1) return;
        const int j0 = tile_token(t);
        const uint8_t* at = src + (size_t)(j0 + 64 * half) * HDP + 64 * SB * step;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int z = 0; z < SB; ++z) x[SB * y + z] = ldg_codes(at + (size_t)(32 * y) * HDP + 64 * z);
        if (++step == STEPS) {
          step = 0;
          if (half == 0 && keys_of(j0) > 64) {
            half = 1;
          } else {
            half = 0;
            ++t;
          }
        }
      };
      int now = 0;
      auto put = [&](const uint4(&x)[2 * SB]) {
        if (now == 0) ok = mbar_wait_warp(&v_empty[slot], ph);
        const uint32_t to = v0 + (uint32_t)slot * VH + (uint32_t)(now * SB) * VB;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int z = 0; z < SB; ++z) widen(x[SB * y + z], to + lo + 4096u * y + VB * z, to + hi + 4096u * y + VB * z);
        if (++now == STEPS) {
          now = 0;
          written(&v_full[slot]);
          if (++slot == VS) {
            slot = 0;
            ph ^= 1u;
          }
        }
      };
      int left = 0;
      for (int q = t0; q < t1; ++q) left += keys_of(tile_token(q)) > 64 ? 2 * STEPS : STEPS;
      load(x0);
      load(x1);
      while (left > 0) {
        load(x2);
        put(x0);
        if (!ok || --left == 0) break;
        load(x0);
        put(x1);
        if (!ok || --left == 0) break;
        load(x1);
        put(x2);
        if (!ok) break;
        --left;
      }
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
    }
  } else {
    regs_up<144>();
    // ---- Q: rows of 8 NB lanes with 8 dims each, scaled by their power of two
    {
      constexpr int LPR = 8 * NB, RPW = 32 / LPR, PASS = 16 / RPW, AHEAD = PASS < 8 ? PASS : 8;
      const int sub = lane / LPR, dl = lane % LPR;
      const bool on = sub < RPW && 8 * dl < L.hd;
      for (int p0 = 0; p0 < PASS; p0 += AHEAD) {
        uint4 x[AHEAD];
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
          const int r = r0 + warp * 16 + (p0 + p) * RPW + sub, i = r / a.G;
          x[p] = make_uint4(0u, 0u, 0u, 0u);
          if (on && i < s.count) {
            const bf16* at = (const bf16*)a.q + (size_t)((long long)b * a.q_robot + (long long)i * a.q_token) +
                             (size_t)(h * a.G + r % a.G) * L.hd + 8 * dl;
            if (a.vec) {
              x[p] = __ldg((const uint4*)at);
            } else {
              bf16 y[8];
#pragma unroll
              for (int z = 0; z < 8; ++z) y[z] = at[z];
              memcpy(&x[p], y, 16);
            }
          }
        }
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
          const uint32_t u[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
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
          for (int z = 0; z < 4; ++z)
            w[z] = pack_f16x2(__uint_as_float(u[z] << 16) * f, __uint_as_float(u[z] & 0xffff0000u) * f);
          const int lr = warp * 16 + (p0 + p) * RPW + sub;
          if (sub < RPW) sts_u4(q0 + (uint32_t)(dl >> 3) * QB + (uint32_t)lr * 128u + (uint32_t)(((dl & 7) ^ (lr & 7)) * 16),
                                make_uint4(w[0], w[1], w[2], w[3]));
          if (sub < RPW && dl == 0) row_top[lr] = top;
        }
      }
      written(q_full);
      asm volatile("bar.sync 5, 256;" ::: "memory");   // row_top
    }
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
      for (int rr = warp; rr < rows; rr += 8) {
        bf16* dst = out_row(r0 + rr) + 8 * lane;
        if (8 * lane < L.hd) {
          const uint4 w = *(const uint4*)(smem + (size_t)(lane >> 3) * QB + (size_t)rr * 128 + (((lane & 7) ^ (rr & 7)) * 16));
          store_bf16x8(dst, w, wide);
        }
      }
    } else {
      // partial [row][d], normalised, with its (max, sum)
      const size_t unit = head * a.row_tiles + tile, at = unit * a.splits + split;
      float* part = a.part + (at * BM + r) * HDP;
      for (int cb = 32 * hf; cb < HDP; cb += 64) {
        uint32_t raw[32];
        tmem_ld32_async(lane_base + o_col + cb, raw);
        tmem_wait_ld();
        tmem_reg_fence16(raw);
        tmem_reg_fence16(raw + 16);
        if (r < rows) {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            __stcg((float4*)(part + cb + 4 * q),
                   real ? make_float4(__uint_as_float(raw[4 * q]) * inv, __uint_as_float(raw[4 * q + 1]) * inv,
                                      __uint_as_float(raw[4 * q + 2]) * inv, __uint_as_float(raw[4 * q + 3]) * inv)
                        : make_float4(0.f, 0.f, 0.f, 0.f));
        }
      }
      if (hf == 0) __stcg(a.part_ml + at * BM + r, make_float2(m_out, l_out));
      __threadfence();
      // the splits' partials joined in their order: up to 8 splits are a cluster, each of
      // which joins a share of the rows once all have stored; of more, the last to arrive
      // joins all rows
      int ra = 0, rb = rows;
      if (a.splits <= kTcCluster) {
        cluster_sync();   // (the other roles arrive below)
        const int share = (rows + a.splits - 1) / a.splits;
        ra = split * share;
        rb = min(rows, ra + share);
      } else {
        asm volatile("bar.sync 5, 256;" ::: "memory");
        if (threadIdx.x == 0) *last_flag = atomicInc(a.arrived + unit, (unsigned)a.splits - 1u) == (unsigned)a.splits - 1u;
        asm volatile("bar.sync 5, 256;" ::: "memory");
        if (!*last_flag) rb = 0;
      }
      __threadfence();
      {
        const bool wide = ((uintptr_t)a.out | (uintptr_t)(a.out_robot * 2) | (uintptr_t)(a.out_token * 2)) % 16 == 0;
        for (int rr = ra + warp; rr < rb; rr += 8) {
          const float2* ml = a.part_ml + unit * a.splits * BM + rr;
          const float* p0 = a.part + (unit * a.splits * BM + rr) * HDP + 8 * lane;
          const bool on = 8 * lane < L.hd;
          float M = -INFINITY, S = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          for (int q = 0; q < a.splits; ++q) M = fmaxf(M, __ldcg(ml + q * BM).x);
  #pragma unroll 4
          for (int q = 0; q < a.splits; ++q) {
            const float2 x = __ldcg(ml + q * BM);
            const float wt = x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y);
            S += wt;
            if (on) {
              const float4* y = (const float4*)(p0 + (size_t)q * BM * HDP);
              const float4 y0 = __ldcg(y), y1 = __ldcg(y + 1);
              acc[0] = fmaf(wt, y0.x, acc[0]);
              acc[1] = fmaf(wt, y0.y, acc[1]);
              acc[2] = fmaf(wt, y0.z, acc[2]);
              acc[3] = fmaf(wt, y0.w, acc[3]);
              acc[4] = fmaf(wt, y1.x, acc[4]);
              acc[5] = fmaf(wt, y1.y, acc[5]);
              acc[6] = fmaf(wt, y1.z, acc[6]);
              acc[7] = fmaf(wt, y1.w, acc[7]);
            }
          }
          const float si = !(S <= 0.f) ? 1.f / S : 0.f;
          if (a.mass && lane == 0) a.row_ml[head * a.n * a.G + r0 + rr] = row_weight(M, S, kTcShift);
          if (on)
            store_bf16x8(out_row(r0 + rr) + 8 * lane,
                         make_uint4(pack_bf16x2(acc[0] * si, acc[1] * si), pack_bf16x2(acc[2] * si, acc[3] * si),
                                    pack_bf16x2(acc[4] * si, acc[5] * si), pack_bf16x2(acc[6] * si, acc[7] * si)),
                         wide);
        }
      }
    }
  }
  if (warp >= 8 && a.splits > 1 && a.splits <= kTcCluster) cluster_sync();
  tc_fence_before();
  cta_sync();
  if (*abort_flag && threadIdx.x == 0) raise_error(a.err, ERR_TIMEOUT);
  if (warp == 16)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int NB>
cudaError_t launch_nb(CacheAttnArgs a, cudaStream_t st) {
  a.row_tiles = (a.n * a.G + BM - 1) / BM;
  const long long tiles = (long long)a.row_tiles * a.c.Hkv * a.batch;
  long long seen = a.max_length;
  if (a.window > 0) seen = std::min(seen, (long long)a.window + a.sinks + BM / a.G + 1 + 2 * BT);
  const long long units = (seen + BT - 1) / BT;
  a.splits = (int)std::max(1ll, std::min((long long)a.num_sms / tiles, units));
  return launch_kernel_cluster(cache_tc_kernel<NB>, dim3(a.row_tiles * a.splits, a.c.Hkv, a.batch), dim3(TCT),
                               TcShape<NB>::bytes, st, dim3(a.splits <= kTcCluster ? a.splits : 1, 1, 1), a);
}

template <int NB>
cudaError_t init_nb() {
  return cudaFuncSetAttribute(cache_tc_kernel<NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<NB>::bytes);
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

cudaError_t init_cache_tc_kernels() {
  cudaError_t e = init_nb<1>();
  if (e == cudaSuccess) e = init_nb<2>();
  if (e == cudaSuccess) e = init_nb<3>();
  if (e == cudaSuccess) e = init_nb<4>();
  return e;
}

}  // namespace ravel
