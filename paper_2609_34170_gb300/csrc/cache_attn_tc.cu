// Attention over the 8-bit context cache for many query rows (an expert's slots,
// prompts), bf16, on the 5th-generation tensor cores.
//
// A CTA owns 128 rows (row r = query * G + head of the group) of one (robot, KV
// head) and a share (split) of the 128-token tiles that they see:
//   S = Q K^T        tcgen05.mma kind::f16, M = 128, N = 128, into TMEM
//   P = 2^(S - m)    softmax warps: TMEM -> registers -> f16 P over S in TMEM
//   O += P V         tcgen05.mma, M = 128, N = head dim, 16 tokens at a time
// Warp roles (416 threads): warps 0-7 softmax and epilogue, two threads per row;
// warps 8, 9 widen K, warps 10, 11 widen V; warp 12 TMEM and MMAs.
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

namespace ravel {
namespace {

constexpr int TCT = 416;
constexpr int BM = 128, BT = 128;              // rows, tokens of a tile
constexpr uint32_t QB = BM * 128;              // bytes of a 64-dim block of Q
constexpr uint32_t KU = BT * 128;              // bytes of a K unit: 128 tokens x 64 dims
constexpr uint32_t VB = 64 * 128;              // bytes of a 64-dim block of a V half
constexpr float kTcShift = 7.f;                // P's largest value is 2^kTcShift (times 2^8 while lazy)
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
  uint64_t* ended = pv_done + 2;
  uint32_t* tmem_slot = (uint32_t*)(ended + 1);
  int* abort_flag = (int*)(tmem_slot + 1);
  int* last_flag = abort_flag + 1;
  uint32_t* row_top = (uint32_t*)(tail + 512);    // [128] bits of the rows' largest |q|
  float2* xm = (float2*)(tail + 1024);            // [2][128] row maxima, then sums, of the two halves
  static_assert((2 * 8 + 2 * 4 + 7) * 8 + 12 <= 512, "barriers");

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
      mbar_init(&k_full[i], 2);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < VS; ++i) {
      mbar_init(&v_full[i], 2);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 256);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(ended, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x < BM) row_top[threadIdx.x] = 0u;
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  cta_sync();
  {
    // Q: the rows' 16-dim pieces, loaded once, scaled by their row's power of two
    constexpr int PIECES = BM * 4 * NB, PER = (PIECES + TCT - 1) / TCT;
    uint4 raw[PER][2];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int x = threadIdx.x + p * TCT;
      const int r = x / (4 * NB), d = x % (4 * NB) * 16, i = (r0 + r) / a.G;
      raw[p][0] = raw[p][1] = make_uint4(0u, 0u, 0u, 0u);
      if (x < PIECES && i < s.count) {
        const bf16* row = (const bf16*)a.q + (size_t)((long long)b * a.q_robot + (long long)i * a.q_token) +
                          (size_t)(h * a.G + (r0 + r) % a.G) * L.hd + d;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (d + 8 * e >= L.hd) continue;
          if (a.vec) {
            raw[p][e] = __ldg((const uint4*)row + e);
          } else {
            bf16 y[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) y[z] = row[8 * e + z];
            memcpy(&raw[p][e], y, 16);
          }
        }
        uint32_t top = 0u;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t u[4] = {raw[p][e].x, raw[p][e].y, raw[p][e].z, raw[p][e].w};
#pragma unroll
          for (int z = 0; z < 4; ++z) top = max(top, max((u[z] & 0x7fffu) << 16, u[z] & 0x7fff0000u));
        }
        atomicMax(&row_top[r], top);
      }
    }
    cta_sync();
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int x = threadIdx.x + p * TCT;
      if (x < PIECES) {
        const int r = x / (4 * NB), c = x % (4 * NB);
        const uint32_t top = row_top[r];
        const float f = top >= 0x7f800000u ? __int_as_float(0x7fffffff) : exp2i(min(14 - ((int)(top >> 23) - 127), 126));
        const uint32_t at = q0 + (uint32_t)(c / 4) * QB + (uint32_t)r * 128u;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t u[4] = {raw[p][e].x, raw[p][e].y, raw[p][e].z, raw[p][e].w};
          uint32_t w[4];
#pragma unroll
          for (int z = 0; z < 4; ++z)
            w[z] = pack_f16x2(__uint_as_float(u[z] << 16) * f, __uint_as_float(u[z] & 0xffff0000u) * f);
          sts_u4(at + (uint32_t)((((c & 3) * 2 + e) ^ (r & 7)) * 16), make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t o_col = 2 * BT;

  if (warp == 8 || warp == 9) {
    // ---- K: units of 64 dims, the next one's codes in flight
    const int ct = threadIdx.x - 8 * 32;
    const uint8_t* src = L.k + head * L.T * HDP + (size_t)(ct >> 2) * HDP + 16 * (ct & 3);
    const uint32_t sw = (uint32_t)(ct >> 2) & 7u, row = (uint32_t)(ct >> 2) * 128u;
    const uint32_t lo = row + ((((uint32_t)ct & 3u) * 2u) ^ sw) * 16u, hi = row + ((((uint32_t)ct & 3u) * 2u + 1u) ^ sw) * 16u;
    uint4 cur[8], nxt[8];
    auto load = [&](uint4* x, int t, int blk) {
      const uint8_t* at = src + (size_t)tile_token(t) * HDP + 64 * blk;
#pragma unroll
      for (int y = 0; y < 8; ++y) x[y] = __ldg((const uint4*)(at + (size_t)(16 * y) * HDP));
    };
    int slot = 0, t = t0, blk = 0;
    uint32_t ph = 1;
    bool ok = true;
    if (n > 0) load(nxt, t, 0);
    while (ok && t < t1) {
#pragma unroll
      for (int y = 0; y < 8; ++y) cur[y] = nxt[y];
      if (++blk == NB) {
        blk = 0;
        ++t;
      }
      if (t < t1) load(nxt, t, blk);
      ok = mbar_wait_warp(&k_empty[slot], ph);
      const uint32_t to = k0 + (uint32_t)slot * KU;
#pragma unroll
      for (int y = 0; y < 8; ++y) widen(cur[y], to + lo + 2048u * y, to + hi + 2048u * y);
      written(&k_full[slot]);
      if (++slot == KS) {
        slot = 0;
        ph ^= 1u;
      }
    }
    if (!ok && lane == 0) *abort_flag = 1;
  } else if (warp == 10 || warp == 11) {
    // ---- V: halves of 64 tokens, in steps of SB blocks of 64 dims
    constexpr int SB = NB == 3 ? 1 : (NB == 1 ? 1 : 2), STEPS = NB / SB;
    const int ct = threadIdx.x - 10 * 32;
    const uint8_t* src = L.v + head * L.T * HDP + (size_t)(ct >> 2) * HDP + 16 * (ct & 3);
    const uint32_t sw = (uint32_t)(ct >> 2) & 7u, row = (uint32_t)(ct >> 2) * 128u;
    const uint32_t lo = row + ((((uint32_t)ct & 3u) * 2u) ^ sw) * 16u, hi = row + ((((uint32_t)ct & 3u) * 2u + 1u) ^ sw) * 16u;
    uint4 cur[4 * SB], nxt[4 * SB];
    auto load = [&](uint4* x, int t, int half, int step) {
      const uint8_t* at = src + (size_t)(tile_token(t) + 64 * half) * HDP + 64 * SB * step;
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int z = 0; z < SB; ++z) x[SB * y + z] = __ldg((const uint4*)(at + (size_t)(16 * y) * HDP + 64 * z));
    };
    int slot = 0, t = t0, half = 0, step = 0;
    uint32_t ph = 1;
    bool ok = true;
    if (n > 0) load(nxt, t, 0, 0);
    while (ok && t < t1) {
#pragma unroll
      for (int y = 0; y < 4 * SB; ++y) cur[y] = nxt[y];
      const int now = step;
      if (++step == STEPS) {
        step = 0;
        if (half == 0 && keys_of(tile_token(t)) > 64) {
          half = 1;
        } else {
          half = 0;
          ++t;
        }
      }
      if (t < t1) load(nxt, t, half, step);
      if (now == 0) ok = mbar_wait_warp(&v_empty[slot], ph);
      const uint32_t to = v0 + (uint32_t)slot * VH + (uint32_t)(now * SB) * VB;
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int z = 0; z < SB; ++z) widen(cur[SB * y + z], to + lo + 2048u * y + VB * z, to + hi + 2048u * y + VB * z);
      if (now == STEPS - 1) {
        written(&v_full[slot]);
        if (++slot == VS) {
          slot = 0;
          ph ^= 1u;
        }
      }
    }
    if (!ok && lane == 0) *abort_flag = 1;
  } else if (warp == 12) {
    // ---- MMAs: S of the next tile as soon as its K is there, P V of the oldest whose P is
    const uint32_t el = elect_one();
    const uint32_t idesc_s = idesc_f16(BM, BT), idesc_o = idesc_f16(BM, HDP) | (1u << 16);
    const uint64_t qd0 = sw128_desc(q0), kd0 = sw128_desc(k0), vd0 = sw128_mn_desc(v0, VB);
    int ns = 0, i = 0, sk = 0, sv = 0;
    uint32_t phk = 0, phv = 0, spins = 0;
    bool ok = true;
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
  } else {
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
      const int per = L.hd / 8;   // 16-byte pieces of a row
      const bool wide = ((uintptr_t)a.out | (uintptr_t)(a.out_robot * 2) | (uintptr_t)(a.out_token * 2)) % 16 == 0;
      for (int x = threadIdx.x; x < rows * per; x += 256) {
        const int rr = x / per, c = x % per;
        const uint4 w = *(const uint4*)(smem + (size_t)(c >> 3) * QB + (size_t)rr * 128 + (((c & 7) ^ (rr & 7)) * 16));
        bf16* dst = out_row(r0 + rr) + 8 * c;
        if (wide) {
          *(uint4*)dst = w;
        } else {
          bf16 y[8];
          memcpy(y, &w, 16);
#pragma unroll
          for (int z = 0; z < 8; ++z) dst[z] = y[z];
        }
      }
    } else {
      // partial [d / 4][row][4], normalised, with its (max, sum); the last split joins them in order
      const size_t unit = head * a.row_tiles + tile, at = unit * a.splits + split;
      float* part = a.part + at * BM * HDP;
      for (int cb = 32 * hf; cb < HDP; cb += 64) {
        uint32_t raw[32];
        tmem_ld32_async(lane_base + o_col + cb, raw);
        tmem_wait_ld();
        tmem_reg_fence16(raw);
        tmem_reg_fence16(raw + 16);
#pragma unroll
        for (int q = 0; q < 8; ++q)
          __stcg((float4*)(part + ((size_t)(cb / 4 + q) * BM + r) * 4),
                 real ? make_float4(__uint_as_float(raw[4 * q]) * inv, __uint_as_float(raw[4 * q + 1]) * inv,
                                    __uint_as_float(raw[4 * q + 2]) * inv, __uint_as_float(raw[4 * q + 3]) * inv)
                      : make_float4(0.f, 0.f, 0.f, 0.f));
      }
      if (hf == 0) __stcg(a.part_ml + at * BM + r, make_float2(m_out, l_out));
      __threadfence();
      asm volatile("bar.sync 5, 256;" ::: "memory");
      if (threadIdx.x == 0) *last_flag = atomicInc(a.arrived + unit, (unsigned)a.splits - 1u) == (unsigned)a.splits - 1u;
      asm volatile("bar.sync 5, 256;" ::: "memory");
      if (*last_flag) {
        __threadfence();
        const float2* ml = a.part_ml + unit * a.splits * BM + r;
        float M = -INFINITY, S = 0.f;
        for (int q = 0; q < a.splits; ++q) M = fmaxf(M, __ldcg(ml + q * BM).x);
        for (int q = 0; q < a.splits; ++q) {
          const float2 x = __ldcg(ml + q * BM);
          S += x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y);
        }
        const float si = !(S <= 0.f) ? 1.f / S : 0.f;
        if (a.mass && hf == 0 && r < rows) a.row_ml[head * a.n * a.G + r0 + r] = row_weight(M, S, kTcShift);
        const float* p0 = a.part + unit * a.splits * BM * HDP;
        bf16* dst = out_row(r0 + min(r, rows - 1));
        for (int d4 = hf; d4 < L.hd / 4; d4 += 2) {
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int q = 0; q < a.splits; ++q) {
            const float2 x = __ldcg(ml + q * BM);
            const float wt = (x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y)) * si;
            const float4 y = __ldcg((const float4*)(p0 + (size_t)q * BM * HDP + ((size_t)d4 * BM + r) * 4));
            acc.x += wt * y.x;
            acc.y += wt * y.y;
            acc.z += wt * y.z;
            acc.w += wt * y.w;
          }
          if (r < rows) {
            bf16* o = dst + 4 * d4;
            o[0] = __float2bfloat16_rn(acc.x);
            o[1] = __float2bfloat16_rn(acc.y);
            o[2] = __float2bfloat16_rn(acc.z);
            o[3] = __float2bfloat16_rn(acc.w);
          }
        }
      }
    }
  }
  tc_fence_before();
  cta_sync();
  if (*abort_flag && threadIdx.x == 0) raise_error(a.err, ERR_TIMEOUT);
  if (warp == 12)
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
  cache_tc_kernel<NB><<<dim3(a.row_tiles * a.splits, a.c.Hkv, a.batch), TCT, TcShape<NB>::bytes, st>>>(a);
  return cudaGetLastError();
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
