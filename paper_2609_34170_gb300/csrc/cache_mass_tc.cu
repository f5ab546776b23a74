// Attention mass of the cached tokens for many query rows, bf16, on the 5th-generation
// tensor cores: token j's softmax weights, 2^(s - x) y with the rows' (x, y) that the
// attention left behind, summed over the rows of its KV head.
//
// The scores are computed again, transposed -- D = K Q^T, tokens on the lanes, rows on
// the columns -- so that a token's sum is one thread's.  What that costs is half an
// attention without the softmax's rescaling and P V; keeping the scores instead would
// take 4 bytes for each of them (8 heads x 816 queries x 816 tokens: 21 MB a robot)
// and a pass over them.  A CTA owns a chunk of a (robot, KV head)'s row tiles and adds
// up in a place of its own, chunks are summed in their order: no order of arrival
// enters the result.
//
// Warp roles (640 threads): warps 0-7 exponentials and sums, two threads per token, 64
// rows each; 8-15 lay out Q, a tile ahead; 16 TMEM and MMAs; 17 loads K (18, 19 idle).
// The exponentials bound it at head dim 64, the MMAs' reads of shared memory at 256.
// Measured: 4 robots x 816 queries x 816 tokens, 8 heads of 256: 26.7 us and 4 for the sums,
// beside 35.4 for the attention.
#include <algorithm>

#include "cache_index.h"
#include "cache_tc.cuh"
#include "launch.h"

namespace ravel {
namespace {

constexpr int MT = 640;

template <int NB> struct MassShape {
  static constexpr int KS = 8;                              // K units in flight
  static constexpr uint32_t q_bytes = 2 * NB * QB;          // a tile of rows in two pieces
  static constexpr uint32_t bytes = 2 * q_bytes + KS * KU + 4096 + 2048 + 512;
  static_assert(bytes <= 227 * 1024, "shared memory");
};

struct MassMaps {
  CUtensorMap k;   // a layer's keys [B Hkv T][hdp]: boxes of 64 dims x 128 rows (swizzled)
};

template <int NB>
__global__ void __launch_bounds__(MT, 1) cache_mass_tc_kernel(const __grid_constant__ MassMaps maps, CacheAttnArgs a) {
  using Shape = MassShape<NB>;
  constexpr int KS = Shape::KS;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t q0 = smem_u32(smem), k0 = q0 + 2 * Shape::q_bytes;
  uint8_t* tail = smem + 2 * Shape::q_bytes + KS * KU;
  // per row (factor, -x) and y, [4][128] by row tile: Q is laid out up to two tiles ahead of the
  // exponentials, which may be two tiles of scores behind the MMAs.  (x is integral: the
  // exponent s - x is rounded once, where log2 y - x would bring a row's own rounding into it.)
  float2* rowc = (float2*)tail;
  float* rowy = (float*)(tail + 4096);
  uint64_t* k_full = (uint64_t*)(tail + 4096 + 2048);
  uint64_t* k_empty = k_full + KS;
  uint64_t* q_full = k_empty + KS;   // [2]
  uint64_t* q_empty = q_full + 2;    // [2]
  uint64_t* s_full = q_empty + 2;    // [2]
  uint64_t* s_free = s_full + 2;     // [2]
  uint64_t* ended = s_free + 2;
  uint32_t* tmem_slot = (uint32_t*)(ended + 1);
  int* abort_flag = (int*)(tmem_slot + 1);
  int* issued_flag = abort_flag + 1;
  static_assert((2 * KS + 9) * 8 + 12 <= 512, "barriers");

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const CacheLayer& L = a.c;
  const int chunk = blockIdx.x % a.splits, head = blockIdx.x / a.splits, b = head / L.Hkv, h = head % L.Hkv;
  pdl_wait();   // (before any TMEM is taken)
  Sight s;
  robot_sight(a, b, s);   // (the attention before has reported what is out of range)
  const int end_row = s.count * a.G;
  // this chunk's row tiles that see something
  const int rt0 = (int)((long long)a.row_tiles * chunk / a.splits);
  const int rt1 = s.len == 0 ? rt0 : min((int)((long long)a.row_tiles * (chunk + 1) / a.splits), (end_row + BM - 1) / BM);
  float* part = a.mass_ws + (size_t)blockIdx.x * 2 * a.mass_pitch;
  for (long long x = threadIdx.x; x < 2 * a.mass_pitch; x += MT) part[x] = 0.f;
  if (rt0 >= rt1) return;
  if (q0 & 1023u) {   // (the swizzled layouts count on it)
    if (threadIdx.x == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < KS; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 8);
      mbar_init(&q_empty[i], 1);
      mbar_init(&s_full[i], 1);
      mbar_init(&s_free[i], 8);
    }
    mbar_init(ended, 1);
    *abort_flag = *issued_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(256u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cta_sync();
  tc_fence_after();
  pdl_trigger();
  const uint32_t tmem = *tmem_slot;
  // tiles of tokens that row tile rt sees, and the first token of its i-th
  auto sight_of = [&](int rt) {
    Sight t = s;
    tile_sight(a, t, rt * BM, rt * BM + BM - 1, BT);
    return t;
  };
  auto token = [&](const Sight& t, int i) { return (i < t.sink_units ? i : i - t.sink_units + t.from) * BT; };
  bool ok = true;

  if (warp >= 8 && warp < 16) {
    // ---- Q: 16 rows per warp
    for (int rt = rt0; ok && rt < rt1; ++rt) {
      const int m = rt - rt0;
      if (m >= 2) ok = wait_phase(&q_empty[m & 1], (uint32_t)((m >> 1) - 1) & 1u);
      if (!ok) break;
      const float2* ml = a.row_ml + (size_t)head * a.n * a.G + rt * BM;
#pragma unroll 1
      for (int rb = (warp - 8) * 16; rb < (warp - 7) * 16; rb += 8)
        stage_q8<NB>(a, s, b, h, rt * BM, rb, q0 + (uint32_t)(m & 1) * Shape::q_bytes, nullptr, [&](int lr, int e) {
          const float2 x = rt * BM + lr < end_row ? ml[lr] : make_float2(0.f, 0.f);
          // (factors as in the attention: not 0, which times an infinite score would not be a number)
          rowc[(m & 3) * BM + lr] = make_float2(q_factor(e, a.scale_log2), -x.x);
          rowy[(m & 3) * BM + lr] = x.y;
        });
      written(&q_full[m & 1]);
    }
  } else if (warp == 16) {
    // ---- MMAs
    const uint32_t el = elect_one();
    const uint32_t idesc = idesc_f16(BT, BM);
    const uint64_t qd0 = sw64_desc(q0), kd0 = sw64_desc(k0);
    int sk = 0, g = 0;
    uint32_t phk = 0;
    for (int rt = rt0; ok && rt < rt1; ++rt) {
      const int m = rt - rt0, n = uniform(sight_of(rt).units);
      const uint64_t qd = qd0 + (uint32_t)(m & 1) * (Shape::q_bytes >> 4);
      ok = wait_phase(&q_full[m & 1], (uint32_t)(m >> 1) & 1u);
      for (int i = 0; ok && i < n; ++i, ++g) {
        if (g >= 2) ok = wait_phase(&s_free[g & 1], (uint32_t)((g >> 1) - 1) & 1u);
        const uint32_t sd = tmem + (uint32_t)(g & 1) * BM;
#pragma unroll 1
        for (int blk = 0; ok && blk < NB; ++blk) {
          ok = wait_phase(&k_full[sk], phk);
          if (!ok) break;
          tc_fence_after();
          const uint64_t kd = kd0 + (uint32_t)sk * (KU >> 4), qb = qd + (uint32_t)blk * (QB >> 4);
#pragma unroll
          for (int k = 0; k < 4; ++k)   // both pieces of Q, the low one first: less is cut off the sums
            umma_f8(sd, kd + 2 * (k & 1), qb + (1 - (k >> 1)) * (NB * QB >> 4) + 2 * (k & 1), k < 2 ? idesc | kE5m2B : idesc, (blk > 0 || k > 0) ? 1u : 0u, el);
          umma_commit(&k_empty[sk], el);
          if (++sk == KS) {
            sk = 0;
            phk ^= 1u;
          }
        }
        if (ok) umma_commit(&s_full[g & 1], el);
      }
      if (ok) umma_commit(&q_empty[m & 1], el);
    }
    if (!ok) {   // what was issued ends before the TMEM goes away
      umma_commit(ended, el);
      wait_phase(ended, 0);
    }
    __syncwarp();
  } else if (warp == 17) {
    // ---- K: units of 64 dims
    const uint32_t el = elect_one();
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
    int slot = 0, issued = 0;
    uint32_t ph = 1;
    for (int rt = rt0; ok && rt < rt1; ++rt) {
      const Sight t = sight_of(rt);
      const int n = uniform(t.units);
      for (int i = 0; ok && i < n; ++i) {
        const int j0 = uniform(head * L.T + token(t, i));
        for (int q = 0; q < NB; ++q) {
          ok = wait_phase(&k_empty[slot], ph);
          if (!ok) break;
          mbar_expect_tx_el(&k_full[slot], KU, el);
          tma_load_2d_el(&maps.k, smem_u32(&k_full[slot]), k0 + (uint32_t)slot * KU, 64 * q, j0, pol, el);
          ++issued;
          if (++slot == KS) {
            slot = 0;
            ph ^= 1u;
          }
        }
      }
    }
    if (lane == 0) *issued_flag = issued;
    __syncwarp();
  } else if (warp < 8) {
    // ---- exponentials and sums: token t (TMEM lane t) of each tile, rows 64 hf .. of the row tile
    const int q4 = warp & 3, hf = warp >> 2, t = q4 * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(q4 * 32) << 16) + 64 * hf;
    const int8_t* KE = L.ke + (size_t)head * (L.T / 16);
    float* own = part + (size_t)hf * a.mass_pitch + t;
    int g = 0;
    for (int rt = rt0; rt < rt1; ++rt) {
      const Sight sg = sight_of(rt);
      const int m = rt - rt0, first = rt * BM + 64 * hf;
      const uint32_t rc = smem_u32(rowc + (m & 3) * BM + 64 * hf), ry = smem_u32(rowy + (m & 3) * BM + 64 * hf);
      for (int i = 0; i < sg.units; ++i, ++g) {
        const int j0 = token(sg, i), j = j0 + t;
        const float old = own[j0], kf = exp2i(KE[j / 16]);
        const RowsThatSee rows = rows_that_see(j, s.len, s.p0, a.G, end_row, a.causal, a.window, a.sinks, first);
        const bool full = __all_sync(0xffffffffu, rows.lo <= 0 && rows.hi >= 64);
        if (ok) ok = wait_phase(&s_full[g & 1], (uint32_t)(g >> 1) & 1u);
        tc_fence_after();
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          uint32_t raw[32];
          tmem_ld32_async(lane_base + (uint32_t)(g & 1) * BM + 32 * c, raw);
          tmem_wait_ld();
          tmem_reg_fence16(raw);
          tmem_reg_fence16(raw + 16);
          // (a hidden row's weight may not be a number: it is left out after the exponent)
          auto add = [&](auto hidden) {
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const float4 y = lds_f4(ry + 128u * c + 4u * k), x0 = lds_f4(rc + 256u * c + 8u * k), x1 = lds_f4(rc + 256u * c + 8u * k + 16u);
              const float2 kf2 = make_float2(kf, kf), none = make_float2(0.f, 0.f);
              const float2 a0 = fma2(make_float2(__uint_as_float(raw[k]), __uint_as_float(raw[k + 1])), kf2, none);
              const float2 a1 = fma2(make_float2(__uint_as_float(raw[k + 2]), __uint_as_float(raw[k + 3])), kf2, none);
              float2 e0 = fma2(a0, make_float2(x0.x, x0.z), make_float2(x0.y, x0.w));
              float2 e1 = fma2(a1, make_float2(x1.x, x1.z), make_float2(x1.y, x1.w));
              e0 = make_float2(fast_exp2(hidden(k) ? -INFINITY : e0.x), fast_exp2(hidden(k + 1) ? -INFINITY : e0.y));
              e1 = make_float2(fast_exp2(hidden(k + 2) ? -INFINITY : e1.x), fast_exp2(hidden(k + 3) ? -INFINITY : e1.y));
              sum[0] = fma2(e0, make_float2(hidden(k) ? 0.f : y.x, hidden(k + 1) ? 0.f : y.y), sum[0]);
              sum[1] = fma2(e1, make_float2(hidden(k + 2) ? 0.f : y.z, hidden(k + 3) ? 0.f : y.w), sum[1]);
            }
          };
          if (full) {
            add([](int) { return false; });
          } else {
            const uint32_t see = RowMask::below(rows.hi - 32 * c) & ~RowMask::below(rows.lo - 32 * c);
            add([see](int k) { return (see & (1u << k)) == 0u; });
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[g & 1]);
        own[j0] = old + ((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
      }
    }
  }
  if (!ok && lane == 0) *abort_flag = 1;
  tc_fence_before();
  cta_sync();
  if (*abort_flag && threadIdx.x == 0) {
    // loads still on their way, at most a ring of them, land before the shared memory goes away
    for (int i = max(0, *issued_flag - KS); i < *issued_flag; ++i) mbar_wait(&k_full[i % KS], (uint32_t)(i / KS) & 1u);
    raise_error(a.err, ERR_TIMEOUT);
  }
  if (warp == 16)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256u) : "memory");
}

// The chunks' sums: eight threads per token, every eighth of them each, then in the
// threads' order -- the same order in every call.
__global__ void __launch_bounds__(256) cache_mass_sum_kernel(CacheAttnArgs a) {
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, eighth = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
  const size_t head = (size_t)blockIdx.z * a.c.Hkv + blockIdx.y;
  pdl_trigger();
  pdl_wait();
  const float* part = a.mass_ws + head * a.splits * 2 * a.mass_pitch + j;   // (j < pitch, a multiple of 32)
  float v = 0.f;
#pragma unroll 8
  for (int c = eighth; c < 2 * a.splits; c += 8) v += ld_l2(part + (size_t)c * a.mass_pitch);
  sums[eighth][lane] = v;
  __syncthreads();
  if (eighth || j >= a.max_length) return;
  v = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) v += sums[e][lane];
  float* mass = a.mass + head * a.mass_stride + j;
  if (!a.mass_add) *mass = v;
  else if (j < a.lengths[blockIdx.z]) *mass += v;
}

template <int NB>
cudaError_t launch_nb(const MassMaps& maps, const CacheAttnArgs& a, cudaStream_t st) {
  const unsigned units = (unsigned)((long long)a.batch * a.c.Hkv * a.splits);
  return launch_kernel(cache_mass_tc_kernel<NB>, dim3(units), dim3(MT), MassShape<NB>::bytes, st, 1, maps, a);
}

template <int NB>
cudaError_t init_nb() {
  return cudaFuncSetAttribute(cache_mass_tc_kernel<NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, MassShape<NB>::bytes);
}

}  // namespace

cudaError_t launch_cache_mass_tc(CacheAttnArgs a, cudaStream_t st) {
  a.row_tiles = (a.n * a.G + BM - 1) / BM;
  a.mass_pitch = (a.max_length + BT - 1) / BT * BT;
  // a CTA per SM, as far as there are row tiles and room for the chunks' sums
  const long long heads = (long long)a.batch * a.c.Hkv;
  long long chunks = std::max(1ll, (a.num_sms + heads - 1) / heads);
  chunks = std::min(chunks, std::max(1ll, (long long)(a.mass_ws_bytes / (8ull * a.mass_pitch)) / heads));
  a.splits = (int)std::min(chunks, (long long)a.row_tiles);
  const MassMaps maps{a.maps->k_tc};
  const Overlap overlap;
  cudaError_t e;
  switch (a.c.hdp) {
    case 64: e = launch_nb<1>(maps, a, st); break;
    case 128: e = launch_nb<2>(maps, a, st); break;
    case 192: e = launch_nb<3>(maps, a, st); break;
    default: e = launch_nb<4>(maps, a, st); break;
  }
  if (e != cudaSuccess) return e;
  return launch_kernel(cache_mass_sum_kernel, dim3((a.max_length + 31) / 32, a.c.Hkv, a.batch), dim3(256), 0, st, 1, a);
}

size_t cache_mass_ws_bytes(int heads, int Hkv, int G, long long rows, int T, int num_sms) {
  // a chunk per head, and the scores of a query; at best a chunk per SM and all scores, up to
  // 64 MB, which stay in L2 until they are summed
  const size_t least = std::max(8ull * heads * T, 4ull * Hkv * G * T);
  const double most = std::max(8.0 * ((double)heads + num_sms) * T, 4.0 * heads * (double)rows * T);
  return std::max(least, (size_t)std::min(most, 64.0 * (1 << 20)));
}

cudaError_t init_cache_mass_tc_kernels() {
  cudaError_t e = init_nb<1>();
  if (e == cudaSuccess) e = init_nb<2>();
  if (e == cudaSuccess) e = init_nb<3>();
  if (e == cudaSuccess) e = init_nb<4>();
  return e;
}

}  // namespace ravel
