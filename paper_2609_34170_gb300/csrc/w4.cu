// Products of few rows with 4-bit weights: y[m, n] = sum_k x[m, k] (c[n, k] - z[n, g(k)]) s[n, g(k)].
#include <algorithm>

#include "common.cuh"
#include "decode.h"
#include "launch.h"
#include "tc_common.cuh"

namespace ravel {
namespace {

// ---- the order in which a matrix is held ------------------------------------------
//
// An MMA m16n8k16 takes 16 weight rows as A and 8 tokens as B.  The order of the ks inside an MMA is
// free as long as A and B agree, so lane 4g + q of a warp takes ks 8q .. 8q + 7 of every 32: its
// piece of a token's row is 16 contiguous bytes, and no operand of B passes through shared memory to be
// put into order.  Two MMAs (s = 0, 1) take the 32: of the lane's eight ks, 4s and 4s + 1 are the k
// pair of the registers a0 (row g), a1 (row g + 8) and b0, and 4s + 2, 4s + 3 that of a2, a3 and b1.
// So a lane's weights of two rows and two 32s are 32 codes, one uint4: word 2 * (which 32) + s holds in
// nibble i the first k of register ai and in nibble 4 + i the second, and a warp reads 16 rows x 64 ks in
// one contiguous 512-byte load.
constexpr int kWarps = 8;
constexpr int kRanks = 8;    // CTAs that share the ks of a pair at most
constexpr int kPitch = 36;   // floats of a token's 32 rows: lanes of a store land in different banks

__device__ __forceinline__ void code_place(int lane, int word, int nibble, int* row, int* k) {
  const int g = lane >> 2, q = lane & 3, i = nibble & 3;
  *row = g + (i & 1) * 8;
  *k = (word >> 1) * 32 + q * 8 + (word & 1) * 4 + (i >> 1) * 2 + (nibble >> 2);
}

// A thread per word: 8 codes from wherever they are.
__global__ void __launch_bounds__(256) w4_load_codes_kernel(W4Matrix w, const uint8_t* codes, const uint8_t* zeros, long long words) {
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  pdl_wait();
  if (idx >= words) return;
  const int word = (int)(idx & 3), lane = (int)(idx >> 2) & 31;
  const long long block = idx >> 7;
  const int tile = (int)(block / w.kblocks), kb = (int)(block % w.kblocks);
  const size_t pitch = (size_t)(w.K + 1) / 2;
  uint32_t out = 0;
#pragma unroll
  for (int nibble = 0; nibble < 8; ++nibble) {
    int row, k;
    code_place(lane, word, nibble, &row, &k);
    row += tile * 16;
    k += kb * 64;
    uint32_t c = 0;
    if (row < w.N && k < w.K) c = (codes[row * pitch + k / 2] >> (k & 1) * 4) & 15u;
    else if (row < w.N && k / w.group < w.groups) c = zeros[(size_t)row * w.groups + k / w.group] & 15u;   // past the end: weight 0
    out |= c << 4 * nibble;
  }
  ((uint32_t*)w.codes)[idx] = out;
}

// Rows g and g + 8 of a tile and group side by side, as (scale, 128 + zero) in bf16.
__global__ void __launch_bounds__(256) w4_load_scales_kernel(W4Matrix w, const uint16_t* scales, const uint8_t* zeros, long long words) {
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  pdl_wait();
  if (idx >= words) return;
  const int which = (int)(idx & 1), g = (int)(idx >> 1) & 7;
  const long long block = idx >> 4;
  const int tile = (int)(block / w.groups), group = (int)(block % w.groups), row = tile * 16 + g + which * 8;
  uint32_t out = 0x4300u;
  if (row < w.N) {
    const size_t at = (size_t)row * w.groups + group;
    out = (uint32_t)scales[at] << 16 | 0x4300u | (zeros[at] & 15u);
  }
  ((uint32_t*)w.sz)[idx] = out;
}

template <typename T>
__global__ void __launch_bounds__(256) w4_read_kernel(W4Matrix w, T* out, int ldo, long long words) {
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  pdl_trigger();
  pdl_wait();
  if (idx >= words) return;
  const int word = (int)(idx & 3), lane = (int)(idx >> 2) & 31;
  const long long block = idx >> 7;
  const int tile = (int)(block / w.kblocks), kb = (int)(block % w.kblocks);
  const uint32_t codes = ((const uint32_t*)w.codes)[idx];
#pragma unroll
  for (int nibble = 0; nibble < 8; ++nibble) {
    int r, k;
    code_place(lane, word, nibble, &r, &k);
    const int row = r + tile * 16;
    k += kb * 64;
    if (row >= w.N || k >= w.K) continue;
    const uint32_t sz = ((const uint32_t*)w.sz)[(((size_t)tile * w.groups + k / w.group) * 8 + (r & 7)) * 2 + (r >> 3)];
    const float c = (float)(int)((codes >> 4 * nibble & 15u) - (sz & 15u));
    out[(size_t)row * ldo + k] = from_f32<T>(c * __uint_as_float(sz & 0xffff0000u));
  }
}

// A warp per row and group.
template <typename T>
__global__ void __launch_bounds__(256) w4_quantize_kernel(const T* W, int N, int K, int ldw, int group, int groups, uint8_t* codes,
                                                          bf16* scales, uint8_t* zeros) {
  const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  if (at >= (long long)N * groups) return;
  const int row = (int)(at / groups), k0 = (int)(at % groups) * group, k1 = min(k0 + group, K);
  const T* in = W + (size_t)row * ldw;
  float lo = 0.f, hi = 0.f;
  for (int k = k0 + lane; k < k1; k += 32) {
    const float x = to_f32(in[k]);
    lo = fminf(lo, x);
    hi = fmaxf(hi, x);
  }
  hi = warp_max(hi);
  lo = -warp_max(-lo);
  const bf16 sb = __float2bfloat16_rn((hi - lo) / 15.f);
  const float s = __bfloat162float(sb);
  const float z = s > 0.f ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
  auto code = [&](int k) -> uint32_t {
    if (!(s > 0.f) || k >= k1) return 0u;
    return (uint32_t)fminf(fmaxf(rintf(to_f32(in[k]) / s + z), 0.f), 15.f);
  };
  for (int k = k0 + 2 * lane; k < k1; k += 64)   // (groups begin at even ks)
    codes[(size_t)row * ((K + 1) / 2) + k / 2] = (uint8_t)(code(k) | code(k + 1) << 4);
  if (lane == 0) {
    scales[at] = sb;
    zeros[at] = (uint8_t)z;
  }
}

// ---- the product -------------------------------------------------------------------

__device__ __forceinline__ void mma_bf16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight codes as c - z in bf16, the four registers of A: 0x43 above a code is 128 + c, and 128 + c less
// 128 + z is exact.
__device__ __forceinline__ void widen(uint32_t w, uint32_t z0, uint32_t z8, uint32_t* a) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = sub_bf16x2((w >> 4 * i & 0x000f000fu) | 0x43004300u, i & 1 ? z8 : z0);
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

__device__ __forceinline__ uint4 ld_weights(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld_weights(const uint2* p) {
  uint2 v;
  asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// What a warp holds of a block of 64 ks: codes of its two tiles and their scales.
template <bool G32>
struct Block {
  uint4 codes[2];
  uint2 sz[2][G32 ? 2 : 1];
};

// Tiles of a pair: side by side, or for GeGLU 16 gate rows and their 16 up rows.
__device__ __forceinline__ int first_tile(int pair, int epi) { return epi == EPI_GEGLU ? pair / 4 * 8 + pair % 4 : 2 * pair; }
__device__ __forceinline__ int second_tile(int pair, int epi) { return first_tile(pair, epi) + (epi == EPI_GEGLU ? 4 : 1); }

// A pair's sums [token][kPitch] in shared memory, this rank's share of them, into the output: threads
// first, first + step, ... of those that work on the pair.
template <int NT>
__device__ __forceinline__ void finish(const W4Args& a, const float* part, int pair, int m0, int ranks, int rank, int first, int step) {
  const bool glu = a.epi == EPI_GEGLU;
  const int t0 = first_tile(pair, a.epi), t1 = second_tile(pair, a.epi);
  const int shift = glu ? 4 : 5, rows = 1 << shift, all = min(NT * 8, a.M - m0) << shift;
  const int e0 = all * rank / ranks, e1 = all * (rank + 1) / ranks;
  for (int e = e0 + first; e < e1; e += step) {
    const int m = e >> shift, r = e & (rows - 1);
    auto total = [&](int row) {
      if (ranks == 1) return part[m * kPitch + row];
      const uint32_t at = smem_u32(part + m * kPitch + row);
      float x[kRanks];   // (all on their way together)
#pragma unroll
      for (int i = 0; i < kRanks; ++i) x[i] = ld_cluster_f(mapa_shared(at, (uint32_t)min(i, ranks - 1)));
      float v = x[0];
#pragma unroll
      for (int i = 1; i < kRanks; ++i) v += i < ranks ? x[i] : 0.f;
      return v;
    };
    auto with_bias = [&](int row, float v) {
      const int n = (row < 16 ? t0 : t1) * 16 + (row & 15);
      return a.bias && n < a.w.N ? v + a.bias[n] : v;
    };
    float v = with_bias(r, total(r));
    int col = (r < 16 ? t0 : t1) * 16 + (r & 15);
    if (glu) {
      v = gelu_tanh_f(v) * with_bias(r + 16, total(r + 16));
      col = pair / 4 * 64 + pair % 4 * 16 + r;
    } else if (col >= a.w.N) {
      continue;
    }
    const size_t to = (size_t)(m0 + m) * a.ldo + col;
    if (a.epi == EPI_STORE_SILU) v = silu_f(v);
    if (a.epi == EPI_ADD_F32) ((float*)a.out)[to] += v;
    else if (a.out_bf16) ((bf16*)a.out)[to] = from_f32<bf16>(v);
    else ((float*)a.out)[to] = v;
  }
}

// A block's weights of a pair of tiles into the registers of A, and the rows' scales.
template <bool G32>
struct Operand {
  uint32_t A[2][4][4];
  float s0[2][G32 ? 2 : 1], s8[2][G32 ? 2 : 1];
  __device__ __forceinline__ void set(const Block<G32>& b) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t* c = (const uint32_t*)&b.codes[t];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2 sz = b.sz[t][G32 ? i >> 1 : 0];
        widen(c[i], __byte_perm(sz.x, 0u, 0x1010), __byte_perm(sz.y, 0u, 0x1010), A[t][i]);
      }
#pragma unroll
      for (int h = 0; h < (G32 ? 2 : 1); ++h) {
        s0[t][h] = __uint_as_float(b.sz[t][h].x & 0xffff0000u);
        s8[t][h] = __uint_as_float(b.sz[t][h].y & 0xffff0000u);
      }
    }
  }
  // acc += the block's product with 8 tokens' values x (of its first and its second 32 ks)
  __device__ __forceinline__ void multiply(const uint4* x, float (*acc)[4], int stride) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int h = 0; h < (G32 ? 2 : 1); ++h) {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int hh = G32 ? h : 0; hh < (G32 ? h + 1 : 2); ++hh) {
          mma_bf16(sum, A[t][2 * hh], x[hh].x, x[hh].y);
          mma_bf16(sum, A[t][2 * hh + 1], x[hh].z, x[hh].w);
        }
        acc[t * stride][0] += s0[t][h] * sum[0];
        acc[t * stride][1] += s0[t][h] * sum[1];
        acc[t * stride][2] += s8[t][h] * sum[2];
        acc[t * stride][3] += s8[t][h] * sum[3];
      }
    }
  }
};

// The sums of a warp into [token][kPitch].
template <int NT>
__device__ __forceinline__ void put_sums(float* to, const float (*acc)[NT][4], int g, int q) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) to[(n * 8 + 2 * q + (i & 1)) * kPitch + t * 16 + g + (i >> 1) * 8] = acc[t][n][i];
}

// A CTA takes two tiles of 16 rows (GeGLU: 16 gate rows and their 16 up rows) and NT * 8 tokens; its eight
// warps, and the CTAs of its cluster, share the ks.
//
// Sums: an MMA chain per group (at most 64 ks of it) starts from zero, and the group's scale
// takes its result into an fp32 sum, so that weights enter as whole numbers and no scaled weight
// is rounded.  Parts of the ks are joined in the order of warps and ranks.
template <int NT, bool G32>
__global__ void __launch_bounds__(256) w4_gemm_kernel(W4Args a) {
  constexpr int kAhead = NT <= 2 ? 4 : 2;   // blocks on their way
  constexpr int kPart = NT * 8 * kPitch;
  extern __shared__ float part[];           // [warp][token][kPitch], then the CTA's sums in the first
  const W4Matrix& w = a.w;
  const int ranks = (int)gridDim.z, rank = ranks > 1 ? (int)cluster_ctarank() : 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  const int pair = blockIdx.x, m0 = blockIdx.y * NT * 8;
  const int t0 = first_tile(pair, a.epi), t1 = second_tile(pair, a.epi);
  const int shares = ranks * kWarps, share = rank * kWarps + warp;
  const int k0 = (int)((long long)w.kblocks * share / shares), k1 = (int)((long long)w.kblocks * (share + 1) / shares);

  Block<G32> held[kAhead];
  auto fetch = [&](Block<G32>& b, int kb) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int tile = t ? t1 : t0;
      b.codes[t] = ld_weights(w.codes + ((size_t)tile * w.kblocks + kb) * 32 + lane);
#pragma unroll
      for (int h = 0; h < (G32 ? 2 : 1); ++h) {
        const int group = min((kb * 64 + h * 32) / w.group, w.groups - 1);
        b.sz[t][h] = ld_weights(w.sz + ((size_t)tile * w.groups + group) * 8 + g);
      }
    }
  };
  // loaded weights do not change: the first blocks are on their way before the launch before has ended
#pragma unroll
  for (int d = 0; d < kAhead; ++d)
    if (k0 + d < k1) fetch(held[d], k0 + d);
  pdl_trigger();
  pdl_wait();

  float acc[2][NT][4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[t][n][i] = 0.f;

  for (int kb0 = k0; kb0 < k1; kb0 += kAhead) {
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
      const int kb = kb0 + d;
      if (kb >= k1) break;
      Operand<G32> op;
      op.set(held[d]);
      if (kb + kAhead < k1) fetch(held[d], kb + kAhead);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int m = m0 + n * 8 + g;
        const bf16* row = (const bf16*)a.x + (long long)m * a.lda;
        uint4 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] = load_x(row, kb * 64 + h * 32 + q * 8, w.K, m < a.M, a.vec);
        op.multiply(x, &acc[0][n], NT);
      }
    }
  }

  float* mine = part + warp * kPart;
  put_sums<NT>(mine, acc, g, q);
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 8 * 32; e += 256) {
    const int at = (e >> 5) * kPitch + (e & 31);
    float v = part[at];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) v += part[i * kPart + at];
    part[at] = v;   // (read by this thread alone so far)
  }
  if (ranks > 1) cluster_sync();
  else __syncthreads();

  finish<NT>(a, part, pair, m0, ranks, rank, threadIdx.x, 256);
  if (ranks > 1) cluster_sync();   // nobody leaves while its sums are read
}

// More tokens, where the rows fill the SMs: a warp takes a pair of tiles with all of the CTA's ks, so that
// eight pairs share each token's values.  Codes, scales and values come by asynchronous copies
// into a ring of stages of 64 ks.  A stage's tokens are rows of 128 bytes, whose halves change
// places in odd rows: the 8 lanes that a shared-memory access serves at a time read 64 bytes of two rows.
constexpr int kStages = 6;
template <int NT>
struct Stage {
  uint4 x[NT * 8][8];
  uint4 codes[kWarps * 2][32];
  uint2 sz[2][kWarps * 2][8];   // by 32 ks where these are a group, otherwise the first
};

__device__ __forceinline__ void copy_async(void* to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}

template <int NT, bool G32>
__global__ void __launch_bounds__(256, 2) w4_wide_kernel(W4Args a) {
  extern __shared__ __align__(16) unsigned char wide_smem[];
  Stage<NT>* ring = (Stage<NT>*)wide_smem;
  const W4Matrix& w = a.w;
  const int ranks = (int)gridDim.z, rank = ranks > 1 ? (int)cluster_ctarank() : 0;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q = lane & 3;
  const int pair0 = blockIdx.x * kWarps, pair = pair0 + warp, pairs = w.tiles / 2, m0 = blockIdx.y * NT * 8;
  const int k0 = (int)((long long)w.kblocks * rank / ranks), k1 = (int)((long long)w.kblocks * (rank + 1) / ranks);

  // a stage's weights: a warp copies its own pair's; of pairs past the end nothing is copied and nothing kept
  auto fetch_weights = [&](int kb) {
    if (pair >= pairs) return;
    Stage<NT>& st = ring[(kb - k0) % kStages];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int tile = t ? second_tile(pair, a.epi) : first_tile(pair, a.epi);
      copy_async(&st.codes[warp * 2 + t][lane], w.codes + ((size_t)tile * w.kblocks + kb) * 32 + lane, true);
    }
    // 64 bytes of scales per tile and group: 4 lanes each
    const int t = lane >> 2 & 1, h = lane >> 3;
    if (h < (G32 ? 2 : 1)) {
      const int tile = t ? second_tile(pair, a.epi) : first_tile(pair, a.epi);
      const int group = min((kb * 64 + h * 32) / w.group, w.groups - 1);
      copy_async(&st.sz[h][warp * 2 + t][(lane & 3) * 2], w.sz + ((size_t)tile * w.groups + group) * 8 + (lane & 3) * 2, true);
    }
  };
  auto fetch_x = [&](int kb) {
    Stage<NT>& st = ring[(kb - k0) % kStages];
#pragma unroll
    for (int i = 0; i < NT * 64 / 256; ++i) {
      const int at = tid + i * 256, token = at >> 3, piece = at & 7, m = m0 + token, k = kb * 64 + piece * 8;
      const bf16* row = (const bf16*)a.x + (long long)m * a.lda;
      uint4* to = &st.x[token][piece ^ (token & 1) * 4];
      if (a.vec) {
        const bool there = m < a.M && k + 8 <= w.K;
        if (m < a.M && k < w.K && !there) *to = load_x(row, k, w.K, true, 0);
        else copy_async(to, there ? (const void*)(row + k) : a.x, there);
      } else {
        *to = load_x(row, k, w.K, m < a.M, 0);
      }
    }
  };
  auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };

#pragma unroll
  for (int i = 0; i < kStages - 1; ++i)   // (weights do not change: ahead of the wait)
    if (k0 + i < k1) fetch_weights(k0 + i);
  pdl_trigger();
  pdl_wait();
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (k0 + i < k1) fetch_x(k0 + i);
    commit();   // (the first group holds all the weights so far)
  }

  float acc[2][NT][4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[t][n][i] = 0.f;

  for (int kb = k0; kb < k1; ++kb) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncthreads();   // everybody's copies are there, and the stage before is read
    if (kb + kStages - 1 < k1) {
      fetch_weights(kb + kStages - 1);
      fetch_x(kb + kStages - 1);
    }
    commit();
    if (pair >= pairs) continue;
    const Stage<NT>& st = ring[(kb - k0) % kStages];
    Operand<G32> op;
    {
      Block<G32> b;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        b.codes[t] = st.codes[warp * 2 + t][lane];
#pragma unroll
        for (int h = 0; h < (G32 ? 2 : 1); ++h) b.sz[t][h] = st.sz[h][warp * 2 + t][g];
      }
      op.set(b);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int token = n * 8 + g;
      uint4 x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) x[h] = st.x[token][(h ^ (token & 1)) * 4 + q];
      op.multiply(x, &acc[0][n], NT);
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  float* part = (float*)wide_smem + warp * NT * 8 * kPitch;
  put_sums<NT>(part, acc, g, q);
  if (ranks > 1) cluster_sync();
  else __syncwarp();
  if (pair < pairs) finish<NT>(a, part, pair, m0, ranks, rank, lane, 32);
  if (ranks > 1) cluster_sync();   // nobody leaves while its sums are read
}

template <int NT>
constexpr size_t wide_smem_of() {
  return sizeof(Stage<NT>) * kStages > sizeof(float) * kWarps * NT * 8 * kPitch ? sizeof(Stage<NT>) * kStages
                                                                                  : sizeof(float) * kWarps * NT * 8 * kPitch;
}

template <int NT>
cudaError_t init_wide() {
  cudaError_t e = cudaFuncSetAttribute(w4_wide_kernel<NT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)wide_smem_of<NT>());
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(w4_wide_kernel<NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)wide_smem_of<NT>());
  return e;
}

template <int NT>
cudaError_t launch_wide(const W4Args& a, cudaStream_t st) {
  const int blocks = (a.w.tiles / 2 + kWarps - 1) / kWarps, tiles = (a.M + NT * 8 - 1) / (NT * 8);
  int ranks = 1;
  while (ranks < kRanks && (long long)blocks * tiles * ranks < 4 * a.num_sms && a.w.kblocks >= ranks * 2 * 4) ranks *= 2;
  const Overlap overlap;
  return launch_kernel_cluster(a.w.group == 32 ? w4_wide_kernel<NT, true> : w4_wide_kernel<NT, false>, dim3(blocks, tiles, ranks),
                               dim3(256), wide_smem_of<NT>(), st, dim3(1, 1, ranks), a);
}

template <int NT>
constexpr size_t smem_of() {
  return sizeof(float) * kWarps * NT * 8 * kPitch;
}

template <int NT>
cudaError_t init_nt() {
  cudaError_t e = cudaFuncSetAttribute(w4_gemm_kernel<NT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of<NT>());
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(w4_gemm_kernel<NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of<NT>());
  return e;
}

template <int NT>
cudaError_t launch_nt(const W4Args& a, cudaStream_t st) {
  const int pairs = a.w.tiles / 2, tiles = (a.M + NT * 8 - 1) / (NT * 8);
  // the ks of a pair over as many CTAs (1, 2, 4, 8) as there are SMs for and blocks for the warps
  int ranks = 1;
  while (ranks < 8 && (long long)pairs * tiles * ranks * 2 <= 2 * a.num_sms && a.w.kblocks >= ranks * 2 * kWarps) ranks *= 2;
  const Overlap overlap;
  return launch_kernel_cluster(a.w.group == 32 ? w4_gemm_kernel<NT, true> : w4_gemm_kernel<NT, false>, dim3(pairs, tiles, ranks),
                               dim3(256), smem_of<NT>(), st, dim3(1, 1, ranks), a);
}

unsigned blocks_of(long long threads) { return (unsigned)((threads + 255) / 256); }

}  // namespace

cudaError_t init_w4_kernels() {
  cudaError_t e = init_nt<1>();
  if (e == cudaSuccess) e = init_nt<2>();
  if (e == cudaSuccess) e = init_nt<4>();
  if (e == cudaSuccess) e = init_nt<8>();
  if (e == cudaSuccess) e = init_wide<4>();
  if (e == cudaSuccess) e = init_wide<8>();
  return e;
}

cudaError_t launch_w4_gemm(const W4Args& a, cudaStream_t st) {
  if (a.M > 16 && a.w.tiles >= 256) return a.M <= 32 ? launch_wide<4>(a, st) : launch_wide<8>(a, st);
  return a.M <= 8 ? launch_nt<1>(a, st) : a.M <= 16 ? launch_nt<2>(a, st) : a.M <= 32 ? launch_nt<4>(a, st) : launch_nt<8>(a, st);
}

cudaError_t launch_w4_load(const W4Matrix& w, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, cudaStream_t st) {
  const long long words = (long long)w.tiles * w.kblocks * 128, szs = (long long)w.tiles * w.groups * 16;
  cudaError_t e = launch_kernel(w4_load_codes_kernel, dim3(blocks_of(words)), dim3(256), 0, st, 1, w, codes, zeros, words);
  if (e == cudaSuccess) e = launch_kernel(w4_load_scales_kernel, dim3(blocks_of(szs)), dim3(256), 0, st, 1, w, scales, zeros, szs);
  return e;
}

cudaError_t launch_w4_read(const W4Matrix& w, void* out, int ldo, Dtype dt, cudaStream_t st) {
  const long long words = (long long)w.tiles * w.kblocks * 128;
  const Overlap overlap;
  if (dt == DT_BF16) return launch_kernel(w4_read_kernel<bf16>, dim3(blocks_of(words)), dim3(256), 0, st, 1, w, (bf16*)out, ldo, words);
  return launch_kernel(w4_read_kernel<float>, dim3(blocks_of(words)), dim3(256), 0, st, 1, w, (float*)out, ldo, words);
}

cudaError_t launch_w4_quantize(const void* W, int N, int K, int ldw, Dtype dt, int group, uint8_t* codes, uint16_t* scales,
                               uint8_t* zeros, cudaStream_t st) {
  const int groups = (K + group - 1) / group;
  const unsigned blocks = blocks_of((long long)N * groups * 32);
  const Overlap overlap;
  if (dt == DT_BF16)
    return launch_kernel(w4_quantize_kernel<bf16>, dim3(blocks), dim3(256), 0, st, 1, (const bf16*)W, N, K, ldw, group, groups, codes,
                         (bf16*)scales, zeros);
  return launch_kernel(w4_quantize_kernel<float>, dim3(blocks), dim3(256), 0, st, 1, (const float*)W, N, K, ldw, group, groups, codes,
                       (bf16*)scales, zeros);
}

}  // namespace ravel
