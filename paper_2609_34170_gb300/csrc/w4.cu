// Products of few rows with 4-bit weights: y[m, n] = sum_k x[m, k] (c[n, k] - z[n, g(k)]) s[n, g(k)].
#include <algorithm>

#include "common.cuh"
#include "decode.h"
#include "launch.h"
#include "tc_common.cuh"
#include "w4.cuh"

namespace ravel {
namespace {

// ---- the order in which a matrix is held ------------------------------------------
//
// An MMA m16n8k16 takes 16 weight rows as A and 8 tokens as B.  The order of the ks inside an MMA is
// free as long as A and B agree, so lane 4g + q of a warp takes ks 8q .. 8q + 7 of every 32: its
// piece of a token's row is 16 contiguous bytes, and no operand of B passes through shared memory to be
// put into order.  Two MMAs (s = 0, 1) take the 32: of the lane's eight ks, 4s and 4s + 1 are the k
// pair of the registers a0 (row g), a1 (row g + 8) and b0, and 4s + 2, 4s + 3 that of a2, a3 and b1.
// So a lane's weights of two rows and two 32s are 32 codes, one uint4: word 2s + (which 32) holds in
// nibble i the first k of register ai and in nibble 4 + i the second, and a warp reads 16 rows x 64 ks in
// one contiguous 512-byte load.
constexpr int kWarps = 8;
constexpr int kPitch = 36;   // floats of a token's 32 rows: lanes of a store land in different banks

__device__ __forceinline__ void code_place(int lane, int word, int nibble, int* row, int* k) {
  const int g = lane >> 2, q = lane & 3, i = nibble & 3;
  *row = g + (i & 1) * 8;
  *k = (word & 1) * 32 + q * 8 + (word >> 1) * 4 + (i >> 1) * 2 + (nibble >> 2);
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
  const float range = hi - lo;   // (of finite values may be infinite)
  const bf16 sb = __float2bfloat16_rn(range < INFINITY ? range / 15.f : hi / 15.f - lo / 15.f);
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

// the same from zero
__device__ __forceinline__ void mma_bf16_first(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// Eight codes as c - z in bf16, the four registers of A: 0x43 above a code is 128 + c, and 128 + c less
// 128 + z is exact.
__device__ __forceinline__ void widen(uint32_t w, uint32_t z0, uint32_t z8, uint32_t* a) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = sub_bf16x2((w >> 4 * i & 0x000f000fu) | 0x43004300u, i & 1 ? z8 : z0);
}

// Tiles of a pair: side by side, or for GeGLU 16 gate rows and their 16 up rows.
__device__ __forceinline__ int first_tile(int pair, int epi) { return epi == EPI_GEGLU ? pair / 4 * 8 + pair % 4 : 2 * pair; }
__device__ __forceinline__ int second_tile(int pair, int epi) { return first_tile(pair, epi) + (epi == EPI_GEGLU ? 4 : 1); }

// A pair's outputs, or this rank's share of them: total(token, row of the pair's 32), computed by threads
// first, first + step, ... of those that work on the pair.
template <int NT, typename Total>
__device__ __forceinline__ void finish(const W4Args& a, int pair, int m0, int ranks, int rank, int first, int step, Total total_of) {
  const bool glu = a.epi == EPI_GEGLU;
  const int t0 = first_tile(pair, a.epi), t1 = second_tile(pair, a.epi);
  const int shift = glu ? 4 : 5, rows = 1 << shift, all = min(NT * 8, a.M - m0) << shift;
  const int e0 = all * rank / ranks, e1 = all * (rank + 1) / ranks;
  for (int e = e0 + first; e < e1; e += step) {
    const int m = e >> shift, r = e & (rows - 1);
    auto total = [&](int row) { return total_of(m, row); };
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

// Two blocks of a warp's codes and their groups' scales; GS: 32s of ks in a group.
template <int GS>
struct Slot {
  uint4 codes[2][2][32];    // [block][tile]
  uint2 sz[4 / GS][2][8];   // [group][tile]
};

// sum += a block's product with NT * 8 tokens' values x, chains of a group from zero; at a group's end acc += scale sum
template <int NT, int GS, int B>
__device__ __forceinline__ void multiply(const Slot<GS>& slot, int lane, int g, const uint4 (*x)[2], float (*sum)[NT][4], float (*acc)[NT][4]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint4 codes = slot.codes[B][t][lane];
    const uint32_t c[4] = {codes.x, codes.z, codes.y, codes.w};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = 2 * B + h;   // of four 32s
      const uint2 sz = slot.sz[at / GS][t][g];
      const uint32_t z0 = __byte_perm(sz.x, 0u, 0x1010), z8 = __byte_perm(sz.y, 0u, 0x1010);
      uint32_t A[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) widen(c[2 * h + i], z0, z8, A[i]);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (at % GS == 0) mma_bf16_first(sum[t][n], A[0], x[n][h].x, x[n][h].y);
        else mma_bf16(sum[t][n], A[0], x[n][h].x, x[n][h].y);
        mma_bf16(sum[t][n], A[1], x[n][h].z, x[n][h].w);
        if (at % GS == GS - 1) {
          const float s0 = __uint_as_float(sz.x & 0xffff0000u), s8 = __uint_as_float(sz.y & 0xffff0000u);
          acc[t][n][0] += s0 * sum[t][n][0];
          acc[t][n][1] += s0 * sum[t][n][1];
          acc[t][n][2] += s8 * sum[t][n][2];
          acc[t][n][3] += s8 * sum[t][n][3];
        }
      }
    }
  }
}

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
// warps, and the CTAs of its cluster, share the ks.  A CTA that has several pairs of tiles goes
// through them one after another, and the copies of the next pair's weights run on under the end of the one
// before: each warp has a ring of its own, filled by asynchronous copies.
//
// Sums: an MMA chain per group (at most 128 ks) starts from zero, and the group's scale
// takes its result into an fp32 sum, so that weights enter as whole numbers and no scaled weight
// is rounded.  Parts of the ks are joined in the order of warps and ranks.
//
// Small matrices are a chain's latency: 1 row x 2560 x 1024 2.1 us (replays from a graph), 16 x 1024 x 4096 4.7 in fp32 to a
// residual.  Large ones are bound by instructions: 191 for 2048 codes, 88 of them the codes' widening (11 for every 8 codes of
// a lane), most of which take the half-rate integer pipe.  1 row x 65536 x 8192: that pipe is busy for 73 % of an SM's active
// cycles, the schedulers issue in 63 %, DRAM gives half its rate; of the 5.3 cycles between a warp's instructions 1.2 wait
// for a full pipe, 1.2 for another warp's turn, 0.9 for the instruction before, 0.3 for memory.  1 row x 65536 x 2048 19.8 us
// (3.6 TB/s of 6.7), x 8192 x 8192 11.0; 16 rows x 8192 x 8192 13.5.  With
// pieces of 64 ks 22.4, 12.3 and 15.7 (the copies' instructions and waits twice as often); those with three CTAs an SM and 80
// registers 23 and 18.5, with a division and 64-bit addresses a piece 27.5 and 23.
constexpr int kRing = 3;   // pieces of 128 ks
constexpr int kHeld = 2;   // CTAs an SM holds, by registers

// FAST: rows of x are 16-byte aligned and K a multiple of 8, so that a lane's eight values are there or not.
template <int NT, int GS, bool FAST>
__global__ void __launch_bounds__(256, kHeld) w4_gemm_kernel(W4Args a) {
  constexpr int kPart = NT * 8 * kPitch;
  extern __shared__ __align__(16) unsigned char few_smem[];
  Slot<GS>* ring = (Slot<GS>*)few_smem + (threadIdx.x >> 5) * kRing;
  float* parts = (float*)((Slot<GS>*)few_smem + kWarps * kRing);   // [2][warp][token][kPitch]
  const W4Matrix& w = a.w;
  const int ranks = (int)gridDim.z, rank = ranks > 1 ? (int)cluster_ctarank() : 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  const int pairs = w.tiles / 2, m0 = blockIdx.y * NT * 8;
  const int shares = ranks * kWarps, share = rank * kWarps + warp;
  const int pieces = (w.kblocks + 1) / 2;
  const int k0 = (int)((long long)pieces * share / shares), k1 = (int)((long long)pieces * (share + 1) / shares);

  // the next piece of the sequence (pair by pair, the warp's pieces of each) into the next slot
  int next_pair = blockIdx.x, next_piece = k1, next_slot = 0;
  const int sz_t = lane >> 2 & 1, sz_g = lane >> 3;   // 64 bytes of scales per tile and group: 4 lanes each
  const uint4 *from0 = nullptr, *from1 = nullptr;
  const uint2* from_sz = nullptr;
  if (k0 == k1) next_pair = pairs;
  else next_pair -= (int)gridDim.x;
  auto fetch = [&] {
    if (next_piece == k1 && next_pair < pairs) {
      next_pair += (int)gridDim.x;
      next_piece = k0;
      const int t0 = first_tile(min(next_pair, pairs - 1), a.epi), t1 = second_tile(min(next_pair, pairs - 1), a.epi);
      from0 = w.codes + ((size_t)t0 * w.kblocks + 2 * k0) * 32 + lane;
      from1 = w.codes + ((size_t)t1 * w.kblocks + 2 * k0) * 32 + lane;
      from_sz = w.sz + (size_t)(sz_t ? t1 : t0) * w.groups * 8 + q * 2;
    }
    if (next_pair < pairs) {
      Slot<GS>& to = ring[next_slot];
      const int second = 2 * next_piece + 1 < w.kblocks ? 32 : 0;   // (past the last block there are no values, and its codes will do)
      copy_async(&to.codes[0][0][lane], from0);
      copy_async(&to.codes[0][1][lane], from1);
      copy_async(&to.codes[1][0][lane], from0 + second);
      copy_async(&to.codes[1][1][lane], from1 + second);
      if (sz_g < 4 / GS)
        copy_async(&to.sz[sz_g][sz_t][q * 2], from_sz + (size_t)min(next_piece * (4 / GS) + sz_g, w.groups - 1) * 8);
      from0 += 64;
      from1 += 64;
      ++next_piece;
      if (++next_slot == kRing) next_slot = 0;
    }
    copies_commit();
  };
  // loaded weights do not change: the first pieces are on their way before the launch before has ended
#pragma unroll 1
  for (int i = 0; i < kRing - 1; ++i) fetch();
  pdl_trigger();
  pdl_wait();

  const bf16* rows[NT];
  bool there[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    there[n] = m0 + n * 8 + g < a.M;
    rows[n] = (const bf16*)a.x + (long long)min(m0 + n * 8 + g, a.M - 1) * a.lda + q * 8;
  }
  auto load = [&](uint4 (*x)[2], int kb) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = kb * 64 + h * 32;
        if constexpr (FAST) {
          x[n][h] = make_uint4(0u, 0u, 0u, 0u);
          if (there[n] && k + q * 8 < w.K) x[n][h] = *(const uint4*)(rows[n] + k);
        } else {
          x[n][h] = load_x(rows[n] - q * 8, k + q * 8, w.K, there[n]);
        }
      }
  };
  int slot = 0, buf = 0;
  float acc[2][NT][4], sum[2][NT][4];
  uint4 xa[NT][2], xb[NT][2];   // a block's tokens, while the next one's are on their way
  if (k0 < k1) load(xa, 2 * k0);
  for (int pair = blockIdx.x; pair < pairs; pair += gridDim.x, buf ^= 1) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][n][i] = 0.f;
#pragma unroll 1
    for (int piece = k0; piece < k1; ++piece) {
      copies_wait<kRing - 2>();
      __syncwarp();
      fetch();   // (into the slot that was read last)
      load(xb, 2 * piece + 1);
      multiply<NT, GS, 0>(ring[slot], lane, g, xa, sum, acc);
      load(xa, piece + 1 < k1 ? 2 * piece + 2 : 2 * k0);
      multiply<NT, GS, 1>(ring[slot], lane, g, xb, sum, acc);
      if (++slot == kRing) slot = 0;
    }
    float* part = parts + buf * kWarps * kPart;   // (two in turn: one barrier a pair)
    put_sums<NT>(part + warp * kPart, acc, g, q);
    __syncthreads();
    auto over_warps = [&](int m, int row) {
      const float* p = part + m * kPitch + row;
      float v = p[0];
#pragma unroll
      for (int i = 1; i < kWarps; ++i) v += p[i * kPart];
      return v;
    };
    if (ranks == 1) {
      finish<NT>(a, pair, m0, 1, 0, threadIdx.x, 256, over_warps);
    } else {   // (one pair a CTA)
      float* sums = parts + (buf ^ 1) * kWarps * kPart;
      for (int e = threadIdx.x; e < NT * 8 * 32; e += 256) sums[(e >> 5) * kPitch + (e & 31)] = over_warps(e >> 5, e & 31);
      cluster_sync();
      finish<NT>(a, pair, m0, ranks, rank, threadIdx.x, 256, [&](int m, int row) { return over_ranks(sums + m * kPitch + row, ranks); });
      cluster_sync();   // nobody leaves while its sums are read
    }
  }
  copies_wait<0>();
}

template <int NT, int GS>
constexpr size_t smem_of() {
  return sizeof(Slot<GS>) * kWarps * kRing + sizeof(float) * 2 * kWarps * NT * 8 * kPitch;
}

template <int NT, int GS>
cudaError_t init_gs() {
  static_assert(kHeld * (smem_of<NT, GS>() + 1024) <= 228 * 1024, "shared memory");
  const cudaError_t e = cudaFuncSetAttribute(w4_gemm_kernel<NT, GS, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of<NT, GS>());
  return e != cudaSuccess ? e : cudaFuncSetAttribute(w4_gemm_kernel<NT, GS, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of<NT, GS>());
}

// CTAs that share a pair of tiles.  Their join costs a microsecond: 1 row x 2048 x 2048 2.7 us, by two CTAs 3.2; 1 x 1024 x 4096
// by four 3.2, by two 3.7.
int few_ranks(const W4Args& a, long long ctas) {
  return a.w.kblocks < 6 * kWarps ? 1 : w4_ranks(ctas, a.w.kblocks, 2 * kWarps, kRanks, a.num_sms);
}

template <int NT, int GS>
cudaError_t launch_few(const W4Args& a, cudaStream_t st) {
  const int pairs = a.w.tiles / 2, tiles = (a.M + NT * 8 - 1) / (NT * 8);
  const int ranks = few_ranks(a, (long long)pairs * tiles);
  // pairs beyond what the SMs hold at once follow one another in a CTA
  const int held = kHeld * a.num_sms;
  const int across = ranks > 1 || pairs <= held ? pairs : std::max(1, held / std::min(tiles, held));
  const Overlap overlap;
  return launch_kernel_cluster(a.vec && a.w.K % 8 == 0 ? w4_gemm_kernel<NT, GS, true> : w4_gemm_kernel<NT, GS, false>, dim3(across, tiles, ranks), dim3(256),
                               smem_of<NT, GS>(), st, dim3(1, 1, ranks), a);
}
template <int NT>
cudaError_t launch_nt(const W4Args& a, cudaStream_t st) {
  return a.w.group == 128 ? launch_few<NT, 4>(a, st) : a.w.group == 64 ? launch_few<NT, 2>(a, st) : launch_few<NT, 1>(a, st);
}

unsigned blocks_of(long long threads) { return (unsigned)((threads + 255) / 256); }

}  // namespace

cudaError_t init_w4_kernels() {
  cudaError_t e = init_gs<1, 1>();
  if (e == cudaSuccess) e = init_gs<1, 2>();
  if (e == cudaSuccess) e = init_gs<1, 4>();
  if (e == cudaSuccess) e = init_gs<2, 1>();
  if (e == cudaSuccess) e = init_gs<2, 2>();
  if (e == cudaSuccess) e = init_gs<2, 4>();
  if (e == cudaSuccess) e = init_w4_tc_kernels();
  return e;
}

W4Kernel w4_kernel(const W4Args& a) {
  if (a.M <= 8) return W4_FEW;
  if (!a.vec) return W4_TILES;   // (TMA takes aligned rows only)
  if (w4_forced() >= 0) return (W4Kernel)w4_forced();
  // Tiles of 16 rows that go through the matrix each, from L2 after the first, or the tcgen05 kernel (an SM a CTA, a longer
  // start), whichever takes less by these times, in 10 ns: of tiles a start, rounds, blocks of 64 ks of a warp (faster where an
  // SM has one CTA) and a cluster's join; of tcgen05 a start and pieces of 128 ks of a CTA, longer where its sums are many.  us,
  // tiles / tcgen05, groups of 128: 16 rows x 4096 x 4096 5.8 / 7.7, x 8192 x 8192 13.5 / 16.3, x 65536 x 2048 26.7 / 26.1; 32 x
  // 2048 x 4096 5.8 / 6.7, x 3000 x 5000 9.3 / 8.2, x 8192 x 8192 25.6 / 16.7, x 1024 x 16384 13.3 / 15.6; 64 x 4096 x 1024
  // 6.4 / 6.7, x 1024 x 4096 5.8 / 7.4, x 2048 x 8192 13.5 / 10.6; 96 x 4096 x 1024 9.3 / 6.8; groups of 32, 16 x 4096 x 8192
  // 14.3 / 12.1, 64 x 512 x 8192 9.2 / 15.2, 48 x 8192 x 1024 9.9 / 8.2.
  const long long tiles = (a.M + 15) / 16, ctas = a.w.tiles / 2 * tiles;
  const int ranks = few_ranks(a, ctas);
  const long long rounds = (ctas * ranks + kHeld * a.num_sms - 1) / (kHeld * a.num_sms), blocks = (a.w.kblocks + kWarps * ranks - 1) / (kWarps * ranks);
  const bool g32 = a.w.group == 32, alone = !g32 && ctas * ranks <= a.num_sms;
  const long long as_tiles = 150 + rounds * (100 + blocks * (alone ? 45 : 70)) + (ranks > 1 ? 200 : 0);
  const long long as_tc = 500 + W4TcPlan(a, w4_tc_tokens(a.M)).pieces * (a.M <= 32 ? (g32 ? 45 : 35) : g32 ? 70 : 40);
  return as_tc < as_tiles ? W4_TC : W4_TILES;
}

cudaError_t launch_w4_gemm(const W4Args& a, cudaStream_t st) {
  switch (w4_kernel(a)) {
    case W4_FEW: return launch_nt<1>(a, st);
    case W4_TILES: return launch_nt<2>(a, st);
    default: return launch_w4_tc(a, st);
  }
}

// For tests: the kernel of this thread's products of more than 8 aligned tokens (else: by the rule), and what a product is
// planned to be: its kernel and, on tcgen05, the tokens of a unit, CTAs, those that share a unit of the last round, and
// whether there are full rounds before it.
extern "C" void ravel_debug_w4(int kernel) { w4_forced() = kernel == W4_TILES || kernel == W4_TC ? kernel : -1; }
// Fault injection for tests: this thread's next `launches` of the tcgen05 kernel load no tokens; every wait for them gives up
// after a second, the CTAs give back what they hold and raise ERR_TIMEOUT, and outputs are not valid (no fault, no hang).
extern "C" void ravel_debug_w4_withhold(int launches) { w4_withheld() = launches; }
extern "C" void ravel_debug_w4_plan(int N, int K, int group, int M, int aligned, int sms, int* out) {
  W4Args a{W4Matrix(N, K, group), nullptr, nullptr, nullptr, M, K, N, EPI_STORE, 0, aligned, sms, nullptr};
  out[0] = w4_kernel(a);
  if (out[0] != W4_TC) return;
  out[1] = w4_tc_tokens(M);
  const W4TcPlan plan(a, out[1]);
  out[2] = plan.grid;
  out[3] = plan.ranks;
  out[4] = (a.w.tiles + 7) / 8 * ((M + out[1] - 1) / out[1]) >= sms;
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
