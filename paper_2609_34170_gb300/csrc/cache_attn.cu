// Attention over the 8-bit context cache for few query rows (single tokens,
// short runs of queries) and in fp32, and the attention mass of its tokens.
//
// Rows: query i, head g of a KV head's group is row r = i * G + g; a CTA owns a
// tile of 8 rows (where a robot's query rows are no more) or 16 of one (robot, KV
// head) and a share (split) of the tokens that the tile sees; its four warps take
// turns at units of 16 * NT tokens, each with its own running maximum, sum and
// output, which are joined in shared memory and then across the splits: up to 8 of
// them as a cluster, through its shared memory, more through L2.
//
// What bounds it on long caches is the cache's bytes: 8 query rows against 16 tokens
// cost one m16n8k16 MMA per 16 dims whatever the group's size, so a token's time does
// not depend on G.  A warp's units (K and V of 16 to 64 tokens, 8 KB) come by TMA into
// a ring of its own that nobody else waits for, three units ahead, 96 KB a CTA and
// two CTAs an SM; loads to registers held half of that in flight (4 robots of 131071
// tokens: 149 us, now 56).  From there the codes go to registers 16 bytes at a time
// and are widened there (e4m3 -> f16 is exact): within an MMA the dims of q k (and the
// tokens of p v) may come in any order that both operands share, so that no load is
// narrower.  tcgen05 would want the widened codes in shared memory first and 128 rows
// to work on.  Few rows take K as the A operand, 16 tokens by 8 rows, and P transposed
// in registers: half the MMAs and exponentials of a tile of 16 rows that is half empty.
//
// Measured (one query per robot, bf16; alone / in a chain of calls): one robot of 816 tokens,
// head dim 256: 10.1 / 8.1 us, a chain of launch, Q, one unit per warp, two joins; 64 robots of
// 1024 to 2048: 19.3 / 17.2 us for 50 MB (2.9 TB/s; a round of unequal robots); 4 robots of
// 131071, 4 heads of 64: 56.5 / 51.7 us for 269 MB (5.2 TB/s; alone, CTAs are on the SMs for
// three quarters of the time: arithmetic 48 % busy meanwhile, tensor pipe 17, exponentials 9, and
// what warps wait for most is their units).  3 robots, 37 queries, 301 tokens in fp32: 9.4 / 8.0.
//
// Numbers: q is scaled by a power of two per row to a maximum in [2^14, 2^15) and
// held in f16 -- exactly for bf16 inputs (8 significant bits; what lies 2^38
// below the row's largest is dropped), in two f16 pieces for fp32 ones (23
// bits).  Products with the codes are exact in the tensor core's fp32 sums;
// block exponents and row scales are applied to the sums in fp32.  P is scaled
// times 2^ve of its block, relative to the largest such product of the row,
// scaled to at most 2^15: one f16 piece (11 bits) for bf16 results, two for fp32
// ones; what contributes less than 2^-39 of the largest is dropped.  The sum of P
// itself takes 2^ve out again, per block.  Both references (the row's largest
// score, and its largest score + ve) are rounded up to integers in the log2
// domain, so that every change of reference is an exact power of two.  Maxima,
// sums and outputs are fp32.
#include <algorithm>

#include "cache_index.h"
#include "cache_tc.cuh"
#include "launch.h"

namespace ravel {
namespace {

constexpr int RW = 4;             // warps of a CTA
constexpr float kPExp = 15.f;     // P's largest value is 2^kPExp

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}

// fp32's sums over MMAs: the tensor core cuts its sums off rather than rounding them, and
// over a long chain that adds up, so that each pair of pieces starts from zero.
__device__ __forceinline__ void add4(float (&d)[4], const float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const float2 y = add2(make_float2(d[i], d[i + 1]), make_float2(x[i], x[i + 1]));
    d[i] = y.x;
    d[i + 1] = y.y;
  }
}

__device__ __forceinline__ uint32_t word(const uint4& x, int i) { return i == 0 ? x.x : (i == 1 ? x.y : (i == 2 ? x.z : x.w)); }

// An 8 x 8 tile of 16-bit values, a row per four lanes, transposed across the warp.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Query rows r0 .. r0 + 15 into shared memory as the A fragments of the MMAs:
// word (piece, k-step, lane) holds rows lane / 4 and + 8, dims 64 j + 16 (lane % 4)
// + 4 s + 0 .. 3 of k-step 4 j + s.  Rows that do not exist are zeros.  fac[r]:
// 2^exponent taken out of the row, times the softmax scale.
// after_loads is called with the loads on their way.
template <int HDP, int NP, typename T, int THREADS, typename F>
__device__ __forceinline__ void stage_q(const CacheAttnArgs& a, const Sight& s, int b, int h, int r0, uint32_t* frag,
                                        float* fac, F after_loads) {
  constexpr int TPR = HDP / 16, ITEMS = (16 * TPR + THREADS - 1) / THREADS;   // threads per row, rows' pieces per thread
  float x[ITEMS][16];
#pragma unroll
  for (int z = 0; z < ITEMS; ++z) {
    const int w = threadIdx.x + z * THREADS, lr = w / TPR, d = (w % TPR) * 16, r = r0 + lr;
    const int i = (int)a.by_G.of((uint32_t)r);
    if (w < 16 * TPR && i < s.count && d < a.c.hd) {
      const T* row = (const T*)a.q + (size_t)((long long)b * a.q_robot + (long long)i * a.q_token) +
                     (size_t)(h * a.G + r - i * a.G) * a.c.hd;
      load16(row, d, a.c.hd, a.vec, x[z]);
    } else {
#pragma unroll
      for (int q = 0; q < 16; ++q) x[z][q] = 0.f;
    }
  }
  after_loads();
#pragma unroll
  for (int z = 0; z < ITEMS; ++z) {
    const int w = threadIdx.x + z * THREADS;
    uint32_t top = 0u;   // bits of the largest magnitude: NaN counts as larger than all
#pragma unroll
    for (int q = 0; q < 16; ++q) top = max(top, __float_as_uint(x[z][q]) & 0x7fffffffu);
    if (w < 16 * TPR) atomicMax((unsigned*)&fac[w / TPR], top);
  }
  __syncthreads();
#pragma unroll
  for (int z = 0; z < ITEMS; ++z) {
    const int w = threadIdx.x + z * THREADS;
    if (w >= 16 * TPR) break;
    const int lr = w / TPR, d = (w % TPR) * 16;
    const uint32_t top = ((const unsigned*)fac)[lr];
    // factor 2^(14 - exponent), at most 2^126 (rows below 2^-112 keep fewer bits)
    const int e = min(14 - ((int)(top >> 23) - 127), 126);
    const bool bad = top >= 0x7f800000u;
    const float f = bad ? __int_as_float(0x7fffffff) : exp2i(e);
    // dims d .. d + 15 are k-steps 4 j + 0 .. 3 of lane (4 (row % 8) + c)
    const int j = d / 64, c = (d / 16) % 4, lane = (lr & 7) * 4 + c;
#pragma unroll
    for (int s4 = 0; s4 < 4; ++s4) {
      const float y0 = x[z][4 * s4] * f, y1 = x[z][4 * s4 + 1] * f, y2 = x[z][4 * s4 + 2] * f, y3 = x[z][4 * s4 + 3] * f;
      uint32_t lo = pack_f16x2(y0, y1), hi = pack_f16x2(y2, y3);
      // fragment registers: a0 (row, dims 0 1), a1 (row + 8, 0 1), a2 (row, 2 3), a3 (row + 8, 2 3)
      uint32_t* at = frag + ((4 * j + s4) * 32 + lane) * 4 + (lr >> 3);
      at[0] = lo;
      at[2] = hi;
      if (NP == 2) {
        at += HDP / 16 * 128;
        at[0] = pack_f16x2(y0 - f16lo(lo), y1 - f16hi(lo));
        at[2] = pack_f16x2(y2 - f16lo(hi), y3 - f16hi(hi));
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < 16) {
    const uint32_t top = ((const unsigned*)fac)[threadIdx.x];
    const int e = min(14 - ((int)(top >> 23) - 127), 126);
    fac[threadIdx.x] = exp2i(-max(e, -126)) * a.scale_log2;   // (e >= -114 for finite rows)
  }
  __syncthreads();
}

// A warp's unit of 16 NT tokens in shared memory: boxes of IN dims x U tokens as TMA
// swizzles them (16-byte pieces of a row permuted by the row), codes of K or of V.
template <int HDP>
struct Unit {
  static constexpr int NT = HDP == 64 ? 4 : (HDP == 128 ? 2 : 1);   // blocks of 16 tokens
  static constexpr int U = 16 * NT, IN = HDP % 128 ? 64 : 128, BOXES = HDP / IN;
  static constexpr uint32_t bytes = U * HDP;
  // byte of a token's row where 16-byte piece p (of HDP / 16) lies
  static __device__ __forceinline__ uint32_t at(int row, int p) {
    constexpr int PP = IN / 16;
    const int q = p % PP;
    return (uint32_t)(p / PP * U * IN + row * IN + ((IN == 128 ? q ^ (row & 7) : q ^ ((row >> 1) & 3)) * 16));
  }
};

// Key fragments of a block of 16 tokens: tokens g and g + 8, dims 64 j + 16 c .. + 15.
template <int HDP>
struct KeyUnit {
  uint4 w[2][HDP / 64];
  __device__ __forceinline__ void load(uint32_t unit, int row0, int g, int c) {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int j = 0; j < HDP / 64; ++j) w[hh][j] = lds_u4(unit + Unit<HDP>::at(row0 + g + 8 * hh, 4 * j + c));
  }
};

// Value fragments: tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9, 16 dims of each 128 from 16 g on
// (8 of a last 64 from 8 g on).
template <int HDP>
struct ValueUnit {
  uint32_t w[4][HDP / 32];
  __device__ __forceinline__ void load(uint32_t unit, int row0, int g, int c) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int row = row0 + 2 * c + (t & 1) + 4 * (t & 2);
#pragma unroll
      for (int j = 0; j < HDP / 128; ++j) {
        const uint4 x = lds_u4(unit + Unit<HDP>::at(row, 8 * j + g));
        w[t][4 * j] = x.x;
        w[t][4 * j + 1] = x.y;
        w[t][4 * j + 2] = x.z;
        w[t][4 * j + 3] = x.w;
      }
      if (HDP % 128) {
        const uint32_t at = unit + Unit<HDP>::at(row, HDP / 128 * 8 + (g >> 1)) + 8u * (g & 1);
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[t][HDP / 32 - 2]), "=r"(w[t][HDP / 32 - 1]) : "r"(at));
      }
    }
  }
  // dim of column n of MMA tile (word wi, byte i)
  static __device__ __forceinline__ int dim(int wi, int i, int n) {
    return wi < HDP / 128 * 4 ? wi / 4 * 128 + 16 * n + wi % 4 * 4 + i
                              : HDP / 128 * 128 + 8 * n + (wi - HDP / 128 * 4) * 4 + i;
  }
};

template <int HDP, int NP, int RT>
struct RowsShape {
  static constexpr int frag = NP * (HDP / 16) * 512;   // bytes of Q's fragments
  // bf16's few rows hold Q in registers: its place then takes what the splits send each other
  static constexpr bool send = RT == 8 && NP == 1;
  static constexpr int pad = send ? 128 : 0;           // (their shares are rounded up)
  // units in flight per warp, K and V (24 KB; fp32's take 16: its fragments are twice as many)
  static constexpr int D = NP == 2 ? 2 : 3;
  static constexpr int ring = RW * D * 2 * (int)Unit<HDP>::bytes;
  // the warps' outputs, over the ring: rows JS floats apart, four floats more per 32 dims, so
  // that the 16-byte pieces of a store (two rows, every 32nd or 16th dim) fall on different banks
  static constexpr int JS = RT == 8 ? (HDP == 64 ? 84 : (HDP == 128 ? 148 : (HDP == 192 ? 228 : 292)))
                                    : (HDP == 64 ? 72 : (HDP == 128 ? 144 : (HDP == 192 ? 240 : 304)));
  static __device__ __forceinline__ int pos(int row, int d) { return row * JS + d + (d >> 5) * 4; }
  static constexpr int join = RW * RT * JS * 4 + RT * HDP * 4;   // and their sum
  static constexpr int bytes = frag + pad + (ring > join ? ring : join);
  static_assert(!send || frag + pad >= RT * HDP * 4 + 7 * 16, "what the splits send");
};

struct RowsMaps {
  CUtensorMap k, v;   // a layer's codes [B Hkv T][HDP] in boxes of Unit::IN dims x U rows, swizzled
};

template <int HDP, int NP, int RT, typename T>
__global__ void __launch_bounds__(RW * 32, 2) cache_rows_kernel(const __grid_constant__ RowsMaps maps, CacheAttnArgs a) {
  using Un = Unit<HDP>;
  using Shape = RowsShape<HDP, NP, RT>;
  constexpr int NT = Un::NT, U = Un::U, KS = HDP / 16, D = Shape::D;
  extern __shared__ __align__(1024) uint8_t smem[];
  float* joint = (float*)smem;                          // [RW][RT][JS] outputs of the warps, over the ring
  float* mine = joint + RW * RT * Shape::JS;            // [RT][HDP] their sum
  uint32_t* frag = (uint32_t*)(smem + Shape::bytes - Shape::pad - Shape::frag);   // [NP][KS][32][4]
  __shared__ float fac[16];
  __shared__ float2 warp_ml[RW][16], split_w[16];
  __shared__ unsigned last;
  __shared__ uint64_t arrived[RW][D];
  __shared__ float split_wt[8][16];
  __shared__ float2 split_in[Shape::send ? 8 : 1][8];   // the splits' (max, sum)

  const int b = blockIdx.z + a.b0, h = blockIdx.y, tile = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const CacheLayer& L = a.c;
  const int r0 = a.i0 * a.G + tile * RT, rows = min(RT, a.i1 * a.G - r0);
  const size_t head = (size_t)b * L.Hkv + h, here = (size_t)blockIdx.z * L.Hkv + h;   // (of the cache, of this launch)
  if (smem_u32(smem) & 1023u) {   // (the swizzled layouts count on it)
    if (threadIdx.x == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  pdl_trigger();
  if (lane == 0) {
    for (int x = 0; x < D; ++x) mbar_init(&arrived[warp][x], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (threadIdx.x < 16) fac[threadIdx.x] = 0.f;
  pdl_wait();   // (the launch before may still write what is read from here on)
  Sight s;
  if (!robot_sight(a, b, s) && threadIdx.x == 0 && blockIdx.x == 0 && h == 0) raise_error(a.err, ERR_SHAPE);
  T* out0 = (T*)a.out + (size_t)((long long)b * a.out_robot) + (size_t)h * a.G * L.hd;
  auto out_row = [&](int r) {
    const int i = (int)a.by_G.of((uint32_t)r);
    return out0 + (size_t)((long long)i * a.out_token) + (size_t)(r - i * a.G) * L.hd;
  };
  if (r0 >= s.count * a.G || s.len == 0) {   // nothing to see: zeros
    if (split == 0)
      for (int w = threadIdx.x; w < rows * L.hd; w += RW * 32) out_row(r0 + w / L.hd)[w % L.hd] = from_f32<T>(0.f);
    if (split == 0 && a.mass && threadIdx.x < rows)
      a.row_ml[head * a.n * a.G + r0 + threadIdx.x] = make_float2(0.f, 0.f);
    return;
  }
  tile_sight(a, s, r0, r0 + RT - 1, U);
  const int u0 = (int)((long long)s.units * split / a.splits), u1 = (int)((long long)s.units * (split + 1) / a.splits);

  // each warp's ring of units: its own loads, which it alone waits for
  const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * D) * 2u * Un::bytes;
  auto unit_token = [&](int u) { return (u < s.sink_units ? u : u - s.sink_units + s.from) * U; };
  uint64_t pol;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
  auto fetch = [&](int u, int slot) {   // (lane 0)
    const int row = (int)(head * L.T) + unit_token(u);
    const uint32_t to = ring + (uint32_t)slot * 2u * Un::bytes, bar = smem_u32(&arrived[warp][slot]);
    mbar_expect_tx(&arrived[warp][slot], 2u * Un::bytes);
#pragma unroll
    for (int x = 0; x < Un::BOXES; ++x) {
      tma_load_2d_el(&maps.k, bar, to + (uint32_t)(x * U * Un::IN), x * Un::IN, row, pol, 1u);
      tma_load_2d_el(&maps.v, bar, to + Un::bytes + (uint32_t)(x * U * Un::IN), x * Un::IN, row, pol, 1u);
    }
  };
  __syncthreads();
  // (Q's loads first: behind the first units of all CTAs, 29 MB, they took 5 us)
  stage_q<HDP, NP, T, RW * 32>(a, s, b, h, r0, frag, fac, [&]() {
    if (lane == 0)
      for (int x = 0; x < D; ++x)
        if (u0 + warp + RW * x < u1) fetch(u0 + warp + RW * x, x);
    __syncwarp();
  });
  // this lane's two rows: scores of rows g, g + 8 by tokens 2 c, 2 c + 1, or (RT = 8) of tokens
  // g, g + 8 by rows 2 c, 2 c + 1
  const int row_of[2] = {RT == 8 ? 2 * c : g, RT == 8 ? 2 * c + 1 : g + 8};
  const RowMask mk[2] = {row_mask(a, s, r0 + row_of[0]), row_mask(a, s, r0 + row_of[1])};
  const float rf[2] = {fac[row_of[0]], fac[row_of[1]]};
  // tokens that every row that exists sees: [full_lo, full_hi) and below a.sinks
  const RowMask first = row_mask(a, s, r0), lastm = row_mask(a, s, min(r0 + RT - 1, s.count * a.G - 1));
  const int full_hi = first.hi, full_lo = lastm.lo;

  const int8_t *KE = L.ke + head * (L.T / 16), *VE = L.ve + head * (L.T / 16);

  // outputs: rows g, g + 8 by dims 2 c, 2 c + 1 of each 8, or (RT = 8) dims g, g + 8 of each 16 by
  // rows 2 c, 2 c + 1
  constexpr int OT = RT == 8 ? HDP / 16 : HDP / 8;
  float o[OT][4];
#pragma unroll
  for (int t = 0; t < OT; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q) o[t][q] = 0.f;
  uint32_t qb[RT == 8 && NP == 1 ? KS : 1][2];   // RT = 8: Q's fragments as B operands
  if (RT == 8 && NP == 1) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qb[ks][0] = frag[(ks * 32 + lane) * 4];
      qb[ks][1] = frag[(ks * 32 + lane) * 4 + 2];
    }
  }
  const bool cluster = a.splits > 1 && a.splits <= 8;
  if (Shape::send && cluster) cluster_arrive_release();   // (Q's place is free)
  float m[2] = {-INFINITY, -INFINITY}, W[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  // the exponents of a unit's blocks, one byte each
  auto exps_of = [&](const int8_t* e, int j0) -> uint32_t {
    if (NT == 4) return *(const uint32_t*)(e + j0 / 16);
    if (NT == 2) return *(const uint16_t*)(e + j0 / 16);
    return (uint8_t)e[j0 / 16];
  };
  int u = u0 + warp;
  uint32_t kes = 0u, ves = 0u;
  if (u < u1) {
    kes = exps_of(KE, unit_token(u));
    ves = exps_of(VE, unit_token(u));
  }
  int slot = 0;
  uint32_t phase = 0u;
  for (; u < u1; u += RW) {
    const int j0 = unit_token(u);
    const uint32_t unit = ring + (uint32_t)slot * 2u * Un::bytes;
    float kf[NT];
    int ve[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      kf[t] = exp2i((int)(int8_t)(kes >> (8 * t)));
      ve[t] = (int)(int8_t)(ves >> (8 * t));
    }
    const int un = u + RW;
    if (un < u1) {
      kes = exps_of(KE, unit_token(un));
      ves = exps_of(VE, unit_token(un));
    }
    if (!wait_phase(&arrived[warp][slot], phase)) {
      // nothing is issued any more, and what is on its way lands before the shared memory is
      // written by others or goes away
      const LoadsLeft left = loads_left((u - u0 - warp) / RW, (u1 - u0 - warp + RW - 1) / RW, D);
      for (int x = left.first; x < left.end; ++x) mbar_wait(&arrived[warp][x % D], load_parity(x, D));
      if (lane == 0) raise_error(a.err, ERR_TIMEOUT);
      break;
    }
    KeyUnit<HDP> kr[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) kr[t].load(unit, 16 * t, g, c);
    // sc[t][hh][rr][q]: this lane's row rr, token 8 hh + 2 c + q of block t, or (RT = 8, q = 0) token
    // 8 hh + g.  Few rows take K as the MMAs' A operand, 16 tokens by 8 rows: half the MMAs.
    constexpr int QN = RT == 8 ? 1 : 2;
    float sc[NT][2][2][QN];
    if constexpr (RT == 8) {
      // (where a unit has few tiles of scores, each has AC accumulators in turn: an MMA waits
      // for the one before it in its tile)
      constexpr int AC = 4 / NT;
      float sa[AC][NT][4];
#pragma unroll
      for (int x = 0; x < AC; ++x)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) sa[x][t][q] = 0.f;
#pragma unroll
      for (int j = 0; j < HDP / 64; ++j)
#pragma unroll
        for (int s4 = 0; s4 < 4; ++s4)
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const uint32_t w0 = word(kr[t].w[0][j], s4), w1 = word(kr[t].w[1][j], s4);
            const uint4 ka = make_uint4(e4m3_lo(w0), e4m3_lo(w1), e4m3_hi(w0), e4m3_hi(w1));
            if constexpr (NP == 1) {
              mma_f16(sa[s4 % AC][t], ka, qb[4 * j + s4][0], qb[4 * j + s4][1]);
            } else {
              float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int p = NP - 1; p >= 0; --p) {
                const uint32_t* at = frag + ((p * KS + 4 * j + s4) * 32 + lane) * 4;
                mma_f16(x, ka, at[0], at[2]);
              }
              add4(sa[s4 % AC][t], x);
            }
          }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x = sa[0][t][q];
#pragma unroll
          for (int y = 1; y < AC; ++y) x += sa[y][t][q];
          sc[t][q >> 1][q & 1][0] = x;
        }
    } else {
      float sa[NT][2][4];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int q = 0; q < 4; ++q) sa[t][hh][q] = 0.f;
#pragma unroll
      for (int j = 0; j < HDP / 64; ++j)
#pragma unroll
        for (int s4 = 0; s4 < 4; ++s4) {
          uint4 qa[NP];
#pragma unroll
          for (int p = 0; p < NP; ++p) qa[p] = *(const uint4*)(frag + ((p * KS + 4 * j + s4) * 32 + lane) * 4);
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
              const uint32_t w = word(kr[t].w[hh][j], s4), k0 = e4m3_lo(w), k1 = e4m3_hi(w);
              if constexpr (NP == 1) {
                mma_f16(sa[t][hh], qa[0], k0, k1);
              } else {
                float x[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(x, qa[NP - 1], k0, k1);
                mma_f16(x, qa[0], k0, k1);
                add4(sa[t][hh], x);
              }
            }
        }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int q = 0; q < 4; ++q) sc[t][hh][q >> 1][(q & 1) % QN] = sa[t][hh][q];
    }
    // token of sc[t][hh][.][q], from the block's first on
    auto place = [&](int hh, int q) { return RT == 8 ? 8 * hh + g : 8 * hh + 2 * c + q; };
    // scores in the log2 domain; hidden ones -inf
    const bool full = j0 + U <= full_hi && (j0 >= full_lo || j0 + U <= a.sinks);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int rr = 0; rr < 2; ++rr)
#pragma unroll
          for (int q = 0; q < QN; ++q) {
            sc[t][hh][rr][q] *= rf[rr] * kf[t];
            if (!full && !mk[rr].sees(j0 + 16 * t + place(hh, q))) sc[t][hh][rr][q] = -INFINITY;
          }
    }
    if (a.scores) {   // kept for the mass
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int rr = 0; rr < 2; ++rr)
            if (row_of[rr] < rows) {
              float* to = a.scores + (here * (a.i1 - a.i0) * a.G + r0 - a.i0 * a.G + row_of[rr]) * a.mass_pitch + j0 + 16 * t + place(hh, 0);
              if (RT == 8) *to = sc[t][hh][rr][0];
              else *(float2*)to = make_float2(sc[t][hh][rr][0], sc[t][hh][rr][QN - 1]);
            }
    }
    float mu[2], wu[2];   // the references, 0 while the row has seen nothing
    bool same = true;
    float fl[2], fo[2];
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      float mx = -INFINITY, wx = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float x = fmaxf(sc[t][0][rr][0], sc[t][1][rr][0]);
        if (QN == 2) x = fmaxf(x, fmaxf(sc[t][0][rr][QN - 1], sc[t][1][rr][QN - 1]));
        mx = fmaxf(mx, x);
        wx = fmaxf(wx, x + (float)ve[t]);
      }
      // over the lanes that hold the row's other tokens
#pragma unroll
      for (int o2 = RT == 8 ? 4 : 1; o2 <= (RT == 8 ? 16 : 2); o2 <<= 1) {
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o2));
        wx = fmaxf(wx, __shfl_xor_sync(0xffffffffu, wx, o2));
      }
      const float mn = fmaxf(m[rr], ceilf(mx)), wn = fmaxf(W[rr], ceilf(wx));
      mu[rr] = mn == -INFINITY ? 0.f : mn;
      wu[rr] = wn == -INFINITY ? 0.f : wn;
      same = same && mn == m[rr] && wn == W[rr];
      fl[rr] = pow2f_down(m[rr] - mu[rr]);
      fo[rr] = pow2f_down(W[rr] - wu[rr]);
      m[rr] = mn;
      W[rr] = wn;
    }
    // (most units change nothing: the maxima settle early)
    if (__any_sync(0xffffffffu, !same)) {
      l[0] *= fl[0];
      l[1] *= fl[1];
#pragma unroll
      for (int t = 0; t < OT; ++t) {
        o[t][0] *= fo[0];
        o[t][1] *= fo[RT == 8 ? 1 : 0];
        o[t][2] *= fo[RT == 8 ? 0 : 1];
        o[t][3] *= fo[1];
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float p[2][2][QN];   // [hh][rr][q]
#pragma unroll
      for (int rr = 0; rr < 2; ++rr) {
        const float vf = fmaxf((float)ve[t], wu[rr] - mu[rr] - kVeBelow);
        const float nb = kPExp + vf - wu[rr];
        float sum = 0.f;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int q = 0; q < QN; ++q) {
            p[hh][rr][q] = NP == 2 ? exp2f(sc[t][hh][rr][q] + nb) : fast_exp2(sc[t][hh][rr][q] + nb);
            sum += p[hh][rr][q];
          }
        l[rr] = fmaf(sum, pow2f(wu[rr] - mu[rr] - vf), l[rr]);
      }
      ValueUnit<HDP> vr;
      vr.load(unit + Un::bytes, 16 * t, g, c);
      if constexpr (RT == 8) {
        // P as the B operand (tokens 2 c, 2 c + 1, row g): the 8 x 8 tiles of scores transposed
        uint32_t pb[NP][2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const uint32_t x = pack_f16x2(p[hh][0][0], p[hh][1][0]);
          pb[0][hh] = transpose8x8(x);
          if (NP == 2) pb[NP - 1][hh] = transpose8x8(pack_f16x2(p[hh][0][0] - f16lo(x), p[hh][1][0] - f16hi(x)));
        }
#pragma unroll
        for (int wi = 0; wi < HDP / 32; ++wi) {
          // bytes i of two tokens' words side by side: dims g (even i) and g + 8 (odd i) of a tile
          const uint32_t x0 = __byte_perm(vr.w[0][wi], vr.w[1][wi], 0x5140), x1 = __byte_perm(vr.w[2][wi], vr.w[3][wi], 0x5140);
          const uint32_t y0 = __byte_perm(vr.w[0][wi], vr.w[1][wi], 0x7362), y1 = __byte_perm(vr.w[2][wi], vr.w[3][wi], 0x7362);
          const uint4 xa = make_uint4(e4m3_lo(x0), e4m3_hi(x0), e4m3_lo(x1), e4m3_hi(x1));
          const uint4 ya = make_uint4(e4m3_lo(y0), e4m3_hi(y0), e4m3_lo(y1), e4m3_hi(y1));
          if constexpr (NP == 1) {
            mma_f16(o[2 * wi], xa, pb[0][0], pb[0][1]);
            mma_f16(o[2 * wi + 1], ya, pb[0][0], pb[0][1]);
          } else {
            float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int z = NP - 1; z >= 0; --z) {
              mma_f16(x, xa, pb[z][0], pb[z][1]);
              mma_f16(y, ya, pb[z][0], pb[z][1]);
            }
            add4(o[2 * wi], x);
            add4(o[2 * wi + 1], y);
          }
        }
      } else {
        uint4 pa[NP];
        pa[0] = make_uint4(pack_f16x2(p[0][0][0], p[0][0][QN - 1]), pack_f16x2(p[0][1][0], p[0][1][QN - 1]),
                           pack_f16x2(p[1][0][0], p[1][0][QN - 1]), pack_f16x2(p[1][1][0], p[1][1][QN - 1]));
        if (NP == 2)
          pa[NP - 1] = make_uint4(pack_f16x2(p[0][0][0] - f16lo(pa[0].x), p[0][0][QN - 1] - f16hi(pa[0].x)),
                                  pack_f16x2(p[0][1][0] - f16lo(pa[0].y), p[0][1][QN - 1] - f16hi(pa[0].y)),
                                  pack_f16x2(p[1][0][0] - f16lo(pa[0].z), p[1][0][QN - 1] - f16hi(pa[0].z)),
                                  pack_f16x2(p[1][1][0] - f16lo(pa[0].w), p[1][1][QN - 1] - f16hi(pa[0].w)));
#pragma unroll
        for (int wi = 0; wi < HDP / 32; ++wi) {
          // bytes i of two tokens' words side by side
          const uint32_t x0 = __byte_perm(vr.w[0][wi], vr.w[1][wi], 0x5140), y0 = __byte_perm(vr.w[0][wi], vr.w[1][wi], 0x7362);
          const uint32_t x1 = __byte_perm(vr.w[2][wi], vr.w[3][wi], 0x5140), y1 = __byte_perm(vr.w[2][wi], vr.w[3][wi], 0x7362);
          const uint32_t b0[4] = {e4m3_lo(x0), e4m3_hi(x0), e4m3_lo(y0), e4m3_hi(y0)};
          const uint32_t b1[4] = {e4m3_lo(x1), e4m3_hi(x1), e4m3_lo(y1), e4m3_hi(y1)};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (NP == 1) {
              mma_f16(o[4 * wi + i], pa[0], b0[i], b1[i]);
            } else {
              float x[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(x, pa[NP - 1], b0[i], b1[i]);
              mma_f16(x, pa[0], b0[i], b1[i]);
              add4(o[4 * wi + i], x);
            }
          }
        }
      }
    }
    // every lane has read the unit: the slot takes the one D turns on
    __syncwarp();
    if (lane == 0 && u + RW * D < u1) fetch(u + RW * D, slot);
    if (++slot == D) {
      slot = 0;
      phase ^= 1u;
    }
  }
  __syncthreads();   // the rings are read: the outputs go over them

  constexpr int QN2 = RT == 8 ? 1 : 2;
  // ---- join the warps: outputs normalised by their own sums, then weighted
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
#pragma unroll
    for (int o2 = RT == 8 ? 4 : 1; o2 <= (RT == 8 ? 16 : 2); o2 <<= 1) l[rr] += __shfl_xor_sync(0xffffffffu, l[rr], o2);
    // (units that every query sees are not masked: a row without a query stops here)
    const bool real = mk[rr].hi > 0;
    if (!real) {
      l[rr] = 0.f;
      m[rr] = -INFINITY;
    }
    const bool has = !(l[rr] <= 0.f);   // (a sum that is not a number stays one)
    const float f = has ? 1.f / l[rr] : 0.f;
    const float e2 = real ? pow2f(W[rr] - m[rr]) : 0.f;
    const int row = row_of[rr];
    if (RT == 8 ? g == 0 : c == 0) warp_ml[warp][row] = make_float2(m[rr], l[rr]);
    float* dst = joint + warp * RT * Shape::JS;
    if (row < rows) {
#pragma unroll
      for (int wi = 0; wi < HDP / 32; ++wi)
#pragma unroll
        for (int q = 0; q < QN2; ++q) {
          float4 x;   // four dims side by side
          if (RT == 8)
            x = make_float4(o[2 * wi % OT][rr], o[2 * wi % OT][2 + rr], o[(2 * wi + 1) % OT][rr], o[(2 * wi + 1) % OT][2 + rr]);
          else
            x = make_float4(o[4 * wi % OT][2 * rr + q], o[(4 * wi + 1) % OT][2 * rr + q], o[(4 * wi + 2) % OT][2 * rr + q],
                            o[(4 * wi + 3) % OT][2 * rr + q]);
          x.x = real ? x.x * f * e2 : 0.f;
          x.y = real ? x.y * f * e2 : 0.f;
          x.z = real ? x.z * f * e2 : 0.f;
          x.w = real ? x.w * f * e2 : 0.f;
          *(float4*)(dst + Shape::pos(row, ValueUnit<HDP>::dim(wi, 0, RT == 8 ? g : 2 * c + q))) = x;
        }
    }
  }
  __syncthreads();
  if (threadIdx.x < RT) {   // the warps' weights, in place of (m, l)
    const int row = threadIdx.x;
    float M = -INFINITY, S = 0.f;
#pragma unroll
    for (int w = 0; w < RW; ++w) M = fmaxf(M, warp_ml[w][row].x);
#pragma unroll
    for (int w = 0; w < RW; ++w) {
      const float2 x = warp_ml[w][row];
      // a NaN sum has no maximum of its own: it counts as it is
      const float wt = x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y);
      warp_ml[w][row].x = wt;
      S += wt;
    }
    const float inv = !(S <= 0.f) ? 1.f / S : 0.f;
#pragma unroll
    for (int w = 0; w < RW; ++w) warp_ml[w][row].x *= inv;
    split_w[row] = make_float2(M, S);
  }
  __syncthreads();
  auto joined = [&](int row, int d) {   // four dims from d on
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < RW; ++w) {
      const float wt = warp_ml[w][row].x;
      const float4 x = *(const float4*)(joint + w * RT * Shape::JS + Shape::pos(row, d));
      acc.x += wt != 0.f ? wt * x.x : 0.f;
      acc.y += wt != 0.f ? wt * x.y : 0.f;
      acc.z += wt != 0.f ? wt * x.z : 0.f;
      acc.w += wt != 0.f ? wt * x.w : 0.f;
    }
    return acc;
  };
  auto store4 = [&](int row, int d, const float4& x) {   // (hd is a multiple of 8)
    T* dst = out_row(r0 + row) + d;
    dst[0] = from_f32<T>(x.x);
    dst[1] = from_f32<T>(x.y);
    dst[2] = from_f32<T>(x.z);
    dst[3] = from_f32<T>(x.w);
  };
  if (a.splits == 1) {
    for (int w = threadIdx.x; w < rows * (HDP / 4); w += RW * 32) {
      const int row = w / (HDP / 4), d = w % (HDP / 4) * 4;
      if (d < L.hd) store4(row, d, joined(row, d));
    }
    if (a.mass && threadIdx.x < rows) {
      const float2 x = split_w[threadIdx.x];
      a.row_ml[head * a.n * a.G + r0 + threadIdx.x] = row_weight(x.x, x.y, kPExp);
    }
    return;
  }
  if (Shape::send && cluster) {
    // the splits are a cluster: each CTA sends every other its share of the rows' columns and the
    // rows' (max, sum), so that one barrier is all that they wait for (each reading its share
    // from all took a remote read's latency twice and a barrier at the end more: 0.7 us)
    const int pieces = rows * (HDP / 4), share = (pieces + a.splits - 1) / a.splits;
    const uint32_t part_of = ((1u << 22) + share - 1) / share;   // (w / share for w < 8 share: the excess stays below 2^22)
    const uint32_t in = smem_u32(frag);
    cluster_wait_acquire();   // (everybody holds Q)
    for (int w = threadIdx.x; w < pieces; w += RW * 32) {
      const uint32_t to = (uint32_t)w * part_of >> 22;
      st_cluster_f4(mapa_shared(in + 16u * (uint32_t)(split * share + w - (int)to * share), to),
                    joined(w / (HDP / 4), w % (HDP / 4) * 4));
    }
    if ((int)threadIdx.x < 8 * a.splits)
      st_cluster_f2(mapa_shared(smem_u32(&split_in[split][threadIdx.x % 8]), threadIdx.x / 8), split_w[threadIdx.x % 8]);
    cluster_sync();
    if ((int)threadIdx.x < rows) {
      float M = -INFINITY, S = 0.f;
      for (int q = 0; q < a.splits; ++q) M = fmaxf(M, split_in[q][threadIdx.x].x);
      for (int q = 0; q < a.splits; ++q) {
        const float2 x = split_in[q][threadIdx.x];
        const float wt = x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y);
        split_wt[q][threadIdx.x] = wt;
        S += wt;
      }
      const float inv = !(S <= 0.f) ? 1.f / S : 0.f;
      for (int q = 0; q < a.splits; ++q) split_wt[q][threadIdx.x] *= inv;
      if (a.mass && split == 0) a.row_ml[head * a.n * a.G + r0 + threadIdx.x] = row_weight(M, S, kPExp);
    }
    __syncthreads();
    for (int w = split * share + threadIdx.x; w < min(pieces, (split + 1) * share); w += RW * 32) {
      const int row = w / (HDP / 4), d = w % (HDP / 4) * 4;
      if (d >= L.hd) continue;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int q = 0; q < a.splits; ++q) {
        const float4 x = lds_f4(in + 16u * (uint32_t)(q * share + w - split * share));
        const float wt = split_wt[q][row];
        acc.x += wt * x.x;
        acc.y += wt * x.y;
        acc.z += wt * x.z;
        acc.w += wt * x.w;
      }
      store4(row, d, acc);
    }
    return;
  }
  if (cluster) {
    // the splits are a cluster: each CTA joins a share of the rows' columns from all of them
    for (int w = threadIdx.x; w < rows * (HDP / 4); w += RW * 32) ((float4*)mine)[w] = joined(w / (HDP / 4), w % (HDP / 4) * 4);
    cluster_sync();
    if ((int)threadIdx.x < rows) {
      const uint32_t at = smem_u32(&split_w[threadIdx.x]);
      float2 x[8];   // (all on their way together)
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const uint32_t from = mapa_shared(at, (uint32_t)min(q, a.splits - 1));
        x[q] = make_float2(ld_cluster_f1(from), ld_cluster_f1(from + 4));
      }
      float M = -INFINITY, S = 0.f, wt[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) M = fmaxf(M, x[q].x);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        wt[q] = q >= a.splits ? 0.f : (x[q].y != x[q].y ? x[q].y : (x[q].x == -INFINITY ? 0.f : exp2f(x[q].x - M) * x[q].y));
        S += wt[q];
      }
      const float inv = !(S <= 0.f) ? 1.f / S : 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) split_wt[q][threadIdx.x] = wt[q] * inv;
      if (a.mass && split == 0) a.row_ml[head * a.n * a.G + r0 + threadIdx.x] = row_weight(M, S, kPExp);
    }
    __syncthreads();
    const int pieces = rows * (HDP / 4), share = (pieces + a.splits - 1) / a.splits;
    for (int w = split * share + threadIdx.x; w < min(pieces, (split + 1) * share); w += RW * 32) {
      const int row = w / (HDP / 4), d = w % (HDP / 4) * 4;
      if (d >= L.hd) continue;
      const uint32_t at = smem_u32(mine + row * HDP + d);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int q = 0; q < a.splits; ++q) {
        const float4 x = ld_cluster_f4(mapa_shared(at, (uint32_t)q));
        const float wt = split_wt[q][row];
        acc.x += wt * x.x;
        acc.y += wt * x.y;
        acc.z += wt * x.z;
        acc.w += wt * x.w;
      }
      store4(row, d, acc);
    }
    cluster_sync();   // nobody leaves while its rows are read
    return;
  }
  const size_t unit = here * a.row_tiles + tile;
  float* part = a.part + (unit * a.splits + split) * 16 * HDP;
  for (int w = threadIdx.x; w < rows * (HDP / 4); w += RW * 32) __stcg((float4*)part + w, joined(w / (HDP / 4), w % (HDP / 4) * 4));
  if (threadIdx.x < rows) __stcg(a.part_ml + (unit * a.splits + split) * 16 + threadIdx.x, split_w[threadIdx.x]);
  // the last split to arrive joins them all, in their order
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicInc(a.arrived + unit, (unsigned)a.splits - 1u) == (unsigned)a.splits - 1u;
  __syncthreads();
  if (!last) return;
  __threadfence();
  // the splits' (max, sum), all on their way together, then their weights in their place
  float2* wts = (float2*)joint;   // [splits][16]
  for (int w = threadIdx.x; w < a.splits * 16; w += RW * 32)
    if (w % 16 < rows) wts[w] = ld_l2(a.part_ml + unit * a.splits * 16 + w);
  __syncthreads();
  if ((int)threadIdx.x < rows) {
    const int row = threadIdx.x;
    float M = -INFINITY, S = 0.f;
    for (int q = 0; q < a.splits; ++q) M = fmaxf(M, wts[q * 16 + row].x);
    for (int q = 0; q < a.splits; ++q) {
      const float2 x = wts[q * 16 + row];
      const float wt = x.y != x.y ? x.y : (x.x == -INFINITY ? 0.f : exp2f(x.x - M) * x.y);
      wts[q * 16 + row].x = wt;
      S += wt;
    }
    const float inv = !(S <= 0.f) ? 1.f / S : 0.f;
    for (int q = 0; q < a.splits; ++q) wts[q * 16 + row].x *= inv;
    if (a.mass) a.row_ml[head * a.n * a.G + r0 + row] = row_weight(M, S, kPExp);
  }
  __syncthreads();
  const float* p0 = a.part + unit * a.splits * 16 * HDP;
  for (int w = threadIdx.x; w < rows * (HDP / 4); w += RW * 32) {
    const int row = w / (HDP / 4), d = w % (HDP / 4) * 4;
    if (d >= L.hd) continue;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int q = 0; q < a.splits; ++q) {
      const float4 x = ld_l2((const float4*)(p0 + ((size_t)q * 16 + row) * HDP + d));
      const float wt = wts[q * 16 + row].x;   // (0 times an empty split's zeros)
      acc.x += wt * x.x;
      acc.y += wt * x.y;
      acc.z += wt * x.z;
      acc.w += wt * x.w;
    }
    store4(row, d, acc);
  }
}

// Attention mass: token j's softmax weights summed over the rows of its KV head, from the
// scores that the attention kept and the rows' (max, 1 / sum): a thread per two tokens
// and, of many queries, every 8th, 16th or 64th of them, summed in a fixed order.  Bound by
// reading them, 4 bytes per row and token, on the way of few loads per thread (4 robots x 16
// rows x 131071 tokens: 34 MB, in L2, 17 us behind the attention, 18.7 alone); computing them
// again would read the keys' 134 MB from HBM.
__global__ void __launch_bounds__(1024) cache_mass_scores_kernel(CacheAttnArgs a, int groups) {
  __shared__ float2 sums[1024];
  const int per = (int)blockDim.x / groups, group = threadIdx.x / per, at = threadIdx.x % per;
  const int j = (blockIdx.x * per + at) * 2;
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.z + a.b0;
  const size_t head = (size_t)b * a.c.Hkv + blockIdx.y, here = (size_t)blockIdx.z * a.c.Hkv + blockIdx.y;
  Sight s;
  robot_sight(a, b, s);
  const float2* ml = a.row_ml + head * a.n * a.G;
  const float* sc = a.scores + here * (a.i1 - a.i0) * a.G * a.mass_pitch + j;
  float v0 = 0.f, v1 = 0.f;
  if (j < s.len)
    for (int i = a.i0 + group; i < min(a.i1, s.count); i += groups) {
      const RowMask mk = row_mask(a, s, i * a.G);
      const bool s0 = mk.sees(j), s1 = mk.sees(j + 1);
      if (!s0 && !s1) continue;
#pragma unroll 4
      for (int g = 0; g < a.G; ++g) {
        const float2 x = ld_once((const float2*)(sc + (size_t)((i - a.i0) * a.G + g) * a.mass_pitch)), y = ld_kept(ml + i * a.G + g);
        v0 += s0 ? exp2f(x.x - y.x) * y.y : 0.f;
        v1 += s1 ? exp2f(x.y - y.x) * y.y : 0.f;
      }
    }
  if (groups > 1) {
    sums[threadIdx.x] = make_float2(v0, v1);
    __syncthreads();
    if (group) return;
    for (int q = 1; q < groups; ++q) {
      v0 += sums[q * per + at].x;
      v1 += sums[q * per + at].y;
    }
  }
  float* mass = a.mass + head * a.mass_stride + j;
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (j + e < a.max_length) {
      const float v = e ? v1 : v0;
      if (!a.mass_add) mass[e] = v;
      else if (j + e < s.len) mass[e] += v;
    }
}

// One launch of the rows kernel, queries i0 .. i1 - 1 of `batch` robots from b0 on, and, where
// the mass is wanted, one over the scores that it left.
template <int HDP, int NP, typename T>
cudaError_t launch_part(CacheAttnArgs a, int batch, cudaStream_t st) {
  constexpr int U = Unit<HDP>::U;
  const int rows = (a.i1 - a.i0) * a.G, RT = rows <= 8 ? 8 : 16;   // rows of a tile
  a.row_tiles = (rows + RT - 1) / RT;
  const long long tiles = (long long)a.row_tiles * a.c.Hkv * batch;
  // tokens that a row tile sees at most, in units
  long long seen = a.max_length;
  if (a.window > 0) seen = min(seen, (long long)a.window + a.sinks + 15 / a.G + 1 + 2 * U);
  const int units = (int)((seen + U - 1) / U);
  a.splits = 1;
  if (tiles < 2 * a.num_sms) {
    // two CTAs per SM, each warp with a unit at least
    // (and no more splits than the joining CTA has weights for in shared memory)
    const long long most = min(min((long long)kCacheSplitCtas, 2ll * a.num_sms) / tiles, (long long)RW * HDP / 2);
    a.splits = (int)max(1ll, min(most, (long long)(units + RW - 1) / RW));
    // up to 8 splits join in distributed shared memory, more through L2, which takes longer
    // than two units more for each warp
    if (a.splits > 8 && units <= 8 * RW * 3) a.splits = 8;
  }
  const RowsMaps maps{a.maps->k_rows, a.maps->v_rows};
  const dim3 grid(a.row_tiles * a.splits, a.c.Hkv, batch), cluster(a.splits <= 8 ? a.splits : 1, 1, 1);
  const cudaError_t e =
      RT == 8 ? launch_kernel_cluster(cache_rows_kernel<HDP, NP, 8, T>, grid, dim3(RW * 32), RowsShape<HDP, NP, 8>::bytes, st,
                                      cluster, maps, a)
              : launch_kernel_cluster(cache_rows_kernel<HDP, NP, 16, T>, grid, dim3(RW * 32), RowsShape<HDP, NP, 16>::bytes, st,
                                      cluster, maps, a);
  if (e != cudaSuccess || !a.scores) return e;
  // groups of a token's queries, and with them threads: as many as the queries fill, 1024 where
  // the tokens are few CTAs otherwise.  Measured, us with 1 / 8 / 16 / 64 groups: 1 robot of 816
  // tokens (8 heads on one), 16 queries 29 / 6.0 / 4.0 / 5.0, 64: 111 / 18 / 11 / 5.3, 512: 871 /
  // 118 / 66 / 22; 26 robots of 1465 (6 heads on each of 2), 16: 35 / 14 / 20 / 58, 64: 243 / 50 /
  // 57 / 78, 128: 900 / 184 / 158 / 160, 512: 19674 / 3132 / 1869 / 879.  (Below 16 queries 8 groups
  // would be the faster ones from four on: 8 of 1 robot 15.4 / 3.7, of 26 robots 19 / 9; at 64 of
  // many robots 8 or 16.)
  const int queries = a.i1 - a.i0;
  const bool few = (long long)((a.max_length + 63) / 64) * a.c.Hkv * batch < 2 * a.num_sms;
  const int groups = queries >= 64 ? 64 : (queries < 16 ? 1 : (few ? 16 : 8)), threads = groups >= 16 ? 1024 : 256;
  const int tokens = 2 * threads / groups;
  return launch_kernel(cache_mass_scores_kernel, dim3((a.max_length + tokens - 1) / tokens, a.c.Hkv, batch), dim3(threads), 0, st, 1,
                       a, groups);
}

template <int HDP, int NP, typename T>
cudaError_t launch_rows(CacheAttnArgs a, cudaStream_t st) {
  const Overlap overlap;
  const bool mass = a.mass && a.max_length > 0;
  // From 17 rows per KV head on, bf16 goes to the tensor cores' kernel.  Measured without the mass,
  // us here / there: 8 heads of 256 on one, 64 robots of 816 tokens, 16 rows 14.7 / 15.7, 24 rows
  // 19.0 / 16.4, 64 rows 24.6 / 17.2; 16 robots, 16 rows 11.5 / 13.0, 64 rows 14.6 / 15.2, 128 rows
  // 19.0 / 18.3; 16 heads of 64 on 4, 64 robots, 16 rows 10.1 / 21.8, 32 rows 19.4 / 21.8, 64 rows
  // 37.6 / 21.9.  (The line fits many robots; of one, whose rows fill few CTAs, this kernel is the
  // faster one up to 128 rows: 10.3 / 20.8 over 816 tokens, 42 / 216 over 8192.)
  if (NP == 1 && a.n * a.G > 16) {
    const cudaError_t e = launch_cache_attend_tc(a, st);
    return e != cudaSuccess || !mass ? e : launch_cache_mass_tc(a, st);
  }
  // For the mass every row's scores are kept, of as many robots (or, of one robot, queries) at
  // a time as the workspace holds: a query of one robot at least.  (Computing them again, from
  // keys in registers with Q laid out in every CTA, took with the attention 879 us instead of 82
  // for one robot's 816 queries and tokens, 8 heads of 256 on one in fp32, and 619 instead of
  // 248 for 4 robots' 1024, 16 heads of 64 on 4.)
  a.mass_pitch = (a.max_length + 127) / 128 * 128;
  a.scores = mass ? a.mass_ws : nullptr;
  int robots = a.batch, queries = a.n;
  if (mass) {
    const size_t query = (size_t)a.c.Hkv * a.G * a.mass_pitch * 4, fit = a.mass_ws_bytes / query;
    if (fit == 0) return cudaErrorInvalidValue;
    robots = (int)std::min<size_t>(a.batch, std::max<size_t>(1, fit / a.n));
    if (robots == 1) queries = (int)std::min<size_t>(a.n, fit >= 16 ? fit / 16 * 16 : fit);
  }
  for (a.b0 = 0; a.b0 < a.batch; a.b0 += robots) {
    CacheAttnArgs part = a;
    for (part.i0 = 0; part.i0 < a.n; part.i0 = part.i1) {
      part.i1 = min(a.n, part.i0 + queries);
      part.mass_add = a.mass_add || part.i0 > 0;
      const cudaError_t e = launch_part<HDP, NP, T>(part, min(robots, a.batch - a.b0), st);
      if (e != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

template <int HDP>
cudaError_t launch_hd(const CacheAttnArgs& a, Dtype dt, cudaStream_t st) {
  return dt == DT_BF16 ? launch_rows<HDP, 1, bf16>(a, st) : launch_rows<HDP, 2, float>(a, st);
}

template <int HDP, int NP, int RT, typename T>
cudaError_t init_rows() {
  return cudaFuncSetAttribute(cache_rows_kernel<HDP, NP, RT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              RowsShape<HDP, NP, RT>::bytes);
}

template <int HDP>
cudaError_t init_hd() {
  cudaError_t e = init_rows<HDP, 1, 8, bf16>();
  if (e == cudaSuccess) e = init_rows<HDP, 1, 16, bf16>();
  if (e == cudaSuccess) e = init_rows<HDP, 2, 8, float>();
  if (e == cudaSuccess) e = init_rows<HDP, 2, 16, float>();
  return e;
}

}  // namespace

cudaError_t launch_cache_attend(const CacheAttnArgs& a, Dtype dt, cudaStream_t st) {
  switch (a.c.hdp) {
    case 64: return launch_hd<64>(a, dt, st);
    case 128: return launch_hd<128>(a, dt, st);
    case 192: return launch_hd<192>(a, dt, st);
    default: return launch_hd<256>(a, dt, st);
  }
}

// The maps of a layer for every robot of the cache: boxes of the kernels' tiles.
cudaError_t encode_layer(CacheMaps* m, const CacheLayer& c, int batch) {
  const int unit = c.hdp == 64 ? 64 : (c.hdp == 128 ? 32 : 16), in = c.hdp % 128 ? 64 : 128;
  cudaError_t e = cache_tc_encoder();
  if (e == cudaSuccess) e = encode_codes(&m->k_tc, c.k, c, batch, 64, BT, true);
  if (e == cudaSuccess) e = encode_codes(&m->v_tc, c.v, c, batch, 64, 64, false);
  if (e == cudaSuccess) e = encode_codes(&m->k_rows, c.k, c, batch, in, unit, true);
  if (e == cudaSuccess) e = encode_codes(&m->v_rows, c.v, c, batch, in, unit, true);
  return e;
}

cudaError_t init_cache_kernels() {
  cudaError_t e = init_hd<64>();
  if (e == cudaSuccess) e = init_hd<128>();
  if (e == cudaSuccess) e = init_hd<192>();
  if (e == cudaSuccess) e = init_hd<256>();
  return e;
}

}  // namespace ravel
