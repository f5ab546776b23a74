// Drawing a token from a row of logits: top-k, top-p, min-p and the draw itself, without a sort.
//
// Weights are whole numbers, 2^43 exp((x - max) / T) rounded, so that their sums are exact and
// the same in any order; a row is at most 2^20 long, its sum below 2^64.  The order of the tokens (by
// logit, equal ones by index) is not made: a limit is a border in it, a key and how many of the
// tokens with that key stay; as one number, (key, ~index) of the last token that stays.
//
// A cluster of CTAs per row.  The row's maximum first; then a histogram of 512 bins between the
// maximum and the least logit that has a weight, of counts or, where top-p alone limits, of weights too (of each warp's
// run of the row): the bin that holds the border.  Where the tokens up to that bin are at most 2048, they are brought
// together in one CTA, which does the rest by itself.  Where they are more, the bin's own tokens are, which gives
// the border, and the weights before it are summed by warps' runs; the run that holds the
// token is gone through again.  Where even the bin holds more (thousands of nearly equal logits), a
// radix selection over the keys' four bytes finds the border.
//
// Measured (replays from a graph): one row of 65536 bf16 logits under top-k 40, top-p and min-p 13 us, a chain of four
// barriers of the cluster (1000 cycles each) and what lies between, a thousand here and there; 24 rows of 32003 under
// settings of their own 27; 64 rows of 128001 fp32 logits under top-p 0.9 53 us, of which the histogram takes 26 (80
// instructions a logit, 50 of them its weight, and three atomics), the list 7, the first
// pass 3 (66 with the weights before the border computed once more, and rows that begin between 16 bytes read value by
// value); the same without limits 29, with top-k 50 24, with top-k 3000 and top-p 68, all logits equal 459.  Weights two
// at a time in packed operations, and 64-bit atomics, are no faster.
//
// A list by all threads / by histograms / sorted, one row of 65536 under top-p 0.95 and top-k 40: 11.7 / 16.7 / 15.0 us;
// 100: 13.2 / 17.4 / 15.4; 200: 17.2 / 17.9 / 17.1; 256: 18.3 / 18.1 / 21.3; 1000: - / 22.3 / 30.2; 2000: - / 26.6 / 32.7.  A
// list of up to 256 sorted by counting, else exchanges: the same row under top-p 0.9, whose border's bin is sorted, 23.2 /
// 27.4.
#include <algorithm>

#include "common.cuh"
#include "decode.h"
#include "launch.h"
#include "tc_common.cuh"

namespace ravel {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kBins = 512, kCap = 2048;
constexpr int kRanks = 8;        // CTAs of a row at most
constexpr int kBits = 43;        // weight of the likeliest token: 2^43
constexpr int kWarpBins = 2 * kWarps * kBins * 4;   // bytes of the weights of warps' runs by bin

typedef unsigned long long u64;

// 2^(j / 1024) = h 2^-30 (1 + d): h, a whole number, and d in units of 2^-42, as a float's bits
struct ExpTable {
  uint2 v[1024];
  constexpr ExpTable() : v() {
    for (int j = 0; j < 1024; ++j) {
      const double x = 0.6931471805599453094 * j / 1024.0;
      double term = 1.0, sum = 1.0;
      for (int i = 1; i < 22; ++i) {
        term *= x / i;
        sum += term;
      }
      const double h = sum * 1073741824.0;
      v[j].x = (uint32_t)(h + 0.5);
      v[j].y = __builtin_bit_cast(uint32_t, (float)((h / v[j].x - 1.0) * 4398046511104.0));
    }
  }
};
__device__ constexpr ExpTable kExp{};

// Ascending as unsigned integers; -0 = +0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// exp((x - top) / T) as a whole number.  In the log2 domain y = (x - top) * c with c = log2(e) / T
// in two floats, and the difference and its product with their rounding errors: yh + ye.  With q
// the nearest whole number to 1024 yh, 2^y = 2^(q / 1024) 2^f, the first factor from a table, 2^f = 1 + r
// from its series, r below 2^-11, whose first term is a product in two floats.  Some 2^-42 of the
// weight off: r's two roundings, and the product of r with the table's own remainder, which is left out.  (In fp32 a
// weight is 2^-22 off and its error grows with x: at 100000 tokens one border in a hundred falls elsewhere than in
// 64 bits.)
// Logits are halved, so that no difference overflows, and where T is above 2^64 taken by 2^-65 (as T by 2^-64), or
// c's second float, from 10^32 on, and its first, from 2 10^38 on, would lack bits.
struct Weigher {
  float scale, top, ch, cl;   // of the logits; the largest one's share of it; twice log2(e) / T
  // (in two floats: 64-bit ones come two to a clock)
  __device__ __forceinline__ Weigher(float max, float temperature) {
    const float c = 2.88539004f, less = 3.851925982e-08f;   // 2 log2(e) = c + less
    scale = temperature > 0x1p64f ? 0x1p-65f : 0.5f;
    temperature *= 2.f * scale;
    top = scale * max;
    ch = __fdiv_rn(c, temperature);
    cl = __fdiv_rn(__fmaf_rn(-ch, temperature, c) + less, temperature);
  }
  __device__ __forceinline__ u64 operator()(float logit, const uint2* table) const {
    const float x = scale * logit;
    const float dh = x - top;
    const float v = dh - x, dl = (x - (dh - v)) - (top + v);
    const float yh = dh * ch;
    if (!(yh > -44.f)) return 0ull;
    const float ye = __fmaf_rn(dh, ch, -yh) + __fmaf_rn(dh, cl, dl * ch);
    const float shifted = __fmaf_rn(yh, 1024.f, 12582912.f);   // 1.5 * 2^23: q in the low bits
    const int q = __float_as_int(shifted) - 0x4b400000;
    const uint2 t = table[__float_as_int(shifted) & 1023];
    const float rest = __fmaf_rn(shifted - 12582912.f, -0x1p-10f, yh);   // exact, up to 2^-11
    // r in units of 2^-42: ln 2 rest as a float and what it lacks, the small terms with the latter
    const float rh = rest * 0.693147182f;
    const float f = (rest + ye) * 0.693147182f;
    const float rl = __fmaf_rn(rest, 0.693147182f, -rh) + __fmaf_rn(rest, -1.90465421e-9f, ye * 0.693147182f) +
                     f * f * __fmaf_rn(f, 0.166666667f, 0.5f);
    const int r = __float2int_rn(rh * 0x1p42f) + __float2int_rn(__fmaf_rn(rl, 0x1p42f, __uint_as_float(t.y)));
    // h (1 + r 2^-42), in units of 2^-52, and rounded to 2^-43
    const long long v52 = (long long)(int)t.x * (1 << 22) + ((long long)(int)t.x * r >> 20);
    return (((u64)v52 >> (51 - kBits - (q >> 10))) + 1ull) >> 1;
  }
};

// ln(p) for 0 < p < 1 in two floats, off by some 2^-43: ln of p's mantissa m from logf, corrected by what
// m lacks of exp of that, and its exponent.
__device__ __forceinline__ float2 log_of(float p, const uint2* table) {
  int e;
  const float m = frexpf(p, &e);   // 1/2 <= m < 1
  const float y = logf(m);
  const Weigher weigh(0.f, 1.f);
  const u64 w = weigh(y, table);
  const float more = (float)((long long)(u64)(m * 0x1p24f) * (1ll << (kBits - 24)) - (long long)w) / (float)w;
  const float a = (float)e * 0.693147182f, al = __fmaf_rn((float)e, 0.693147182f, -a) + (float)e * -1.90465421e-9f;
  const float h = a + y, v = h - a, hl = (a - (h - v)) + (y - v);
  return make_float2(h, hl + al + more);
}

// floor(f * s), or the next whole number at or above, for a finite f >= 0
__device__ __noinline__ u64 times_fraction(u64 s, float f, bool up) {
  const uint32_t bits = __float_as_uint(f), e = bits >> 23;
  const u64 mant = e ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
  const int shift = 150 - (int)(e ? e : 1u);   // f = mant * 2^-shift
  const u64 hi = __umul64hi(s, mant), lo = s * mant;
  u64 whole, rest;
  if (shift >= 128) {
    whole = 0;
    rest = hi | lo;
  } else if (shift >= 64) {
    whole = shift == 64 ? hi : hi >> (shift - 64);
    rest = lo | (shift == 64 ? 0ull : hi << (128 - shift));
  } else {
    whole = hi << (64 - shift) | lo >> shift;   // (f < 1: shift is at least 24)
    rest = lo << (64 - shift);
  }
  return whole + (up && rest ? 1ull : 0ull);
}

__device__ __forceinline__ u64 ld_cluster_u64(uint32_t a) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ u64 warp_max_u64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const u64 x = __shfl_xor_sync(0xffffffffu, v, o);
    v = x > v ? x : v;
  }
  return v;
}
__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

struct DrawShared {
  uint2 table[1024];
  union {
    struct {
      uint32_t bins[kBins];     // of a CTA: counts
      u64 weights[kBins];       // and weights
    };
    u64 hist[2][256];           // radix selection
    struct {
      u64 hist[kBins];          // selection within the list
      u64 few[256];
    } pick;
  };
  u64 list[kCap];               // (key, ~index)
  union {
    u64 sorted[kCap];           // the same, from the largest down
    u64 few_weights[256];
    ulonglong2 pairs[256];      // values and weights
    float keep[kWarps][64];     // a warp's logits that wait for their weights
  };
  u64 slot[2][2];               // what this CTA gives to a reduction
  u64 warp_a[kWarps], runs[kWarps];
  u64 sel, sel_before, sel_in;
  uint32_t sel_bin, few_n, listed, counts[kRanks], found_run;
};

// What is not in a loop over the row is called, not inlined (the times are the same).

// Sum of x over the threads before this one, and over the CTA.
__device__ __noinline__ ulonglong2 scan_block(DrawShared& s, u64 x) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 upto = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 up = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += up;
  }
  __syncthreads();
  if (lane == 31) s.warp_a[warp] = upto;
  __syncthreads();
  const u64 w = s.warp_a[lane];
  u64 ws = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 up = __shfl_up_sync(0xffffffffu, ws, o);
    if (lane >= o) ws += up;
  }
  return make_ulonglong2(__shfl_sync(0xffffffffu, ws - w, warp) + upto - x, __shfl_sync(0xffffffffu, ws, 31));
}

__device__ __noinline__ u64 weight_of(const Weigher& weigh, u64 order, const uint2* table) {
  return weigh(value_of((uint32_t)(order >> 32)), table);
}

// Of values c with weights w, two to a thread, that at which the weights, summed from the largest down in the order
// of c (or, by_index, of their index), reach `target`: a histogram by bins (of kBins, monotone), then the values of the
// bin that holds it, each with the sum of those before it.  0: the bin has more than 256 of them.
__device__ __noinline__ u64 pick(DrawShared& s, ulonglong2 c, ulonglong2 w, u64 target, int bin0, int bin1, bool by_index) {
  const int tid = threadIdx.x;
  if (tid < kBins) s.pick.hist[tid] = 0ull;
  if (tid == 0) s.few_n = 0u;
  __syncthreads();
  if (w.x) atomicAdd(&s.pick.hist[bin0], w.x);
  if (w.y) atomicAdd(&s.pick.hist[bin1], w.y);
  __syncthreads();
  const u64 in = tid < kBins ? s.pick.hist[tid] : 0ull, cum = scan_block(s, in).x;
  if (cum < target && cum + in >= target) s.sel_bin = tid, s.sel_before = cum;
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i < 2; ++i)
    if ((i ? w.y : w.x) && (i ? bin1 : bin0) == (int)s.sel_bin) {
      const uint32_t at = atomicAdd(&s.few_n, 1u);
      if (at < 256u) s.pick.few[at] = i ? c.y : c.x, s.few_weights[at] = i ? w.y : w.x;
    }
  __syncthreads();
  const int few = (int)s.few_n;
  if (few > 256) return 0ull;
  if (tid < few) {
    const u64 mine = s.pick.few[tid], order = by_index ? mine << 32 : mine;
    u64 before = s.sel_before;
    for (int j = 0; j < few; ++j) {
      const u64 other = s.pick.few[j];
      before += (by_index ? other << 32 : other) > order ? s.few_weights[j] : 0ull;
    }
    if (before < target && before + s.few_weights[tid] >= target) s.sel = mine;
  }
  __syncthreads();
  return s.sel;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) draw_kernel(DrawArgs a) {
  __shared__ DrawShared s;
  extern __shared__ uint4 draw_smem[];
  uint32_t* warp_bins = (uint32_t*)draw_smem;   // weights of a warp's run by bin: [low, high word][warp][bin]
  constexpr int V = 16 / sizeof(T);
  constexpr uint32_t kAll = 0xffffffffu;
  const int ranks = (int)gridDim.x, rank = ranks > 1 ? (int)cluster_ctarank() : 0, b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float inf = __uint_as_float(0x7f800000u);
  s.table[tid] = kExp.v[tid];
  auto clear_warp_bins = [&] {
    for (int i = tid; i < 2 * kWarps * kBins / 4; i += kThreads) draw_smem[i] = make_uint4(0u, 0u, 0u, 0u);
  };
  if (a.top_p) clear_warp_bins();
  if (tid < kBins) s.bins[tid] = 0u;
  if (tid == 0) s.listed = 0u;
  pdl_trigger();
  pdl_wait();
  const float u = a.u[b], t = a.temperature ? a.temperature[b] : 1.f, p = a.top_p ? a.top_p[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  int k = a.top_k ? a.top_k[b] : 0;
  const T* row = (const T*)a.logits + (long long)b * a.row;
  // this warp's run of the row: whole steps of 32 lanes x V values, from the 16 bytes on in which the row begins
  const int shift = (int)((uintptr_t)row % 16 / sizeof(T)), past = shift + a.vocab;
  const T* from16 = row - shift;
  const int steps_all = (past + 32 * V - 1) / (32 * V), shares = ranks * kWarps, share = rank * kWarps + warp;
  auto first_step = [&](int share) { return (int)((long long)steps_all * share / shares); };
  const int step0 = first_step(share), step1 = first_step(share + 1);

  auto fetch = [&](int step) {   // V values; before the row and past it -inf
    const int i = (step * 32 + lane) * V;
    if (i >= shift && i + V <= past) return *(const uint4*)(from16 + i);
    T t[V];
#pragma unroll
    for (int j = 0; j < V; ++j) t[j] = i + j >= shift && i + j < past ? from16[i + j] : from_f32<T>(-inf);
    uint4 w;
    memcpy(&w, t, 16);
    return w;
  };
  auto widen = [&](const uint4& w, float* x) {
    T t[V];
    memcpy(t, &w, 16);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = to_f32(t[j]);
  };
  auto load = [&](int step, float* x) { widen(fetch(step), x); };
  // f(step, values) for the steps of this warp's run, a step's values on their way while the one before is worked on
  auto for_steps = [&](auto f) {
    if (step0 >= step1) return;
    uint4 next = fetch(step0);
#pragma unroll 1
    for (int step = step0; step < step1; ++step) {
      float x[V];
      widen(next, x);
      if (step + 1 < step1) next = fetch(step + 1);
      f(step, x);
    }
  };
  auto index_of = [&](int step, int j) { return (step * 32 + lane) * V + j - shift; };
  auto there = [&](int i) { return (uint32_t)i < (uint32_t)a.vocab; };
  auto order_of = [&](float x, int i) { return (u64)key_of(x) << 32 | (kAll - (uint32_t)i); };
  int turn = 0;
  auto barrier = [&] {
    if (ranks > 1) cluster_sync();
    else __syncthreads();
  };
  // sum of a word of all ranks (the loads on their way together)
  auto sum_of = [&](const auto* p) {
    if (ranks == 1) return (u64)*p;
    u64 x[kRanks], n = 0;
#pragma unroll
    for (int i = 0; i < kRanks; ++i) {
      const uint32_t at = mapa_shared(smem_u32(p), (uint32_t)min(i, ranks - 1));
      x[i] = sizeof(*p) == 8 ? ld_cluster_u64(at) : ld_cluster_u32(at);
    }
#pragma unroll
    for (int i = 0; i < kRanks; ++i) n += i < ranks ? x[i] : 0u;
    return n;
  };
  auto from_rank = [&](const u64* p, int i) { return ranks > 1 ? ld_cluster_u64(mapa_shared(smem_u32(p), (uint32_t)i)) : *p; };
  // maxima of x and of y over the row's threads, for every thread
  auto reduce_max = [&](u64& x, u64& y) {
    x = warp_max_u64(x);
    y = warp_max_u64(y);
    if (lane == 0) s.warp_a[warp] = x, s.runs[warp] = y;
    __syncthreads();
    if (warp == 0) {
      x = warp_max_u64(s.warp_a[lane]);
      y = warp_max_u64(s.runs[lane]);
      if (lane == 0) s.slot[turn][0] = x, s.slot[turn][1] = y;
    }
    barrier();
    // lane i takes rank i's
    x = warp_max_u64(lane < ranks ? from_rank(&s.slot[turn][0], lane) : 0ull);
    y = warp_max_u64(lane < ranks ? from_rank(&s.slot[turn][1], lane) : 0ull);
    turn ^= 1;
  };
  // sum of x over the threads before this one and, in all, over the CTA
  auto block_scan = [&](u64 x, u64& all) {
    const ulonglong2 r = scan_block(s, x);
    all = r.y;
    return r.x;
  };

  // the largest logit, the least finite one, and what is no number: +inf and NaN are the largest as signed words, or, with
  // the sign set, the largest as unsigned ones
  float most = -inf, least = inf;
  int words = 0;
  uint32_t uwords = 0u;
#pragma unroll 4
  for (int step = step0; step < step1; ++step) {
    float x[V];
    load(step, x);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      most = fmaxf(most, x[j]);
      least = fminf(least, x[j] == -inf ? inf : x[j]);
      words = max(words, __float_as_int(x[j]));
      uwords = max(uwords, __float_as_uint(x[j]));
    }
  }
  u64 best = key_of(most), low = words >= 0x7f800000 || uwords > 0xff800000u ? 1ull << 32 : (u64)~key_of(least);
  reduce_max(best, low);
  const float top = value_of((uint32_t)best);
  const Weigher weigh(top, t);
  // log of the share of a token of logit x: x's part in the log2 domain and the sum's, in two floats
  auto answer = [&](int token, float x, u64 total) {
    a.tokens[b] = token;
    if (!a.log_probs) return;
    const float d = weigh.scale * x - weigh.top, yh = d * weigh.ch, yl = __fmaf_rn(d, weigh.ch, -yh) + d * weigh.cl;
    const int e = 63 - __clzll((long long)total);
    const float m = (float)total * exp2f((float)-e);   // total = m 2^e
    const float h = yh - (float)(e - kBits), v = h - yh, l = (yh - (h - v)) + (-(float)(e - kBits) - v) + yl;
    a.log_probs[b] = __fmaf_rn(h, 0.693147182f, __fmaf_rn(l, 0.693147182f, h * -1.90465421e-9f) - logf(m));
  };
  const bool none = low >> 32 || !(top > -inf) || !(u >= 0.f && u < 1.f) || !(t < inf) || p != p || mp != mp;
  if (none || t < 0x1p-20f) {
    // (the first of the largest)
    u64 first = 0ull, ignored = 0ull;
    if (!none)
      for (int step = step0; step < step1; ++step) {
        float x[V];
        load(step, x);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (x[j] == top) first = max(first, (u64)(kAll - (uint32_t)index_of(step, j)));
      }
    reduce_max(first, ignored);
    if (rank == 0 && tid == 0) {
      a.tokens[b] = none ? -1 : (int)(kAll - (uint32_t)first);
      if (a.log_probs) a.log_probs[b] = none ? -inf : 0.f;
    }
    barrier();   // (nobody leaves while its slot is read)
    return;
  }
  // the last of the order that min-p lets through: key of the least logit that is not below
  // top + T ln(min_p), any index
  u64 last = 0ull;
  if (mp > 0.f) {
    float limit = top;
    if (mp < 1.f) {
      // (logits and T by a power of two, as Weigher takes them: T ln(min_p) may be beyond fp32 where the limit is not)
      const float2 l = log_of(mp, s.table);
      const float by = 2.f * weigh.scale, tt = by * t, most = by * top;
      const float h = tt * l.x, hl = __fmaf_rn(tt, l.x, -h) + tt * l.y;
      limit = most + h;
      const float v = limit - most, rest = (most - (limit - v)) + (h - v) + hl;
      if (rest > 0.f) limit = nextafterf(limit, inf);
      limit = fminf(limit * (by < 1.f ? 0x1p64f : 1.f), top);
    }
    last = (u64)key_of(limit) << 32;
  }

  // Bins of the order: equal parts of the log2 domain from the maximum down to the least logit or
  // to 2^-44, where weights end.  Every step of the formula is monotone in x, rounding included.
  const float d_least = weigh.scale * value_of(~(uint32_t)low) - weigh.top, y_least = fmaxf(d_least * weigh.ch, -44.f);
  const float to_place = -weigh.ch * ((float)(kBins - 1) / fmaxf(-y_least, 0x1p-40f));
  // place in bins, for bin i from i up to below i + 1 (the last but one: from there on)
  auto place_of = [&](float x) { return (weigh.scale * x - weigh.top) * to_place; };
  auto weighs = [&](float x) { return (weigh.scale * x - weigh.top) * weigh.ch > -44.f; };
  auto bin_of = [&](float x) { return min((int)place_of(x), kBins - 2); };
  // The bin at which the counts or the weights, summed from the first on, reach `target`, what comes
  // before it and what is in it; target > all: the last one.  For every thread of the row.
  auto bin_at = [&](u64 n, u64 target, u64 cum, u64 all, uint32_t& bin, u64& before, u64& in) {
    if (tid == 0) s.sel_bin = kBins - 1, s.sel_before = all, s.sel_in = 0;
    __syncthreads();
    if (tid < kBins && cum < target && cum + n >= target) s.sel_bin = tid, s.sel_before = cum, s.sel_in = n;
    __syncthreads();
    bin = s.sel_bin, before = s.sel_before, in = s.sel_in;
  };
  // The lists of the ranks one behind the other in rank 0; their number there.
  auto bring_together = [&] {
    barrier();
    int own = (int)min(s.listed, (uint32_t)kCap), total = own;   // (the counts said that all fit)
    if (rank == 0 && ranks > 1) {
      if (tid < ranks) s.counts[tid] = ld_cluster_u32(mapa_shared(smem_u32(&s.listed), (uint32_t)tid));
      __syncthreads();
      for (int r = 1; r < ranks; ++r) total += (int)s.counts[r];
      total = min(total, kCap);
      for (int flat = own + tid; flat < total; flat += kThreads) {
        int i = flat - own, r = 1;
        while (i >= (int)s.counts[r]) i -= (int)s.counts[r++];
        s.list[flat] = from_rank(&s.list[i], r);
      }
      __syncthreads();
    }
    return total;
  };
  // of a step's V values per lane those whose bit is set in `in`, behind those that are listed
  auto list_up = [&](uint32_t in, const float* x, int step) {
    if (!__any_sync(kAll, in != 0u)) return;
    uint32_t upto = __popc(in);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(kAll, upto, o);
      if (lane >= o) upto += up;
    }
    uint32_t at = 0;
    if (lane == 31) at = atomicAdd(&s.listed, upto);
    at = __shfl_sync(kAll, at, 31) + upto - __popc(in);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (in >> j & 1u) {
        if (at < (uint32_t)kCap) s.list[at] = order_of(x[j], index_of(step, j));
        ++at;
      }
  };
  // s.sorted: the n values of s.list from the largest down, zeros behind.  Few: each value's place is the number of
  // larger ones, counted by four threads.  Many: a bitonic network, two values to a thread, that exchanges within a
  // warp by shuffles and beyond through s.sorted.
  auto sort = [&](int n) {
    if (n <= 256) {
      for (int i = n + tid; i < kCap; i += kThreads) s.sorted[i] = 0ull;
      const int i = tid / 4, part = tid % 4;
      const u64 x = i < n ? s.list[i] : 0ull;
      uint32_t larger = 0;
      if (i - lane / 4 < n)   // (whole warps)
        for (int j = part; j < n; j += 4) larger += s.list[j] > x;
      larger += __shfl_xor_sync(kAll, larger, 1);
      larger += __shfl_xor_sync(kAll, larger, 2);
      if (part == 0 && i < n) s.sorted[larger] = x;
      __syncthreads();
      return;
    }
    int size = 512;
    while (size < n) size *= 2;
    u64 x = 2 * tid < n ? s.list[2 * tid] : 0ull, y = 2 * tid + 1 < n ? s.list[2 * tid + 1] : 0ull;
    for (int run = 2; run <= size; run *= 2) {
      const bool down = (2 * tid & run) == 0;
      for (int apart = run / 4; apart > 0; apart /= 2) {   // in threads
        u64 px, py;
        if (apart >= 32) {
          __syncthreads();
          s.sorted[2 * tid] = x, s.sorted[2 * tid + 1] = y;
          __syncthreads();
          px = s.sorted[2 * (tid ^ apart)], py = s.sorted[2 * (tid ^ apart) + 1];
        } else {
          px = __shfl_xor_sync(kAll, x, apart), py = __shfl_xor_sync(kAll, y, apart);
        }
        const bool larger = ((tid & apart) == 0) == down;
        x = larger == (px > x) ? px : x;
        y = larger == (py > y) ? py : y;
      }
      if ((x < y) == down) {
        const u64 z = x;
        x = y, y = z;
      }
    }
    __syncthreads();
    s.sorted[2 * tid] = x, s.sorted[2 * tid + 1] = y;   // (threads past `size` hold zeros throughout)
    __syncthreads();
  };
  auto weight_at = [&](u64 order) { return weight_of(weigh, order, s.table); };
  // Of s.sorted's first n the one at which the weights from the first on, `before` being those before them, reach
  // `want` (the last one if they do not).  two: this thread's two weights.
  auto reach = [&](int n, u64 before, const u64* two, u64 want) {
    u64 all;
    const u64 cum = before + block_scan(two[0] + two[1], all);
    if (tid == 0) s.sel = s.sorted[n - 1];
    __syncthreads();
    if (cum < want && cum + two[0] >= want) s.sel = s.sorted[2 * tid];
    else if (cum + two[0] < want && cum + two[0] + two[1] >= want) s.sel = s.sorted[2 * tid + 1];
    __syncthreads();
    return s.sel;
  };
  auto share_of = [&](u64 all) { return max(1ull, p > 0.f ? times_fraction(all, p, true) : 0ull); };   // top-p's

  // The token at which the sum of value_at(x, order) in the order of the index exceeds target_of(all): given
  // the warps' sums, `sum` of each lane's, the run that holds it is gone through once more, by all warps of its CTA,
  // a step to a warp.  found(index, x, all) is called by the thread that has it.
  auto locate = [&](u64 sum, auto value_at, auto target_of, auto found) {
    sum = warp_sum_u64(sum);
    __syncthreads();
    if (lane == 0) s.runs[warp] = sum;
    __syncthreads();
    u64 w0, w1;   // before warp `lane` of this CTA, and with it
    auto scan = [&](const u64* of, u64 before) {
      const u64 w = of[lane];
      w1 = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 up = __shfl_up_sync(kAll, w1, o);
        if (lane >= o) w1 += up;
      }
      w1 += before;
      w0 = w1 - w;
      return __shfl_sync(kAll, w1, 31);
    };
    const u64 mine = scan(s.runs, 0ull);
    if (tid == 0) s.slot[turn][0] = mine;
    barrier();
    const u64 of_rank = lane < ranks ? from_rank(&s.slot[turn][0], lane) : 0ull;
    turn ^= 1;
    const u64 all = warp_sum_u64(of_rank), at = target_of(all);
    u64 before = warp_sum_u64(lane < rank ? of_rank : 0ull);
    if (before <= at && at < before + mine) {   // (all of the CTA)
      w0 += before, w1 += before;
      if (warp == 0 && w0 <= at && at < w1) s.found_run = (uint32_t)lane, s.sel = w0;
      __syncthreads();
      const int f0 = first_step(rank * kWarps + (int)s.found_run), f1 = first_step(rank * kWarps + (int)s.found_run + 1);
      before = s.sel;
      for (int base = f0; base < f1; base += kWarps) {
        const int step = base + warp;
        float x[V];
        u64 w[V], ws = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = -inf;
        if (step < f1) load(step, x);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          w[j] = step < f1 && there(index_of(step, j)) ? value_at(x[j], order_of(x[j], index_of(step, j))) : 0ull;
          ws += w[j];
        }
        u64 wi = ws;   // up to and with this lane
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const u64 up = __shfl_up_sync(kAll, wi, o);
          if (lane >= o) wi += up;
        }
        __syncthreads();
        if (lane == 31) s.warp_a[warp] = wi;
        __syncthreads();
        before = scan(s.warp_a, before);
        u64 c = __shfl_sync(kAll, w0, warp) + wi - ws;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (c <= at && at < c + w[j]) found(index_of(step, j), x[j], all);
          c += w[j];
        }
        if (before > at) break;   // (all threads: the same sums)
      }
    }
  };
  auto weight_from = [&](float x, u64 order) { return order >= last ? weigh(x, s.table) : 0ull; };
  auto draw = [&](u64 sum) {
    locate(sum, weight_from, [&](u64 all) { return times_fraction(all, u, false); },
           [&](int i, float x, u64 all) { answer(i, x, all); });
    barrier();   // nobody leaves while its sums are read
  };
  // this lane's share of the weights of tokens that `takes` says yes to: their logits are collected until there are
  // weights for a whole warp to compute
  auto sum_weights = [&](auto takes, auto lists) {
    float* keep = s.keep[warp];
    uint32_t n = 0;
    u64 sum = 0;
    for_steps([&](int step, const float* x) {
      lists(x, step);
      uint32_t in = 0u;
#pragma unroll
      for (int j = 0; j < V; ++j) in |= (takes(x[j], order_of(x[j], index_of(step, j))) ? 1u : 0u) << j;
      while (const uint32_t mask = __ballot_sync(kAll, in != 0u)) {   // one of each lane's at a time
        const int at = __ffs(in) - 1;
        float of = x[0];
#pragma unroll
        for (int j = 1; j < V; ++j) of = at == j ? x[j] : of;
        if (in) keep[n + __popc(mask & ((1u << lane) - 1u))] = of;
        in &= in - 1u;
        n += __popc(mask);
        __syncwarp();
        if (n >= 32u) {
          n -= 32u;
          sum += weigh(keep[n + lane], s.table);
          __syncwarp();
        }
      }
    });
    if ((uint32_t)lane < n) sum += weigh(keep[lane], s.table);
    __syncwarp();
    return sum;
  };

  auto no_list = [](const float*, int) {};
  const bool by_weight = p < 1.f;
  bool by_count = k > 0 && k < a.vocab, radix = false;
  u64 stays = 0ull;   // the last of the order that top-k lets through, once it is known by itself
  // (twice where top-k's border has to be found before top-p's sum: its tokens are more than a list holds)
  while (by_count || by_weight) {
    if (by_count) {
      for_steps([&](int step, const float* x) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (weighs(x[j])) atomicAdd(&s.bins[bin_of(x[j])], 1u);
      });
    } else {
      uint32_t *low = warp_bins + warp * kBins, *high = low + kWarps * kBins;
      for_steps([&](int step, const float* x) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (!weighs(x[j]) || (stays != 0ull && order_of(x[j], index_of(step, j)) < stays)) continue;
          const int bin = bin_of(x[j]);
          const u64 w = weigh(x[j], s.table);
          atomicAdd(&s.bins[bin], 1u);
          const uint32_t lo = (uint32_t)w, was = atomicAdd(low + bin, lo);
          atomicAdd(high + bin, (uint32_t)(w >> 32) + (was + lo < was ? 1u : 0u));
        }
      });
      __syncthreads();
      if (tid < kBins) {
        u64 lo = 0ull, hi = 0ull;
#pragma unroll 8
        for (int i = 0; i < kWarps; ++i) lo += warp_bins[i * kBins + tid], hi += warp_bins[(kWarps + i) * kBins + tid];
        s.weights[tid] = lo + (hi << 32);
      }
    }
    barrier();
    uint32_t bin;
    u64 before = 0, in = 0, want = 0, all;
    const u64 n = tid < kBins ? sum_of(&s.bins[tid]) : 0ull;
    u64 upto = block_scan(n, all), count, cin;   // tokens up to the bin, in it
    if (by_count) {
      bin_at(n, (u64)k, upto, all, bin, before, in);
      cin = in, count = before + in;
    } else {
      const u64 w = tid < kBins ? sum_of(&s.weights[tid]) : 0ull;
      const u64 cum = block_scan(w, all);
      want = share_of(all);
      bin_at(w, want, cum, all, bin, before, in);
      __syncthreads();
      if (tid == (int)bin) s.sel = upto + n, s.sel_in = n;
      __syncthreads();
      count = s.sel, cin = s.sel_in;
    }
    // (before the last but one nothing is without weight)
    const float from = (float)bin, to = bin == kBins - 2 ? inf : (float)(bin + 1);
    auto again = [&] {   // (nobody reads this CTA's any more)
      if (tid < kBins) s.bins[tid] = 0u;
      if (tid == 0) s.listed = 0u;
      __syncthreads();
    };
    if (by_count && bin == kBins - 1) {   // what top-k leaves out has no weight
      by_count = false;
      k = 0;
      barrier();
      again();
      continue;
    }
    // a step's tokens of the border's bin
    auto in_bin = [&](const float* x, int step) {
      uint32_t in = 0u;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float place = place_of(x[j]);
        in |= (place >= from && place < to ? 1u : 0u) << j;
      }
      if (bin == kBins - 2) {
#pragma unroll
        for (int j = 0; j < V; ++j) in &= ~((weighs(x[j]) ? 0u : 1u) << j);
      }
      if (stays != 0ull) {
#pragma unroll
        for (int j = 0; j < V; ++j) in &= ~((order_of(x[j], index_of(step, j)) < stays ? 1u : 0u) << j);
      }
      return in;
    };
    if (count <= kCap) {
      // all that can stay comes together in rank 0, which goes on alone
      for_steps([&](int step, const float* x) {
        uint32_t in = 0u;
#pragma unroll
        for (int j = 0; j < V; ++j)
          in |= (place_of(x[j]) < to && weighs(x[j]) && (stays == 0ull || order_of(x[j], index_of(step, j)) >= stays) ? 1u : 0u) << j;
        list_up(in, x, step);
      });
      const int n = bring_together();
      // by sorting
      auto by_sort = [&] {
        sort(n);
        const int kept = by_count ? min(k, n) : n;
        // two tokens per thread, from the first of the order on
        u64 w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = 2 * tid + i < kept ? weight_at(s.sorted[2 * tid + i]) : 0ull;
        if (by_weight) {
          u64 all;
          if (by_count) {
            block_scan(w[0] + w[1], all);
            want = share_of(all);
          }
          last = max(last, reach(kept, 0ull, w, want));
        } else {
          last = max(last, s.sorted[kept - 1]);
        }
        // the draw, in the order of the index: what stays, sorted by ~index
        int stay = 0;   // tokens that do
#pragma unroll
        for (int i = 0; i < 2; ++i) stay += 2 * tid + i < kept && s.sorted[2 * tid + i] >= last;
        u64 left;
        block_scan((u64)stay, left);
        const int m = (int)left;
        __syncthreads();
        for (int i = tid; i < m; i += kThreads) {
          const u64 c = s.sorted[i];
          s.list[i] = c << 32 | c >> 32;   // (~index, key): the first token has the largest
        }
        __syncthreads();
        sort(m);
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = 2 * tid + i < m ? weigh(value_of((uint32_t)s.sorted[2 * tid + i]), s.table) : 0ull;
        u64 total;
        const u64 sum = block_scan(w[0] + w[1], total);
        const u64 at = times_fraction(total, u, false);
        if (sum <= at && at < sum + w[0] + w[1]) {
          const u64 c = s.sorted[2 * tid + (sum + w[0] <= at)];
          answer((int)(kAll - (uint32_t)(c >> 32)), value_of((uint32_t)c), total);
        }
      };
      // by histograms of the list
      auto by_picks = [&] {
        const float per = (float)kBins / (float)(bin + 1), per_index = (float)kBins / (float)a.vocab;
        u64 border = 0ull, c[2], w[2], of[2] = {};
        int by_key[2], by_index[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = tid + i * kThreads;
          c[i] = at < n ? s.list[at] : 0ull;
          w[i] = at < n ? weight_at(c[i]) : 0ull;
          by_key[i] = min((int)(fminf(place_of(value_of((uint32_t)(c[i] >> 32))), (float)kBins) * per), kBins - 1);
          by_index[i] = min((int)((float)(kAll - (uint32_t)c[i]) * per_index), kBins - 1);
        }
        __syncthreads();   // (the histograms of the row are read)
        auto pick_of = [&](u64 target, const int* bins, bool index) {
          return pick(s, make_ulonglong2(c[0], c[1]), make_ulonglong2(of[0], of[1]), target, bins[0], bins[1], index);
        };
        if (by_count) {
#pragma unroll
          for (int i = 0; i < 2; ++i) of[i] = tid + i * kThreads < n;
          if (!(border = pick_of((u64)min(k, n), by_key, false))) return false;
        }
        auto sums = [&](u64 from) {   // of: the weights of what stays; their sum
#pragma unroll
          for (int i = 0; i < 2; ++i) of[i] = c[i] >= from ? w[i] : 0ull;
          u64 all;
          block_scan(of[0] + of[1], all);
          return all;
        };
        if (by_weight) {
          const u64 all = sums(border);
          if (by_count) want = share_of(all);
          if (!(border = pick_of(want, by_key, false))) return false;
        }
        const u64 total = sums(max(last, border));
        const u64 found = pick_of(times_fraction(total, u, false) + 1ull, by_index, true);
        if (!found) return false;
        if (tid == 0) answer((int)(kAll - (uint32_t)found), value_of((uint32_t)(found >> 32)), total);
        return true;
      };
      // few: a thread per value goes through all of them, and knows how many and what weights come before its own
      auto by_all = [&] {
        u64 c = 0ull, w = 0ull;
        if (tid < n) {
          c = s.list[tid];
          w = weight_at(c);
          s.pairs[tid] = make_ulonglong2(c, w);
        }
        __syncthreads();
        const bool mine = tid < n;
        if (by_count || by_weight) {
          int place = 0;
          u64 cum = 0ull;
          if (warp * 32 < n)
            for (int j = 0; j < n; ++j) {
              const ulonglong2 of = s.pairs[j];
              if (of.x > c) ++place, cum += of.y;
            }
          const int kept = by_count ? min(k, n) : n;
          if (mine && place == kept - 1) s.sel = c, s.sel_in = cum + w;   // the last one, and the sum of all
          if (by_weight) {
            __syncthreads();
            if (by_count) want = share_of(s.sel_in);
            if (mine && place < kept && cum < want && cum + w >= want) s.sel = c;   // (the last one again, or an earlier one)
          }
          __syncthreads();
          last = max(last, s.sel);
        }
        u64 cum = 0ull, total = 0ull;
        if (warp * 32 < n)
          for (int j = 0; j < n; ++j) {
            const ulonglong2 of = s.pairs[j];
            if (of.x < last) continue;
            total += of.y;
            if ((uint32_t)of.x > (uint32_t)c) cum += of.y;   // (~index: the earlier ones are larger)
          }
        const u64 at = times_fraction(total, u, false);
        if (mine && c >= last && cum <= at && at < cum + w) answer((int)(kAll - (uint32_t)c), value_of((uint32_t)(c >> 32)), total);
      };
      if (rank == 0) {
        if (n <= 256) by_all();
        else if (!by_picks()) by_sort();
      }
      barrier();   // nobody leaves while its list is read
      return;
    } else if (cin <= kCap) {
      // the border's bin alone, whose sorted tokens hold the border; meanwhile the weights before it
      u64 sum = 0ull;
      if (by_count && by_weight) {
        for_steps([&](int step, const float* x) { list_up(in_bin(x, step), x, step); });
      } else {
        last = max(last, stays);
        if (by_count || place_of(value_of((uint32_t)(last >> 32))) < from) {
          // (no sums by bin, or min-p's border before the bin's)
          sum = sum_weights([&](float x, u64 order) { return place_of(x) < from && (last == 0ull || order >= last); },
                            [&](const float* x, int step) { list_up(in_bin(x, step), x, step); });
        } else {
          const uint32_t *low = warp_bins + warp * kBins, *high = low + kWarps * kBins;
          for (int i = lane; i < (int)bin; i += 32) sum += (u64)low[i] + ((u64)high[i] << 32);
          for_steps([&](int step, const float* x) { list_up(in_bin(x, step), x, step); });
        }
      }
      const int n = bring_together();
      if (rank == 0) {
        sort(n);
        u64 border;
        if (by_count) {
          border = s.sorted[min(max(k - (int)before - 1, 0), kCap - 1)];
        } else {
          u64 w[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) w[i] = 2 * tid + i < n ? weight_at(s.sorted[2 * tid + i]) : 0ull;
          border = reach(n, before, w, want);
        }
        if (tid == 0) s.slot[turn][0] = border;
      }
      barrier();
      const u64 border = from_rank(&s.slot[turn][0], 0);
      turn ^= 1;
      if (by_count && by_weight) {
        stays = border;
        by_count = false;
        again();
        continue;
      }
      last = max(last, border);
      // the bin's tokens that stay, into the sums of their runs: this CTA's, in its list
      if (lane == 0) s.runs[warp] = 0ull;
      const int own = rank == 0 && ranks > 1 ? (int)s.counts[0] : (int)min(s.listed, (uint32_t)kCap);
      __syncthreads();
      for (int i = tid; i < own; i += kThreads) {
        const u64 c = s.list[i];
        if (c < last) continue;
        const int step = (int)((kAll - (uint32_t)c + shift) / (32 * V));
        int w = (int)(((long long)step * shares + shares - 1) / steps_all) - rank * kWarps;   // its run, or one beside it
        w = min(max(w, 0), kWarps - 1);
        while (w > 0 && first_step(rank * kWarps + w) > step) --w;
        while (w < kWarps - 1 && first_step(rank * kWarps + w + 1) <= step) ++w;
        atomicAdd(&s.runs[w], weight_at(c));
      }
      __syncthreads();
      if (lane == 0) sum += s.runs[warp];
      draw(sum);
      return;
    }
    radix = true;
    break;
  }

  if (radix) {
    // Key of the token at which the sum over the tokens of keys above `above`, from the first of the
    // order on, reaches `target`; left: what of the target its key's tokens have to give.
    auto select = [&](u64 target, uint32_t above, bool weights, u64& left) -> uint32_t {
      uint32_t prefix = 0u, mask = 0u;
      for (int shift = 24; shift >= 0; shift -= 8) {
        u64* hist = s.hist[turn];
        if (tid < 256) hist[tid] = 0ull;
        __syncthreads();
        for (int step = step0; step < step1; ++step) {
          float x[V];
          load(step, x);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const uint32_t key = key_of(x[j]);
            u64 w = 0ull;
            if (key > above && (key & mask) == prefix && there(index_of(step, j))) w = weights ? weigh(x[j], s.table) : 1ull;
            // lanes of the first one's digit together (many equal logits would queue up at one address)
            const uint32_t digit = (key >> shift) & 255u, active = __ballot_sync(kAll, w != 0ull);
            if (!active) continue;
            const uint32_t lead = __shfl_sync(kAll, digit, __ffs(active) - 1);
            const bool with = w != 0ull && digit == lead;
            const u64 sum = warp_sum_u64(with ? w : 0ull);
            if (lane == 0) atomicAdd(&hist[lead], sum);
            if (w && !with) atomicAdd(&hist[digit], w);
          }
        }
        barrier();
        // bins from the first of the order down
        u64 n = 0;
        if (tid < 256)
          for (int i = 0; i < ranks; ++i) n += from_rank(&hist[255 - tid], i);
        u64 all;
        const u64 cum = block_scan(n, all);
        if (tid < 256 && cum < target && cum + n >= target) s.sel_bin = 255u - tid, s.sel = target - cum;
        __syncthreads();
        prefix |= s.sel_bin << shift;
        mask |= 255u << shift;
        target = s.sel;
        turn ^= 1;
      }
      left = target;
      return prefix;
    };
    uint32_t border = 0u;   // tokens of keys above it stay, and of those with its key the first `ties`
    u64 ties = 0ull;
    barrier();   // (the histograms lie where the bins are read)
    if (k > 0 && k < a.vocab) border = select((u64)k, 0u, false, ties);
    if (by_weight) {
      u64 all = sum_weights([&](float x, u64 order) { return (uint32_t)(order >> 32) > border; }, no_list), ignored;
      all = warp_sum_u64(all);
      block_scan(lane == 0 ? all : 0ull, ignored);
      if (tid == 0) s.slot[turn][0] = ignored;
      barrier();
      all = warp_sum_u64(lane < ranks ? from_rank(&s.slot[turn][0], lane) : 0ull);
      turn ^= 1;
      const u64 one = ties ? weigh(value_of(border), s.table) : 0ull;
      const u64 want = share_of(all + ties * one);
      if (want <= all) {
        u64 left;
        border = select(want, border, true, left);
        const u64 w = weigh(value_of(border), s.table);
        ties = (left + w - 1) / max(w, 1ull);
      } else {   // the tokens that top-k left at its border
        ties = min(ties, (want - all + one - 1) / max(one, 1ull));
      }
    }
    if (border > 0u) {
      // the last of the ties that stay
      auto tie = [&](float x, u64 order) { return (uint32_t)(order >> 32) == border ? 1ull : 0ull; };
      u64 n = 0;
      for (int step = step0; step < step1; ++step) {
        float x[V];
        load(step, x);
#pragma unroll
        for (int j = 0; j < V; ++j) n += there(index_of(step, j)) ? tie(x[j], order_of(x[j], index_of(step, j))) : 0ull;
      }
      if (tid == 0) s.sel_in = 0ull;
      locate(n, tie, [&](u64 all) { return min(ties, all) - 1ull; }, [&](int i, float x, u64 all) { s.sel_in = order_of(x, i); });
      __syncthreads();
      if (tid == 0) s.slot[turn][0] = s.sel_in;
      barrier();
      last = max(last, warp_max_u64(lane < ranks ? from_rank(&s.slot[turn][0], lane) : 0ull));
      turn ^= 1;
    }
  }

  // What stays, summed by warps' runs.
  u64 sum = 0;
  if (last == 0ull) {
    for_steps([&](int step, const float* x) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum += weigh(x[j], s.table);
    });
  } else {
    sum = sum_weights([&](float x, u64 order) { return order >= last; }, no_list);
  }
  draw(sum);
}

}  // namespace

cudaError_t init_draw_kernels() {
  const cudaError_t e = cudaFuncSetAttribute(draw_kernel<bf16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWarpBins);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(draw_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWarpBins);
}

cudaError_t launch_draw(const DrawArgs& a, Dtype dt, cudaStream_t st) {
  // CTAs of a row: up to 8 while there are SMs for all, and 4096 logits for each.  One bf16 row under top-k 40 and top-p
  // 0.95 with 2048 / 4096 / 8192 logits to a CTA, us: 4096 logits 11.3 / 9.1 / 9.1, 8192 11.7 / 11.2 / 9.1, 16384 11.7 /
  // 11.4 / 11.1, 32768 11.7 / 11.7 / 11.5; under top-p 0.9 alone 19.5 / 16.9 / 16.8, 20.7 / 19.8 / 17.0, 21.8 / 22.1 /
  // 21.2, 25.1 / 25.1 / 25.5.  (8192 would be the better line for rows of 8192 to 16384.)
  int ranks = 1;
  while (ranks < kRanks && (long long)a.batch * ranks * 2 <= a.num_sms && a.vocab >= ranks * 2 * 4096) ranks *= 2;
  const Overlap overlap;
  return launch_kernel_cluster(dt == DT_BF16 ? draw_kernel<bf16> : draw_kernel<float>, dim3(ranks, a.batch), dim3(kThreads), kWarpBins, st, dim3(ranks, 1, 1), a);
}

}  // namespace ravel
