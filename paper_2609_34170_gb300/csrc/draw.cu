// Drawing a token from a row of logits: top-k, top-p, min-p and the draw itself, without a sort.
//
// Weights are whole numbers, 2^43 exp((x - max) / T) rounded, so that their sums are exact and
// the same in any order; a row is at most 2^20 long, its sum below 2^64.  The order of the tokens (by
// logit, equal ones by index) is not made: a limit is a border in it, a key and how many of the
// tokens with that key stay.
//
// A cluster of CTAs per row.  The row's maximum first; then a histogram of 512 bins between the
// maximum and the least logit that has a weight, of counts and, where top-p alone limits, of weights: the
// bin that holds the border.  Where the tokens up to that bin are at most 2048, they are brought
// together in one CTA, which sorts them and does the rest by itself.  Where they are more, the
// bin's own tokens are, which gives the border, and the cluster sums what stays in the order of the index: by
// warps' runs first, then within the run that holds the token.  Where even the bin holds more
// (thousands of nearly equal logits), a radix selection over the keys' four bytes finds the border.
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

typedef unsigned long long u64;

// 2^(j / 1024) in units of 2^-62
struct ExpTable {
  u64 v[1024];
  constexpr ExpTable() : v() {
    for (int j = 0; j < 1024; ++j) {
      const double x = 0.6931471805599453094 * j / 1024.0;
      double term = 1.0, sum = 1.0;
      for (int i = 1; i < 22; ++i) {
        term *= x / i;
        sum += term;
      }
      v[j] = (u64)(sum * 4611686018427387904.0);
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
// from its series, r below 2^-11, whose first term is a product in two floats.  About 2^-43 of the
// weight off.  (In fp32 a weight is 2^-22 off and its error grows with x: at 100000 tokens one
// border in a hundred falls elsewhere than in 64 bits.)
struct Weigher {
  float top, ch, cl;   // half the largest logit; twice log2(e) / T
  __device__ __forceinline__ u64 operator()(float logit, const u64* table) const {
    const float x = 0.5f * logit;   // (halves, so that no difference overflows)
    const float dh = x - top;
    const float v = dh - x, dl = (x - (dh - v)) - (top + v);
    const float yh = dh * ch;
    if (!(yh > -44.f)) return 0ull;
    const float ye = __fmaf_rn(dh, ch, -yh) + __fmaf_rn(dh, cl, dl * ch);
    const float shifted = __fmaf_rn(yh, 1024.f, 12582912.f);   // 1.5 * 2^23: q in the low bits
    const int q = __float_as_int(shifted) - 0x4b400000;
    const float rest = __fmaf_rn(shifted - 12582912.f, -0x1p-10f, yh);   // exact, up to 2^-11
    // r in units of 2^-42: ln 2 rest as a float and what it lacks, the small terms with the latter
    const float rh = rest * 0.693147182f;
    const float f = (rest + ye) * 0.693147182f;
    const float rl = __fmaf_rn(rest, 0.693147182f, -rh) + __fmaf_rn(rest, -1.90465421e-9f, ye * 0.693147182f) +
                     f * f * __fmaf_rn(f, 0.166666667f, 0.5f);
    const int r = __float2int_rn(rh * 0x1p42f) + __float2int_rn(rl * 0x1p42f);
    const u64 t = table[q & 1023];   // in units of 2^-62
    const u64 w = t + (u64)((long long)(uint32_t)(t >> 31) * r >> 11);
    const int down = 62 - kBits - (q >> 10);
    return (w + (1ull << (down - 1))) >> down;
  }
};

// floor(f * s), or the next whole number at or above, for a finite f >= 0
__device__ __forceinline__ u64 times_fraction(u64 s, float f, bool up) {
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
  u64 table[1024];
  union {
    uint32_t bins[3][kBins];    // of a CTA: counts, weights' low and high words
    u64 hist[2][256];           // radix selection
  };
  u64 list[kCap];               // (key, ~index), in the order of the index
  union {
    u64 sorted[kCap];           // the same, from the largest down
    float keep[kWarps][64];     // a warp's logits that wait for their weights
  };
  u64 slot[2][2];               // what this CTA gives to a reduction
  u64 warp_a[kWarps], warp_b[kWarps];
  u64 sel_left, sel_before, sel_in;
  double per_t, least;          // 1 / T; T log(min_p)
  float ch, cl;                 // Weigher's
  uint32_t counts[kRanks];
  uint32_t sel_bin, sel_key, listed, found_run;
  u64 run_at, run_equal;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) draw_kernel(DrawArgs a) {
  __shared__ DrawShared s;
  constexpr int V = 16 / sizeof(T);
  constexpr uint32_t kAll = 0xffffffffu;
  const int ranks = (int)gridDim.x, rank = ranks > 1 ? (int)cluster_ctarank() : 0, b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float inf = __uint_as_float(0x7f800000u);
  s.table[tid] = kExp.v[tid];
  pdl_trigger();
  pdl_wait();
  const float u = a.u[b], t = a.temperature ? a.temperature[b] : 1.f, p = a.top_p ? a.top_p[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  int k = a.top_k ? a.top_k[b] : 0;
  if (tid == kThreads - 1) {   // (one thread: 64-bit floats come two to a clock)
    const double c = 2.0 * 1.4426950408889634074 / (double)t;
    s.ch = (float)c;
    s.cl = (float)(c - (double)s.ch);
    s.per_t = 1.0 / (double)t;
    s.least = mp > 0.f ? (double)t * log((double)fminf(mp, 1.f)) : 0.0;
  }
  const T* row = (const T*)a.logits + (long long)b * a.row;
  // this warp's run of the row: whole steps of 32 lanes x V values
  const int steps_all = (a.vocab + 32 * V - 1) / (32 * V), shares = ranks * kWarps, share = rank * kWarps + warp;
  const int step0 = (int)((long long)steps_all * share / shares), step1 = (int)((long long)steps_all * (share + 1) / shares);

  auto load = [&](int step, float* x) {   // values past the end: -inf
    const int i = (step * 32 + lane) * V;
    if (a.vec && i + V <= a.vocab) {
      const uint4 w = *(const uint4*)(row + i);
      T t[V];
      memcpy(t, &w, 16);
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = to_f32(t[j]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = i + j < a.vocab ? to_f32(row[i + j]) : -inf;
    }
  };
  auto index_of = [&](int step, int j) { return (step * 32 + lane) * V + j; };
  int turn = 0;
  auto barrier = [&] {
    if (ranks > 1) cluster_sync();
    else __syncthreads();
  };
  // sum of 32-bit words of all ranks (the loads on their way together)
  auto sum_of = [&](const uint32_t* p) {
    if (ranks == 1) return (u64)*p;
    uint32_t x[kRanks];
#pragma unroll
    for (int i = 0; i < kRanks; ++i) x[i] = ld_cluster_u32(mapa_shared(smem_u32(p), (uint32_t)min(i, ranks - 1)));
    u64 n = 0;
#pragma unroll
    for (int i = 0; i < kRanks; ++i) n += i < ranks ? x[i] : 0u;
    return n;
  };
  auto from_rank = [&](const u64* p, int i) { return ranks > 1 ? ld_cluster_u64(mapa_shared(smem_u32(p), (uint32_t)i)) : *p; };
  // maxima or sums of x and of y over the row's threads, for every thread
  u64 before_x, before_y;
  auto reduce = [&](u64 x, u64 y, bool maximum, u64& rx, u64& ry) {
    x = maximum ? warp_max_u64(x) : warp_sum_u64(x);
    y = maximum ? warp_max_u64(y) : warp_sum_u64(y);
    if (lane == 0) s.warp_a[warp] = x, s.warp_b[warp] = y;
    __syncthreads();
    if (warp == 0) {
      u64 p = s.warp_a[lane], r = s.warp_b[lane];
      p = maximum ? warp_max_u64(p) : warp_sum_u64(p);
      r = maximum ? warp_max_u64(r) : warp_sum_u64(r);
      if (lane == 0) s.slot[turn][0] = p, s.slot[turn][1] = r;
    }
    barrier();
    // lane i takes rank i's
    x = lane < ranks ? from_rank(&s.slot[turn][0], lane) : 0ull;
    y = lane < ranks ? from_rank(&s.slot[turn][1], lane) : 0ull;
    rx = maximum ? warp_max_u64(x) : warp_sum_u64(x);
    ry = maximum ? warp_max_u64(y) : warp_sum_u64(y);
    before_x = warp_sum_u64(lane < rank ? x : 0ull);   // of the ranks before this one
    before_y = warp_sum_u64(lane < rank ? y : 0ull);
    turn ^= 1;
  };
  // sum of x over the threads before this one and, in all, over the CTA
  auto block_scan = [&](u64 x, u64& all) {
    u64 upto = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 up = __shfl_up_sync(kAll, upto, o);
      if (lane >= o) upto += up;
    }
    __syncthreads();
    if (lane == 31) s.warp_a[warp] = upto;
    __syncthreads();
    u64 w = s.warp_a[lane], ws = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 up = __shfl_up_sync(kAll, ws, o);
      if (lane >= o) ws += up;
    }
    all = __shfl_sync(kAll, ws, 31);
    return __shfl_sync(kAll, ws - w, warp) + upto - x;
  };

  // the first of the order, the least finite logit, and what is no number
  u64 best = 0, low = 0;
#pragma unroll 2
  for (int step = step0; step < step1; ++step) {
    float x[V];
    load(step, x);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint32_t key = key_of(x[j]);
      const u64 c = (u64)key << 32 | (kAll - (uint32_t)index_of(step, j));
      best = c > best ? c : best;
      if (!(x[j] < inf)) low |= 1ull << 32;
      else if (x[j] > -inf) low = (low & 1ull << 32) | max((uint32_t)low, ~key);
    }
  }
  reduce(best, low, true, best, low);
  const float top = value_of((uint32_t)(best >> 32));
  auto answer = [&](int token, float log_prob) {
    a.tokens[b] = token;
    if (a.log_probs) a.log_probs[b] = log_prob;
  };
  const bool none = low >> 32 || !(top > -inf) || !(u >= 0.f && u < 1.f) || !(t < inf) || p != p || mp != mp;
  if (none || t < 0x1p-20f) {
    if (rank == 0 && tid == 0) {
      if (none) answer(-1, -inf);
      else answer((int)(kAll - (uint32_t)best), 0.f);
    }
    barrier();   // (nobody leaves while its slot is read)
    return;
  }
  const Weigher weigh{0.5f * top, s.ch, s.cl};
  auto log_prob = [&](float x, u64 total) {
    const int e = 63 - __clzll((long long)total);
    const float m = (float)total * exp2f((float)-e);   // total = m 2^e
    return (float)(((double)x - (double)top) * s.per_t - (double)(e - kBits) * 0.6931471805599453094 - (double)logf(m));
  };
  // least key that min-p lets through
  uint32_t least = 0u;
  if (mp > 0.f) {
    const double limit = (double)top + s.least;
    float f = (float)limit;
    if ((double)f < limit) f = nextafterf(f, inf);
    least = key_of(f);
  }

  // Bins of the order: equal parts of the log2 domain from the maximum down to the least logit or
  // to 2^-44, where weights end; the last one for what has none.  Every step of the formula is
  // monotone in x, rounding included.
  const float y_least = fmaxf((0.5f * value_of(~(uint32_t)low) - weigh.top) * weigh.ch, -44.f);
  const float per_bin = (float)(kBins - 1) / fmaxf(-y_least, 0x1p-40f);
  // place in bins, for bin i from i up to below i + 1 (the last but one: from there on); -1: no weight
  auto place_of = [&](float x) {
    const float y = (0.5f * x - weigh.top) * weigh.ch;
    return y > -44.f ? fminf(-y * per_bin, (float)(kBins - 2)) : -1.f;
  };
  // The bin at which `part` 0 (counts) or 1 (weights), summed from the first on, reaches `target`, what
  // comes before it and what is in it; target > all: the last one.  For every thread of the row.
  auto bin_at = [&](int part, auto target_of, uint32_t& bin, u64& before, u64& in) {
    u64 n = 0;
    if (tid < kBins) n = part == 0 ? sum_of(&s.bins[0][tid]) : sum_of(&s.bins[1][tid]) + (sum_of(&s.bins[2][tid]) << 32);
    u64 all;
    const u64 cum = block_scan(n, all);
    const u64 target = target_of(all);
    if (tid == 0) s.sel_bin = kBins - 1, s.sel_before = all, s.sel_in = 0;
    __syncthreads();
    if (tid < kBins && cum < target && cum + n >= target) s.sel_bin = tid, s.sel_before = cum, s.sel_in = n;
    __syncthreads();
    bin = s.sel_bin, before = s.sel_before, in = s.sel_in;
  };
  // Tokens of the bins first .. last, in the order of the index, into rank 0's list; their number.
  auto gather = [&](uint32_t first, uint32_t last) {
    const float from = (float)first, to = (float)(last + 1);
    auto wanted = [&](float x) {   // (past the end there is no weight)
      const float place = place_of(x);
      return place >= from && place < to;
    };
    uint32_t n = 0;
#pragma unroll 2
    for (int step = step0; step < step1; ++step) {
      float x[V];
      load(step, x);
#pragma unroll
      for (int j = 0; j < V; ++j) n += wanted(x[j]);
    }
    n = __reduce_add_sync(kAll, n);
    u64 all;
    u64 at = block_scan(lane == 0 ? n : 0ull, all);
    at = __shfl_sync(kAll, at, 0);
    if (n) {
      for (int step = step0; step < step1; ++step) {
        float x[V];
        load(step, x);
        uint32_t mine = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) mine += wanted(x[j]);
        if (!__any_sync(kAll, mine)) continue;
        uint32_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t up = __shfl_up_sync(kAll, upto, o);
          if (lane >= o) upto += up;
        }
        uint32_t put = (uint32_t)at + upto - mine;
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (wanted(x[j]) && put < kCap) s.list[put++] = (u64)key_of(x[j]) << 32 | (kAll - (uint32_t)index_of(step, j));
        at += __shfl_sync(kAll, upto, 31);
      }
    }
    if (tid == 0) s.slot[turn][0] = all;
    barrier();
    int total = (int)min(all, (u64)kCap);
    if (rank == 0 && ranks > 1) {
      if (tid < ranks) s.counts[tid] = (uint32_t)from_rank(&s.slot[turn][0], tid);
      __syncthreads();
      for (int r = 1; r < ranks; ++r) total += (int)s.counts[r];
      total = min(total, kCap);   // (the counts said so; logits that change under the kernel must not write past the list)
      for (int flat = (int)min(all, (u64)kCap) + tid; flat < total; flat += kThreads) {   // behind its own
        int i = flat - (int)all, r = 1;
        while (i >= (int)s.counts[r]) i -= (int)s.counts[r++];
        s.list[flat] = from_rank(&s.list[i], r);
      }
      __syncthreads();
    }
    turn ^= 1;
    return total;   // (of rank 0)
  };
  // s.sorted: the n values of s.list from the largest down, zeros behind; a bitonic network
  auto sort = [&](int n) {
    int size = 64;
    while (size < n) size *= 2;
    for (int i = tid; i < size; i += kThreads) s.sorted[i] = i < n ? s.list[i] : 0ull;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
      for (int stride = run / 2; stride > 0; stride /= 2) {
        if (tid < size / 2) {
          const int i = 2 * tid - (tid & (stride - 1)), j = i + stride;
          const u64 x = s.sorted[i], y = s.sorted[j];
          if ((x < y) == ((i & run) == 0)) s.sorted[i] = y, s.sorted[j] = x;
        }
        // (up to 32 apart, a warp's pairs stay within its own 64 values)
        if (stride > 32 || (stride == 1 && run >= 64)) __syncthreads();
        else __syncwarp();
      }
    __syncthreads();
  };

  // The border: tokens of keys above it stay, and of those with its key the first `ties`.
  uint32_t border = 0u;   // (below every key)
  u64 ties = 0ull;
  const bool by_count = k > 0 && k < a.vocab, by_weight = p < 1.f;
  bool radix = false;
  if (by_count || by_weight) {
    for (int i = tid; i < kBins; i += kThreads) s.bins[0][i] = s.bins[1][i] = s.bins[2][i] = 0u;
    __syncthreads();
#pragma unroll 2
    for (int step = step0; step < step1; ++step) {
      float x[V];
      load(step, x);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float place = place_of(x[j]);
        if (place < 0.f) continue;
        const int bin = (int)place;
        atomicAdd(&s.bins[0][bin], 1u);
        if (!by_count) {
          const u64 w = weigh(x[j], s.table);
          const uint32_t lo = (uint32_t)w, was = atomicAdd(&s.bins[1][bin], lo);
          atomicAdd(&s.bins[2][bin], (uint32_t)(w >> 32) + (was + lo < was ? 1u : 0u));
        }
      }
    }
    barrier();
    uint32_t bin, cbin;
    u64 before = 0, in = 0, count = 0, cin = 0, want = 0;
    if (by_count) {
      bin_at(0, [&](u64) { return (u64)k; }, cbin, count, cin);
      bin = cbin;
      if (bin == kBins - 1) k = 0;   // what top-k leaves out has no weight
      count += cin;
    } else {
      bin_at(1, [&](u64 all) { return want = max(1ull, p > 0.f ? times_fraction(all, p, true) : 0ull); }, bin, before, in);
      // tokens up to that bin and in it
      const u64 n = tid <= bin ? sum_of(&s.bins[0][tid]) : 0ull;
      block_scan(n, count);
      block_scan(tid == bin ? n : 0ull, cin);
    }
    if (by_count && k == 0 && by_weight) {
      radix = true;
    } else if (by_count && k == 0) {
      // nothing is left out
    } else if (count <= kCap) {
      // all that can stay comes together in rank 0, which goes on alone
      const int n = gather(0u, bin);
      if (rank == 0) {
        sort(n);
        const int kept = by_count ? k : n;   // (k <= n)
        // two tokens per thread, from the first of the order on
        u64 w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = 2 * tid + i < kept ? weigh(value_of((uint32_t)(s.sorted[2 * tid + i] >> 32)), s.table) : 0ull;
        u64 all;
        const u64 cum = block_scan(w[0] + w[1], all);
        if (by_count) want = by_weight ? max(1ull, p > 0.f ? times_fraction(all, p, true) : 0ull) : all;
        if (!by_weight) want = ~0ull;   // (what stays ends with the kept)
        if (tid == 0) s.sel_left = s.sorted[kept - 1];
        __syncthreads();
        if (cum < want && cum + w[0] >= want) s.sel_left = s.sorted[2 * tid];
        else if (cum + w[0] < want && cum + w[0] + w[1] >= want) s.sel_left = s.sorted[2 * tid + 1];
        __syncthreads();
        const u64 last = max(s.sel_left, (u64)least << 32);
        // the draw, in the order of the index
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u64 c = 2 * tid + i < n ? s.list[2 * tid + i] : 0ull;
          w[i] = 2 * tid + i < n && c >= last ? weigh(value_of((uint32_t)(c >> 32)), s.table) : 0ull;
        }
        u64 total;
        const u64 sum = block_scan(w[0] + w[1], total);
        const u64 at = times_fraction(total, u, false);
        if (sum <= at && at < sum + w[0] + w[1]) {
          const u64 c = s.list[2 * tid + (sum + w[0] <= at)];
          answer((int)(kAll - (uint32_t)c), log_prob(value_of((uint32_t)(c >> 32)), total));
        }
      }
      barrier();   // nobody leaves while its list is read
      return;
    } else if (cin <= kCap && !(by_count && by_weight)) {
      // the border's bin alone, whose sorted tokens hold the border
      const int n = gather(bin, bin);
      if (rank == 0) {
        sort(n);
        u64 last;
        if (by_count) {
          last = s.sorted[k - (int)(count - cin) - 1];
        } else {
          u64 w[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) w[i] = 2 * tid + i < n ? weigh(value_of((uint32_t)(s.sorted[2 * tid + i] >> 32)), s.table) : 0ull;
          u64 all;
          const u64 cum = before + block_scan(w[0] + w[1], all);
          if (cum < want && cum + w[0] >= want) s.sel_left = s.sorted[2 * tid];
          else if (cum + w[0] < want && cum + w[0] + w[1] >= want) s.sel_left = s.sorted[2 * tid + 1];
          __syncthreads();
          last = s.sel_left;
        }
        u64 equal = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u64 c = 2 * tid + i < n ? s.sorted[2 * tid + i] : 0ull;
          equal += c >> 32 == last >> 32 && c >= last;
        }
        u64 all;
        block_scan(equal, all);
        if (tid == 0) s.slot[turn][0] = last >> 32, s.slot[turn][1] = all;
      }
      barrier();
      border = (uint32_t)from_rank(&s.slot[turn][0], 0);
      ties = from_rank(&s.slot[turn][1], 0);
      turn ^= 1;
    } else {
      radix = true;
    }
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
            if (key > above && (key & mask) == prefix && index_of(step, j) < a.vocab) {
              const u64 w = weights ? weigh(x[j], s.table) : 1ull;
              if (w) atomicAdd(&hist[(key >> shift) & 255u], w);
            }
          }
        }
        barrier();
        // bins from the first of the order down
        u64 n = 0;
        if (tid < 256)
          for (int i = 0; i < ranks; ++i) n += from_rank(&hist[255 - tid], i);
        u64 all;
        const u64 cum = block_scan(n, all);
        if (tid < 256 && cum < target && cum + n >= target) s.sel_bin = 255u - tid, s.sel_left = target - cum;
        __syncthreads();
        prefix |= s.sel_bin << shift;
        mask |= 255u << shift;
        target = s.sel_left;
        turn ^= 1;
      }
      left = target;
      return prefix;
    };
    barrier();   // (the histograms lie where the bins are read)
    if (k > 0 && by_count) border = select((u64)k, 0u, false, ties);
    if (by_weight) {
      u64 all = 0, nothing;
      for (int step = step0; step < step1; ++step) {
        float x[V];
        load(step, x);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (key_of(x[j]) > border) all += weigh(x[j], s.table);
      }
      reduce(all, 0ull, false, all, nothing);
      const u64 one = ties ? weigh(value_of(border), s.table) : 0ull;
      const u64 want = max(1ull, p > 0.f ? times_fraction(all + ties * one, p, true) : 0ull);
      if (want <= all) {
        u64 left;
        border = select(want, border, true, left);
        const u64 w = weigh(value_of(border), s.table);
        ties = (left + w - 1) / w;
      } else {   // the tokens that top-k left at its border
        ties = min(ties, (want - all + one - 1) / max(one, 1ull));
      }
    }
  }
  if (least > border) {
    border = least - 1u;
    ties = 0ull;
  }

  // What stays, summed by warps' runs.  Its logits are collected until there are weights for a
  // whole warp to compute.
  const u64 one = ties ? weigh(value_of(border), s.table) : 0ull;
  u64 sum = 0, equal = 0;
  if (border == 0u) {
    for (int step = step0; step < step1; ++step) {
      float x[V];
      load(step, x);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += weigh(x[j], s.table);
    }
  } else {
    float* keep = s.keep[warp];
    uint32_t n = 0;
#pragma unroll 2
    for (int step = step0; step < step1; ++step) {
      float x[V];
      load(step, x);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const uint32_t key = key_of(x[j]);
        equal += key == border && index_of(step, j) < a.vocab;
        const uint32_t mask = __ballot_sync(kAll, key > border);
        if (mask == 0u) continue;
        if (key > border) keep[n + __popc(mask & ((1u << lane) - 1u))] = x[j];
        n += __popc(mask);
        __syncwarp();
        if (n >= 32u) {
          n -= 32u;
          sum += weigh(keep[n + lane], s.table);
          __syncwarp();
        }
      }
    }
    if ((uint32_t)lane < n) sum += weigh(keep[lane], s.table);
  }
  u64 all, all_equal;
  reduce(sum, equal, false, all, all_equal);
  const u64 total = all + min(ties, all_equal) * one;
  const u64 at = times_fraction(total, u, false);   // the token's part of the sum holds this
  auto upto = [&](u64 w, u64 n) { return w + min(ties, n) * one; };
  u64 before = before_x, equal_before = before_y;
  const u64 mine = s.slot[turn ^ 1][0], mine_equal = s.slot[turn ^ 1][1];
  if (upto(before, equal_before) <= at && at < upto(before + mine, equal_before + mine_equal)) {
    // the token is in this CTA: in which warp's run
    u64 w0, w1, e0, e1;   // before warp `lane`, and with it
    auto scan_warps = [&] {
      const u64 w = s.warp_a[lane], e = s.warp_b[lane];
      w1 = w, e1 = e;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 wu = __shfl_up_sync(kAll, w1, o), eu = __shfl_up_sync(kAll, e1, o);
        if (lane >= o) w1 += wu, e1 += eu;
      }
      w1 += before, e1 += equal_before;
      w0 = w1 - w, e0 = e1 - e;
    };
    scan_warps();
    if (warp == 0 && upto(w0, e0) <= at && at < upto(w1, e1)) s.found_run = (uint32_t)lane, s.run_at = w0, s.run_equal = e0;
    __syncthreads();
    // that run again, by all warps: 32 of its steps at a time, a step to a warp
    const int fshare = rank * kWarps + (int)s.found_run;
    const int f0 = (int)((long long)steps_all * fshare / shares), f1 = (int)((long long)steps_all * (fshare + 1) / shares);
    before = s.run_at, equal_before = s.run_equal;
    for (int base = f0; base < f1; base += kWarps) {
      const int step = base + warp;
      float x[V];
      u64 w[V], ws = 0, ns = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = -inf;
      if (step < f1) load(step, x);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const uint32_t key = key_of(x[j]);
        w[j] = key > border ? weigh(x[j], s.table) : 0ull;
        ws += w[j];
        ns += key == border && index_of(step, j) < a.vocab && step < f1;
      }
      u64 wi = ws, ni = ns;   // up to and with this lane
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 wu = __shfl_up_sync(kAll, wi, o), nu = __shfl_up_sync(kAll, ni, o);
        if (lane >= o) wi += wu, ni += nu;
      }
      __syncthreads();
      if (lane == 31) s.warp_a[warp] = wi, s.warp_b[warp] = ni;
      __syncthreads();
      scan_warps();
      u64 c = __shfl_sync(kAll, w0, warp) + wi - ws, e = __shfl_sync(kAll, e0, warp) + ni - ns;
      before = __shfl_sync(kAll, w1, 31), equal_before = __shfl_sync(kAll, e1, 31);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const u64 was = upto(c, e);
        c += w[j];
        e += key_of(x[j]) == border && index_of(step, j) < a.vocab && step < f1;
        if (was <= at && upto(c, e) > at) answer(index_of(step, j), log_prob(x[j], total));
      }
      if (upto(before, equal_before) > at) break;   // (all threads: the same sums)
    }
  }
  barrier();   // nobody leaves while its sums are read
}

}  // namespace

cudaError_t launch_draw(const DrawArgs& a, Dtype dt, cudaStream_t st) {
  // CTAs of a row: up to 8 while there are SMs for all, and work for their warps
  int ranks = 1;
  while (ranks < kRanks && (long long)a.batch * ranks * 2 <= a.num_sms && a.vocab >= ranks * 2 * 4096) ranks *= 2;
  const Overlap overlap;
  return launch_kernel_cluster(dt == DT_BF16 ? draw_kernel<bf16> : draw_kernel<float>, dim3(ranks, a.batch), dim3(kThreads), 0, st, dim3(ranks, 1, 1), a);
}

}  // namespace ravel
