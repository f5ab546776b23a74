// Drawing a token from a row of logits: top-k, top-p, min-p and the draw itself, without a sort.
//
// Weights are whole numbers, 2^43 exp((x - max) / T) rounded, so that their sums are exact and
// the same in any order; a row is at most 2^20 long, its sum below 2^64.  The order of the tokens (by
// logit, equal ones by index) is never made: each limit is a border in it, a key and how many of the
// tokens with that key stay, found by a radix selection over the keys, whose histograms count tokens
// (top-k) or add weights (top-p).  The draw sums what stays in the order of the index: sums of runs
// first, then a walk through the run that holds the token.
#include <algorithm>

#include "common.cuh"
#include "decode.h"
#include "launch.h"
#include "tc_common.cuh"

namespace ravel {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kRanks = 8;        // CTAs of a row at most
constexpr int kBits = 43;        // weight of the likeliest token: 2^43

typedef unsigned long long u64;

// 2^(-j / 1024) in units of 2^-62
struct ExpTable {
  u64 v[1024];
  constexpr ExpTable() : v() {
    for (int j = 0; j < 1024; ++j) {
      const double x = -0.6931471805599453094 * j / 1024.0;
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
// in two floats and the difference and its product with their rounding errors, then in units of
// 2^-46: 2^y = 2^-n 2^(-j / 1024) 2^-g with the middle one from a table and 2^-g = 1 - r, r below 2^-10,
// from its series (the first term as a whole number, the others in fp32).  About 2^-43 of the
// weight off.  (In fp32 a weight is 2^-22 off and its error grows with x: at 100000 tokens one
// border in a hundred falls elsewhere than in 64 bits.)
struct Weigher {
  float top, ch, cl;   // half the largest logit; twice log2(e) / T
  __device__ __forceinline__ void set(float max, double temperature) {
    const double c = 2.0 * 1.4426950408889634074 / temperature;
    top = 0.5f * max;   // (halves, so that no difference overflows)
    ch = (float)c;
    cl = (float)(c - (double)ch);
  }
  __device__ __forceinline__ u64 operator()(float logit, const u64* table) const {
    const float x = 0.5f * logit;
    const float dh = x - top;
    const float v = dh - x, dl = (x - (dh - v)) - (top + v);
    const float yh = dh * ch;
    if (!(yh > -44.f)) return 0ull;
    const float ye = __fmaf_rn(dh, ch, -yh) + __fmaf_rn(dh, cl, dl * ch);
    const int i1 = __float2int_rn(yh * 0x1p24f);
    const float rest = __fmaf_rn(-(float)i1, 0x1p-24f, yh) + ye;
    const long long Y = ((long long)i1 << 22) + __float2int_rn(rest * 0x1p46f);
    const u64 U = Y < 0 ? (u64)-Y : 0ull;
    const int n = (int)(U >> 46);
    const u64 t = table[(U >> 36) & 1023];
    const uint32_t g = (uint32_t)((U & 0xfffffffffull) >> 4);   // 2^-42
    const uint32_t gl = __umulhi(g, 0xb17217f8u);               // times ln 2
    const float gf = (float)gl * 0x1p-42f;
    const uint32_t r = gl - __float2uint_rn(gf * gf * (0.5f - gf * 0.16666667f) * 0x1p42f);
    const u64 w = t - (((u64)(uint32_t)(t >> 32) * r + __umulhi((uint32_t)t, r)) >> 10);
    return (w + (1ull << (62 - kBits - 1 + n))) >> (62 - kBits + n);
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
  u64 hist[2][256], sums[256];
  u64 slot[2][2];             // what this CTA gives to a reduction
  u64 warp_a[kWarps], warp_b[kWarps];
  u64 all_a, all_b;           // of a reduction
  u64 sel_left;
  uint32_t sel_bin;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) draw_kernel(DrawArgs a) {
  __shared__ DrawShared s;
  constexpr int V = 16 / sizeof(T);
  const int ranks = (int)gridDim.x, rank = ranks > 1 ? (int)cluster_ctarank() : 0, b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < 1024; i += kThreads) s.table[i] = kExp.v[i];
  pdl_trigger();
  pdl_wait();
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
      for (int j = 0; j < V; ++j) x[j] = i + j < a.vocab ? to_f32(row[i + j]) : __uint_as_float(0xff800000u);
    }
  };
  int turn = 0;
  auto barrier = [&] {
    if (ranks > 1) cluster_sync();
    else __syncthreads();
  };
  // maximum (or sum) of x and sum of y over the row's threads, for every thread
  auto reduce = [&](u64 x, u64 y, bool maximum, u64& rx, u64& ry) {
    x = maximum ? warp_max_u64(x) : warp_sum_u64(x);
    y = warp_sum_u64(y);
    if (lane == 0) s.warp_a[warp] = x, s.warp_b[warp] = y;
    __syncthreads();
    if (warp == 0) {
      u64 p = lane < kWarps ? s.warp_a[lane] : 0ull, r = lane < kWarps ? s.warp_b[lane] : 0ull;
      p = maximum ? warp_max_u64(p) : warp_sum_u64(p);
      r = warp_sum_u64(r);
      if (lane == 0) s.slot[turn][0] = p, s.slot[turn][1] = r;
    }
    barrier();
    rx = ry = 0ull;
    for (int i = 0; i < ranks; ++i) {
      u64 p, r;
      if (ranks > 1) {
        const uint32_t at = mapa_shared(smem_u32(&s.slot[turn][0]), (uint32_t)i);
        p = ld_cluster_u64(at);
        r = ld_cluster_u64(at + 8);
      } else {
        p = s.slot[turn][0], r = s.slot[turn][1];
      }
      rx = maximum ? (p > rx ? p : rx) : rx + p;
      ry += r;
    }
    turn ^= 1;
  };

  // the first of the order, and what is no number
  u64 best = 0, bad = 0;
  for (int step = step0; step < step1; ++step) {
    float x[V];
    load(step, x);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      bad += !(x[j] < __uint_as_float(0x7f800000u));
      const u64 c = (u64)key_of(x[j]) << 32 | (0xffffffffu - (uint32_t)((step * 32 + lane) * V + j));
      best = c > best ? c : best;
    }
  }
  reduce(best, bad, true, best, bad);
  const float top = value_of((uint32_t)(best >> 32));
  const float u = a.u[b], t = a.temperature ? a.temperature[b] : 1.f, p = a.top_p ? a.top_p[b] : 1.f, mp = a.min_p ? a.min_p[b] : 0.f;
  const int k = a.top_k ? a.top_k[b] : 0;
  const float inf = __uint_as_float(0x7f800000u);
  if (bad || !(top > -inf) || !(u >= 0.f && u < 1.f) || !(t < inf) || p != p || mp != mp) {
    if (rank == 0 && tid == 0) {
      a.tokens[b] = -1;
      if (a.log_probs) a.log_probs[b] = -inf;
    }
    barrier();   // (nobody leaves while its slot is read)
    return;
  }
  if (t < 0x1p-20f) {
    if (rank == 0 && tid == 0) {
      a.tokens[b] = (int)(0xffffffffu - (uint32_t)best);
      if (a.log_probs) a.log_probs[b] = 0.f;
    }
    barrier();
    return;
  }
  Weigher weigh;
  weigh.set(top, (double)t);

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
          if (key > above && (key & mask) == prefix && (step * 32 + lane) * V + j < a.vocab) {
            const u64 w = weights ? weigh(x[j], s.table) : 1ull;
            if (w) atomicAdd(&hist[(key >> shift) & 255u], w);
          }
        }
      }
      barrier();
      if (tid < 256) {
        u64 n = 0;
        for (int i = 0; i < ranks; ++i) n += ranks > 1 ? ld_cluster_u64(mapa_shared(smem_u32(&hist[tid]), (uint32_t)i)) : hist[tid];
        s.sums[tid] = n;
      }
      __syncthreads();
      if (warp == 0) {
        // lane i holds bins 255 - 8i .. 248 - 8i, from the first of the order down
        u64 n[8], sum = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          n[q] = s.sums[255 - 8 * lane - q];
          sum += n[q];
        }
        u64 before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const u64 up = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += up;
        }
        before -= sum;
        if (before < target && before + sum >= target) {
          bool found = false;
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            if (!found && before + n[q] >= target) {
              s.sel_bin = (uint32_t)(255 - 8 * lane - q);
              s.sel_left = target - before;
              found = true;
            }
            before += n[q];
          }
        }
      }
      __syncthreads();
      prefix |= s.sel_bin << shift;
      mask |= 255u << shift;
      target = s.sel_left;
      turn ^= 1;
    }
    left = target;
    return prefix;
  };

  // The border: tokens of keys above it stay, and of those with its key the first `ties`.
  uint32_t border = 0u;   // (below every key)
  u64 ties = 0ull;
  if (k > 0 && k < a.vocab) border = select((u64)k, 0u, false, ties);
  if (p < 1.f) {
    u64 all = 0, none;
    for (int step = step0; step < step1; ++step) {
      float x[V];
      load(step, x);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (key_of(x[j]) > border) all += weigh(x[j], s.table);
    }
    reduce(all, 0ull, false, all, none);
    const u64 one = ties ? weigh(value_of(border), s.table) : 0ull;
    const u64 want = max(1ull, p > 0.f ? times_fraction(all + ties * one, p, true) : 0ull);
    u64 left;
    if (want <= all) {
      border = select(want, border, true, left);
      const u64 w = weigh(value_of(border), s.table);
      ties = (left + w - 1) / w;
    } else {   // the tokens that top-k left at its border
      ties = min(ties, (want - all + one - 1) / max(one, 1ull));
    }
  }
  if (mp > 0.f) {
    const double least = (double)top + (double)t * log((double)fminf(mp, 1.f));
    float f = (float)least;
    if ((double)f < least) f = nextafterf(f, inf);
    const uint32_t key = key_of(f);
    if (key > border) {
      border = key - 1u;
      ties = 0ull;
    }
  }

  // What stays, summed by warps' runs.
  const u64 one = ties ? weigh(value_of(border), s.table) : 0ull;
  u64 sum = 0, equal = 0;
  for (int step = step0; step < step1; ++step) {
    float x[V];
    load(step, x);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint32_t key = key_of(x[j]);
      if (key > border) sum += weigh(x[j], s.table);
      equal += key == border && (step * 32 + lane) * V + j < a.vocab;
    }
  }
  u64 all, all_equal;
  reduce(sum, equal, false, all, all_equal);
  sum = warp_sum_u64(sum);
  equal = warp_sum_u64(equal);
  const u64 total = all + min(ties, all_equal) * one;
  const u64 at = times_fraction(total, u, false);   // the token's run of the sum holds this
  // before this warp's run: the ranks before, the warps before
  u64 before = 0, equal_before = 0;
  for (int i = 0; i < rank; ++i) {
    const uint32_t from = mapa_shared(smem_u32(&s.slot[turn ^ 1][0]), (uint32_t)i);
    before += ld_cluster_u64(from);
    equal_before += ld_cluster_u64(from + 8);
  }
  for (int i = 0; i < warp; ++i) before += s.warp_a[i], equal_before += s.warp_b[i];
  auto upto = [&](u64 w, u64 n) { return w + min(ties, n) * one; };
  if (upto(before, equal_before) <= at && at < upto(before + sum, equal_before + equal)) {
    for (int step = step0; step < step1; ++step) {
      float x[V];
      load(step, x);
      u64 w = 0, n = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const uint32_t key = key_of(x[j]);
        if (key > border) w += weigh(x[j], s.table);
        n += key == border && (step * 32 + lane) * V + j < a.vocab;
      }
      u64 wi = w, ni = n;   // up to and with this lane
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 wu = __shfl_up_sync(0xffffffffu, wi, o), nu = __shfl_up_sync(0xffffffffu, ni, o);
        if (lane >= o) wi += wu, ni += nu;
      }
      const bool there = upto(before + wi, equal_before + ni) > at;
      const unsigned mask = __ballot_sync(0xffffffffu, there);
      if (mask) {
        if (lane == __ffs(mask) - 1) {
          u64 c = before + wi - w, e = equal_before + ni - n;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const uint32_t key = key_of(x[j]);
            const int i = (step * 32 + lane) * V + j;
            const u64 was = upto(c, e);
            if (key > border) c += weigh(x[j], s.table);
            e += key == border && i < a.vocab;
            if (was <= at && upto(c, e) > at) {
              a.tokens[b] = i;
              if (a.log_probs) a.log_probs[b] = (float)(((double)x[j] - (double)top) / (double)t - log((double)total * 0x1p-43));
            }
          }
        }
        break;
      }
      before += __shfl_sync(0xffffffffu, wi, 31);
      equal_before += __shfl_sync(0xffffffffu, ni, 31);
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
  return launch_kernel_cluster(dt == DT_BF16 ? draw_kernel<bf16> : draw_kernel<float>, dim3(ranks, a.batch), dim3(kThreads), 0, st,
                               dim3(ranks, 1, 1), a);
}

}  // namespace ravel
