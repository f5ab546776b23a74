// What the attention kernels of the 8-bit context cache share: which tokens a
// row (a query of one head) sees.
#pragma once

#include "cache.cuh"
#include "tc_common.cuh"

namespace ravel {

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// What a tile of rows sees: tokens [0, sink) and [from, to) in units, and the
// numbers that decide single tokens.
struct Sight {
  int len, count;     // the robot's tokens and queries
  int p0;             // position of query 0 (len - count)
  int sink_units, from, units;   // unit t is t < sink_units ? t : t - sink_units + from
};

struct RowMask {
  int hi, lo, sinks;   // sees j < hi and (j >= lo or j < sinks)
  __device__ __forceinline__ bool sees(int j) const { return j < hi && (j >= lo || j < sinks); }
  // tokens j .. j + 31 that it sees
  __device__ __forceinline__ uint32_t bits(int j) const { return below(hi - j) & (~below(lo - j) | below(sinks - j)); }
  // the lowest x bits
  static __device__ __forceinline__ uint32_t below(int x) { return x <= 0 ? 0u : (x >= 32 ? 0xffffffffu : (1u << x) - 1u); }
};

__device__ __forceinline__ RowMask row_mask(const CacheAttnArgs& a, const Sight& s, int r) {
  RowMask m;
  const int i = (int)a.by_G.of((uint32_t)r);
  m.sinks = a.sinks;
  m.lo = 0;
  if (i >= s.count) m.hi = 0;
  else if (!a.causal) m.hi = s.len;
  else {
    m.hi = s.p0 + i + 1;
    if (a.window > 0) m.lo = max(0, m.hi - a.window);
  }
  return m;
}

// The robot's length and count, checked; a robot out of range sees nothing.
__device__ __forceinline__ bool robot_sight(const CacheAttnArgs& a, int b, Sight& s) {
  s.len = a.lengths[b];
  s.count = a.counts ? a.counts[b] : a.n;
  const bool ok = s.len >= 0 && s.len <= a.max_length && s.count >= 0 && s.count <= a.n &&
                  (!a.causal || s.count <= s.len);
  if (!ok) s.len = s.count = 0;
  s.p0 = s.len - s.count;
  return ok;
}

// Units of `U` tokens that rows r0 .. r1 (r0 < count * G) see between them.
__device__ __forceinline__ void tile_sight(const CacheAttnArgs& a, Sight& s, int r0, int r1, int U) {
  const RowMask first = row_mask(a, s, r0), last = row_mask(a, s, min(r1, s.count * a.G - 1));
  s.from = first.lo / U;
  s.sink_units = a.window > 0 ? min((a.sinks + U - 1) / U, s.from) : 0;
  s.units = s.sink_units + (last.hi + U - 1) / U - s.from;
}

// 2^x for an integral x of at most 127, 2^-126 below -126 ...
__device__ __forceinline__ float pow2f(float x) { return exp2i(__float2int_rn(fmaxf(x, -126.f))); }
// ... and for the step from one reference to a larger one: from none (-inf) it is 0
__device__ __forceinline__ float pow2f_down(float x) { return x == -INFINITY ? 0.f : pow2f(x); }

// A block whose value exponent lies this far below the row's W - m (see the
// kernels) counts as if it did not: its P, then below 2^-45, leaves nothing in O
// and still counts in the sum.
constexpr float kVeBelow = 60.f;

// What an attention launch leaves per row for the mass: the weight of a score s
// (log2 domain) is 2^(s - x) * y; rows without a query or a token: (0, 0).
// sum: of 2^(s - max + shift).
__device__ __forceinline__ float2 row_weight(float max, float sum, float shift) {
  return make_float2(max == -INFINITY ? 0.f : max, !(sum <= 0.f) ? exp2f(shift) / sum : 0.f);
}

}  // namespace ravel
