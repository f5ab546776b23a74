// Rotary positions of rows of heads.
#include <algorithm>

#include "launch.h"
#include "rotary.cuh"

namespace ravel {
namespace {

template <typename T, int V>
struct Piece {
  T v[V];
};
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> load_piece(const T* p) {
  Piece<T, V> r;
  if constexpr (V * sizeof(T) == 16) {
    const uint4 w = *(const uint4*)p;
    memcpy(&r, &w, 16);
  } else if constexpr (V * sizeof(T) == 8) {
    const uint2 w = *(const uint2*)p;
    memcpy(&r, &w, 8);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = p[i];
  }
  return r;
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, V>& r) {
  if constexpr (V * sizeof(T) == 16) {
    uint4 w;
    memcpy(&w, &r, 16);
    *(uint4*)p = w;
  } else if constexpr (V * sizeof(T) == 8) {
    uint2 w;
    memcpy(&w, &r, 8);
    *(uint2*)p = w;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = r.v[i];
  }
}

// A thread holds the cosines and sines of V pairs of one token and turns them in one head after
// another: two vectors of V values in, two out.  threadIdx.x: the pairs' place, or beyond them V
// of the dims that stay (copied where out is not x); threadIdx.y: the token; blockIdx.z: a run of
// heads.  Nothing but bytes bounds it for many tokens, and a launch, one load and V sines one
// after another for few.
template <typename T, int V, bool IL>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs a, int heads_per) {
  const int i = blockIdx.x * blockDim.y + threadIdx.y, b = blockIdx.y;
  const int half = a.r.dims / 2, d = threadIdx.x * V;   // first pair, or past them a dim
  unsigned long long f[V];   // (the table is constant: it may be read ahead of the wait)
#pragma unroll
  for (int j = 0; j < V; ++j) f[j] = d < half ? a.r.f[d + j] : 0ull;
  pdl_trigger();
  pdl_wait();
  const int count = a.counts ? a.counts[b] : a.n;
  if (i >= a.n || i >= count) return;
  const int h0 = blockIdx.z * heads_per, h1 = min(h0 + heads_per, a.heads);
  const T* x = (const T*)a.x + (long long)b * a.x_robot + (long long)i * a.x_token;
  T* out = (T*)a.out + (long long)b * a.out_robot + (long long)i * a.out_token;
  if (d >= half) {
    const int at = a.r.dims + d - half;
#pragma unroll 4
    for (int h = h0; h < h1; ++h) store_piece<T, V>(out + (long long)h * a.hd + at, load_piece<T, V>(x + (long long)h * a.hd + at));
    return;
  }
  const long long position = a.positions ? a.positions[(long long)b * a.n + i] : (a.starts ? (long long)a.starts[b] : 0ll) + i;
  float2 cs[V];
#pragma unroll
  for (int j = 0; j < V; ++j) cs[j] = turn_of(f[j], position, a.r.amplitude);
  const int p0 = IL ? 2 * d : d, p1 = IL ? 2 * d + V : d + half;
#pragma unroll 4
  for (int h = h0; h < h1; ++h) {
    const T* row = x + (long long)h * a.hd;
    const Piece<T, V> u = load_piece<T, V>(row + p0), w = load_piece<T, V>(row + p1);
    Piece<T, V> y, z;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if constexpr (IL) {
        // values 2j, 2j + 1 of the two vectors together
        const float p = to_f32(2 * j < V ? u.v[2 * j % V] : w.v[2 * j % V]);
        const float q = to_f32(2 * j + 1 < V ? u.v[(2 * j + 1) % V] : w.v[(2 * j + 1) % V]);
        const T r0 = from_f32<T>(turned(p, q, cs[j], true)), r1 = from_f32<T>(turned(q, p, cs[j], false));
        (2 * j < V ? y : z).v[2 * j % V] = r0;
        (2 * j + 1 < V ? y : z).v[(2 * j + 1) % V] = r1;
      } else {
        const float p = to_f32(u.v[j]), q = to_f32(w.v[j]);
        y.v[j] = from_f32<T>(turned(p, q, cs[j], true));
        z.v[j] = from_f32<T>(turned(q, p, cs[j], false));
      }
    }
    T* to = out + (long long)h * a.hd;
    store_piece<T, V>(to + p0, y);
    store_piece<T, V>(to + p1, z);
  }
}

template <typename T, int V>
cudaError_t launch_v(const RotaryArgs& a, cudaStream_t st) {
  const int stay = a.x == a.out ? 0 : a.hd - a.r.dims;
  const int places = (a.r.dims / 2 + stay) / V;
  const int tokens = std::max(1, std::min(a.n, 256 / places));
  // as many heads to a thread as leave every SM 1024 threads: each run of heads computes its own sines
  const long long all = (long long)a.batch * a.n * places * a.heads;
  const int per = (int)std::min((long long)a.heads, std::max(1ll, all / ((long long)a.num_sms * 1024)));
  const dim3 grid((a.n + tokens - 1) / tokens, a.batch, (a.heads + per - 1) / per);
  const Overlap overlap;
  return launch_kernel(a.r.interleaved ? rotary_kernel<T, V, true> : rotary_kernel<T, V, false>, grid, dim3(places, tokens), 0, st,
                       1, a, per);
}

template <typename T>
cudaError_t launch_t(const RotaryArgs& a, cudaStream_t st) {
  // V pairs per thread: vectors of V values must be whole and aligned in both halves and in what stays
  auto fits = [&](int v) {
    return a.align % (v * sizeof(T)) == 0 && (a.r.dims / 2) % v == 0 && a.hd % v == 0;
  };
  constexpr int V16 = 16 / sizeof(T);
  if (fits(V16)) return launch_v<T, V16>(a, st);
  if (fits(V16 / 2)) return launch_v<T, V16 / 2>(a, st);
  return launch_v<T, 1>(a, st);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, Dtype dt, cudaStream_t st) {
  return dt == DT_BF16 ? launch_t<bf16>(a, st) : launch_t<float>(a, st);
}

}  // namespace ravel
