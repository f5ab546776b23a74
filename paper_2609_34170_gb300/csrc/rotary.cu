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

constexpr int kTable = 2048;   // cosines and sines of a CTA's tokens

// A CTA takes a run of tokens with all their heads.  It computes their cosines and sines into shared
// memory once and then streams the heads through: a thread turns one vector of V values
// (interleaved: V / 2 pairs side by side; V 1: one pair) or two (half layout: V pairs, a vector from
// either half) per turn, kAhead rows of heads at a time.  threadIdx.x: the vector's place in the head, of
// the dims that turn and, where out is not x, of those that stay.  Nothing but bytes bounds it for many
// tokens; for few a launch, a load and the sines.  Measured: 816 tokens of 16 robots, 9 of 10 heads of 256 in
// bf16, half layout, 120 MB, 20.9 us (5.8 TB/s; two turns' vectors on their way 24.6, four 34); 65536 tokens of
// 20 heads of 64 in fp32, 32 dims interleaved, 671 MB, 98 us (6.8 TB/s; one turn's 102).  With the sines in
// registers, a thread taking one head after another, 25.8 and 124 to 144.
template <typename T, int V, bool IL>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs a, int tokens, LaunchDiv by_heads) {
  constexpr int P = IL ? (V + 1) / 2 : V;
  constexpr bool kTwo = !IL || V == 1;
  constexpr int kAhead = kTwo ? 1 : 2;   // two vectors on their way to a thread: more cost more CTAs than they hide
  constexpr int kVec = P % 2 == 0 ? 2 : 1;   // pairs to an access of the table
  __shared__ __align__(16) float2 cs[kTable];   // [token][P / kVec][place][kVec]: lanes side by side
  const int b = blockIdx.y, half = a.r.dims / 2, turning = half / P;
  const int threads = blockDim.x * blockDim.y, tid = threadIdx.y * blockDim.x + threadIdx.x;
  pdl_trigger();
  pdl_wait();
  int count = min(a.counts ? a.counts[b] : a.n, a.n);
  if (a.room > 0) {
    const int first = a.starts ? a.starts[b] : 0;
    if (first < 0 || (a.counts && a.counts[b] > a.n) || first > a.room - count) count = 0;
  }
  const int i0 = blockIdx.x * tokens, here = min(tokens, count - i0);
  if (here <= 0) return;
  const long long start = (a.starts ? (long long)a.starts[b] : 0ll) + i0;
  const int on_token = threads / half, on_pair = threads - on_token * half;
  for (int token = tid / half, pair = tid - token * half; token < here;) {
    const long long position = a.positions ? a.positions[(long long)b * a.n + i0 + token] : start + token;
    const int place = pair / P, j = pair - place * P;   // (P is a power of two)
    cs[token * half + (j / kVec * turning + place) * kVec + j % kVec] = turn_of(a.r.f[pair], position, a.r.amplitude);
    token += on_token, pair += on_pair;
    if (pair >= half) pair -= half, ++token;
  }
  __syncthreads();
  const bool stays = (int)threadIdx.x >= turning;
  // dims of the two vectors (interleaved: of one, or of V 1 of both values)
  const int d0 = stays ? a.r.dims + ((int)threadIdx.x - turning) * V : IL ? 2 * P * (int)threadIdx.x : P * (int)threadIdx.x;
  const int d1 = stays ? d0 : IL ? (V == 1 ? d0 + 1 : d0) : d0 + half;
  const T* x = (const T*)a.x + (long long)b * a.x_robot + (long long)i0 * a.x_token;
  T* out = (T*)a.out + (long long)b * a.out_robot + (long long)i0 * a.out_token;
  const int rows = here * a.heads;   // (below 2^31: at most 2048 tokens of 65535 heads)
  for (int row0 = threadIdx.y; row0 < rows; row0 += kAhead * blockDim.y) {
    Piece<T, V> u[kAhead], w[kAhead];
    int token[kAhead], head[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int row = row0 + k * blockDim.y;
      token[k] = (int)by_heads.of((uint32_t)row);
      head[k] = row - token[k] * a.heads;
      if (row < rows) {
        const T* from = x + (long long)token[k] * a.x_token + head[k] * a.hd;
        u[k] = load_piece<T, V>(from + d0);
        if (kTwo && !stays) w[k] = load_piece<T, V>(from + d1);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (row0 + k * (int)blockDim.y >= rows) break;
      T* to = out + (long long)token[k] * a.out_token + head[k] * a.hd;
      if (!stays) {
        float2 t[P];
#pragma unroll
        for (int j = 0; j < P; j += kVec) {
          const float2* at = &cs[token[k] * half + (j / kVec * turning + threadIdx.x) * kVec];
          if constexpr (kVec == 2) {
            const float4 v = *(const float4*)at;
            t[j] = make_float2(v.x, v.y), t[j + 1] = make_float2(v.z, v.w);
          } else {
            t[j] = *at;
          }
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
          T& first = kTwo ? u[k].v[j] : u[k].v[2 * j % V];
          T& second = kTwo ? w[k].v[j] : u[k].v[(2 * j + 1) % V];
          const float p = to_f32(first), q = to_f32(second);
          first = from_f32<T>(turned(p, q, t[j], true));
          second = from_f32<T>(turned(q, p, t[j], false));
        }
        if constexpr (kTwo) store_piece<T, V>(to + d1, w[k]);
      }
      store_piece<T, V>(to + d0, u[k]);
    }
  }
}

template <typename T, int V, bool IL>
cudaError_t launch_v(const RotaryArgs& a, cudaStream_t st) {
  constexpr int P = IL ? (V + 1) / 2 : V;
  const int places = a.r.dims / 2 / P + (a.x == a.out ? 0 : (a.hd - a.r.dims) / V), across = 256 / places;
  // tokens of a CTA: as many as the table holds, as give each thread four turns, as fill the SMs
  int tokens = std::min(a.n, kTable / (a.r.dims / 2));
  tokens = (int)std::min((long long)tokens, std::max(1ll, (long long)across * 4 / a.heads));
  tokens = (int)std::min((long long)tokens, std::max(1ll, (long long)a.batch * a.n / (2 * a.num_sms)));
  const int deep = (int)std::min((long long)across, (long long)tokens * a.heads);
  const dim3 grid((a.n + tokens - 1) / tokens, a.batch);
  const Overlap overlap;
  return launch_kernel(rotary_kernel<T, V, IL>, grid, dim3(places, deep), 0, st, 1, a, tokens, LaunchDiv(a.heads));
}

template <typename T, bool IL>
cudaError_t launch_t(const RotaryArgs& a, cudaStream_t st) {
  // vectors of V values must be whole and aligned in what turns and in what stays
  auto fits = [&](int v) {
    return a.align % (v * sizeof(T)) == 0 && (IL ? a.r.dims : a.r.dims / 2) % v == 0 && a.hd % v == 0;
  };
  constexpr int V16 = 16 / sizeof(T);
  if (fits(V16)) return launch_v<T, V16, IL>(a, st);
  if (fits(V16 / 2)) return launch_v<T, V16 / 2, IL>(a, st);
  return launch_v<T, 1, IL>(a, st);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, Dtype dt, cudaStream_t st) {
  if (a.r.interleaved) return dt == DT_BF16 ? launch_t<bf16, true>(a, st) : launch_t<float, true>(a, st);
  return dt == DT_BF16 ? launch_t<bf16, false>(a, st) : launch_t<float, false>(a, st);
}

}  // namespace ravel
