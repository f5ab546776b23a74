// Storing into the 8-bit context cache, reading it back and eviction by
// attention mass.
#include <algorithm>

#include "cache.cuh"
#include "launch.h"
#include "rotary.cuh"
#include "tc_common.cuh"

namespace ravel {
namespace {

// One block of 16 tokens of one robot and KV head, keys and values: thread t
// holds 16 values of each of token t / (hdp / 16) of the block.  `fresh` tokens
// bring new values in kx / vx; `stay` tokens are in the cache already, under
// the exponents ke_old / ve_old, and are rounded again where those rise.  kx / vx are the new
// values times 2^-UP.
struct BlockShared {
  int bad[kCacheBlock];      // the token has a value that is not finite
  uint32_t kmax, vmax;       // bits of the largest finite magnitudes
};

__device__ __forceinline__ bool finite_f(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

template <int UP>
__device__ __forceinline__ void store_block(BlockShared& s, float* kx, float* vx, bool fresh, bool stay,
                                            bool has_old, int token, const CacheLayer& c, size_t row, size_t block,
                                            int d) {
  if (threadIdx.x < kCacheBlock) s.bad[threadIdx.x] = 0;
  if (threadIdx.x == kCacheBlock) s.kmax = s.vmax = 0u;
  const int ke_old = has_old ? c.ke[block] : kCacheExpMin, ve_old = has_old ? c.ve[block] : kCacheExpMin;
  __syncthreads();
  float km = 0.f, vm = 0.f;
  if (fresh) {
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      ok = ok && finite_f(kx[i]) && finite_f(vx[i]);
      km = fmaxf(km, fabsf(kx[i]));
      vm = fmaxf(vm, fabsf(vx[i]));
    }
    if (!ok) s.bad[token] = 1;
  }
  __syncthreads();
  const bool bad = s.bad[token] != 0;
  uint32_t kb = __float_as_uint(fresh && !bad ? km : 0.f), vb = __float_as_uint(fresh && !bad ? vm : 0.f);
  kb = __reduce_max_sync(0xffffffffu, kb);
  vb = __reduce_max_sync(0xffffffffu, vb);
  if ((threadIdx.x & 31) == 0) {
    atomicMax(&s.kmax, kb);
    atomicMax(&s.vmax, vb);
  }
  __syncthreads();
  const int ke = max(block_exponent(s.kmax, UP), ke_old), ve = max(block_exponent(s.vmax, UP), ve_old);
  uint4 *kd = (uint4*)(c.k + row + d), *vd = (uint4*)(c.v + row + d);
  if (fresh) {
    const uint32_t nan4 = 0x7f7f7f7fu;
    *kd = bad ? make_uint4(nan4, nan4, nan4, nan4) : f32_to_e4m3x16(kx, exp2i(UP - ke));
    *vd = bad ? make_uint4(0u, 0u, 0u, 0u) : f32_to_e4m3x16(vx, exp2i(UP - ve));
  } else if (stay) {
    float x[16];
    if (ke != ke_old) {
      e4m3x16_to_f32(*kd, exp2i(max(ke_old - ke, -126)), x);   // (below 2^-126 all round to zero anyway)
      *kd = f32_to_e4m3x16(x, 1.f);
    }
    if (ve != ve_old) {
      e4m3x16_to_f32(*vd, exp2i(max(ve_old - ve, -126)), x);
      *vd = f32_to_e4m3x16(x, 1.f);
    }
  }
  if (threadIdx.x == 0) {
    c.ke[block] = (int8_t)ke;
    c.ve[block] = (int8_t)ve;
  }
}

// Bandwidth-bound for many tokens, latency for few (a launch, the loads, three
// barriers).  A CTA per block: its exponent needs the whole block's maximum
// before the first value is rounded, and 16 tokens x 16 values per thread hold
// it in registers, so the inputs are read once.  Measured (alone / in a chain, inputs then in
// L2): a token of 64 robots 4.3 / 2.2 us; 816 tokens of 16 robots (one KV head of 256), 20 MB,
// 8.2 / 4.6; 4096 of 64, 403 MB, 79 (5.1 TB/s).
template <typename T>
__global__ void __launch_bounds__(256) cache_append_kernel(AppendArgs a) {
  __shared__ BlockShared s;
  pdl_trigger();
  pdl_wait();
  const CacheLayer& c = a.c;
  const int b = blockIdx.z, h = blockIdx.y;
  const int start = a.starts ? a.starts[b] : 0, count = a.counts ? a.counts[b] : a.n;
  if (start < 0 || count < 0 || count > a.n || start > a.max_tokens - count) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && h == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  const int blk = start / kCacheBlock + blockIdx.x, end = start + count;
  if (count == 0 || blk * kCacheBlock >= end) return;
  const int tpt = c.hdp / 16;   // threads per token
  const int token = threadIdx.x / tpt, d = (threadIdx.x % tpt) * 16;
  const int pos = blk * kCacheBlock + token;
  const bool fresh = pos >= start && pos < end, stay = pos < start;
  float kx[16], vx[16];
  if (fresh) {
    const size_t at = (size_t)((long long)b * a.robot + (long long)(pos - start) * a.token) + (size_t)h * c.hd;
    load16((const T*)a.k + at, d, c.hd, a.vec, kx);
    load16((const T*)a.v + at, d, c.hd, a.vec, vx);
  }
  const size_t head = (size_t)b * c.Hkv + h;
  store_block<0>(s, kx, vx, fresh, stay, blk * kCacheBlock < start, token, c, (head * c.T + pos) * c.hdp,
              head * (c.T / kCacheBlock) + blk, d);
}

template <typename T>
__device__ __forceinline__ void store16(T* row, int d, int hd, int vec, const float* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int d8 = d + 8 * h;
    if (d8 >= hd) break;
    T y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = from_f32<T>(x[8 * h + i]);
    if (vec) {
      constexpr int NV = 8 * sizeof(T) / 16;
      uint4 w[NV];
      memcpy(w, y, sizeof y);
#pragma unroll
      for (int i = 0; i < NV; ++i) *((uint4*)(row + d8) + i) = w[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) row[d8 + i] = y[i];
    }
  }
}

// Where a token's cosine and sine of a pair lie: the w = 2^log pairs that a thread of Turned16 takes are
// half / w apart, so that threads side by side read side by side (with a thread's pairs side by side their reads
// fell into one bank: keys alone of 816 tokens of 16 robots, one head of 256, 14.6 us, so 11.9).
__device__ __forceinline__ int turn_log(const RotaryTable& r) {
  return r.interleaved ? (r.dims % 16 == 0 ? 3 : 0) : r.dims % 32 == 0 ? 4 : 0;
}
__device__ __forceinline__ int turn_at(int pair, int half, int log) { return (pair & ((1 << log) - 1)) * (half >> log) + (pair >> log); }

// 16 values of a row as they lie in memory (zeros from hd on): to be on their way while something else is done.
template <typename T>
struct Raw16 {
  uint4 w[sizeof(T)];
  __device__ __forceinline__ void load(const T* row, int d, int hd, int vec) {
    constexpr int NV = sizeof(T) / 2;   // of 8 values
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int d8 = d + 8 * h;
      T y[8];
      if (d8 < hd && !vec) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = row[d8 + i];
        memcpy(&w[h * NV], y, sizeof y);
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) w[h * NV + i] = d8 < hd ? *((const uint4*)(row + d8) + i) : make_uint4(0u, 0u, 0u, 0u);
      }
    }
  }
  __device__ __forceinline__ void values(float* x) const {
    T y[16];
    memcpy(y, w, sizeof y);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = to_f32(y[i]);
  }
};

// 16 values from dim d on of a row of heads, turned: loaded first, then (behind the cosines and sines cs of the
// token, see turn_at) turned.  The pair of a dim may be anywhere in the row where the halves are not whole multiples
// of 16: then both are loaded one by one.
template <typename T>
struct Turned16 {
  Raw16<T> own, other;
  __device__ __forceinline__ static int kind(int d, const RotaryTable& r) {
    return d >= r.dims ? 0 : r.interleaved && r.dims % 16 == 0 ? 1 : !r.interleaved && r.dims % 32 == 0 ? 2 : 3;
  }
  __device__ __forceinline__ void load(const T* row, int d, int hd, int vec, const RotaryTable& r) {
    const int of = kind(d, r), half = r.dims / 2;
    if (of < 3) own.load(row, d, hd, vec);
    if (of == 2) other.load(row, d < half ? d + half : d - half, hd, vec);
  }
  __device__ __forceinline__ void values(const T* row, int d, int hd, const RotaryTable& r, const float2* cs, float* x) const {
    const int of = kind(d, r), half = r.dims / 2;
    if (of < 3) own.values(x);
    if (of == 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 t = cs[i * (half >> 3) + d / 16];
        const float p = x[2 * i], q = x[2 * i + 1];
        x[2 * i] = turned(p, q, t, true);
        x[2 * i + 1] = turned(q, p, t, false);
      }
    } else if (of == 2) {
      const bool first = d < half;
      const int pair = first ? d : d - half;
      float z[16];
      other.values(z);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = turned(x[i], z[i], cs[i * (half >> 4) + pair / 16], first);
    } else if (of == 3) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = d + i;
        x[i] = at < hd ? to_f32(row[at]) : 0.f;
        if (at < r.dims) {
          const bool first = r.interleaved ? at % 2 == 0 : at < half;
          const int pair = r.interleaved ? at ^ 1 : first ? at + half : at - half;
          x[i] = turned(x[i], to_f32(row[pair]), cs[r.interleaved ? at / 2 : first ? at : at - half], first);
        }
      }
    }
  }
};

// cache_append_kernel with the keys turned on their way in and, by CTAs of their own, the G query heads of
// the KV head turned beside them.  A CTA's 16 tokens share one table of cosines and sines.  Keys alone of 816
// tokens of 16 robots, one head of 256: 11.3 us where cache_append_kernel takes 4.8, for one and a third rounds of
// CTAs (64 registers; 48 or 40 spill and cost more) that compute 2048 sines each before anything is stored.
template <typename T>
__global__ void __launch_bounds__(256) cache_append_rotary_kernel(AppendRotaryArgs a) {
  __shared__ BlockShared s;
  __shared__ float2 cs[kCacheBlock * 128];   // [token][pair]
  pdl_trigger();
  pdl_wait();
  const CacheLayer& c = a.c;
  const bool queries = (int)blockIdx.y >= c.Hkv;
  const int b = blockIdx.z, h = queries ? blockIdx.y - c.Hkv : blockIdx.y;
  const int start = a.starts ? a.starts[b] : 0, count = a.counts ? a.counts[b] : a.n;
  if (start < 0 || count < 0 || count > a.n || start > a.max_tokens - count) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) raise_error(a.err, ERR_SHAPE);
    return;
  }
  const int blk = start / kCacheBlock + blockIdx.x, end = start + count;
  if (count == 0 || blk * kCacheBlock >= end) return;
  const int half = a.r.dims / 2;
  const int p0 = max(blk * kCacheBlock, start), tokens = min((blk + 1) * kCacheBlock, end) - p0;   // the new ones here
  const int tpt = c.hdp / 16, log = turn_log(a.r);   // threads per token
  const int token = threadIdx.x / tpt, d = (threadIdx.x % tpt) * 16;
  const int pos = blk * kCacheBlock + token;
  const bool fresh = pos >= start && pos < end, stay = pos < start;
  const T* k = (const T*)a.k + (long long)b * a.k_robot + (long long)(pos - start) * a.k_token + (long long)h * c.hd;
  const T* v = (const T*)a.v + (long long)b * a.v_robot + (long long)(pos - start) * a.v_token + (long long)h * c.hd;
  Turned16<T> key;
  Raw16<T> value;
  if (!queries && fresh) {   // (on their way while the sines are computed)
    key.load(k, d, c.hd, a.kv_vec, a.r);
    value.load(v, d, c.hd, a.kv_vec);
  }
  const int on_t = blockDim.x / half, on_pair = blockDim.x - on_t * half;
  for (int t = threadIdx.x / half, pair = threadIdx.x - t * half; t < tokens;) {
    const long long position = a.positions ? a.positions[(long long)b * a.n + p0 - start + t] : (long long)p0 + t;
    cs[t * half + turn_at(pair, half, log)] = turn_of(a.r.f[pair], position, a.r.amplitude);
    t += on_t, pair += on_pair;
    if (pair >= half) pair -= half, ++t;
  }
  __syncthreads();
  if (queries) {
    // 16 dims of one head and token per turn.  A thread's 16 dims may be read by others as their pairs'
    // other halves, so where q is written in place a turn's heads are read before any is written.
    const int items = tokens * a.G * tpt;
    for (int i0 = 0; i0 < items; i0 += blockDim.x) {
      const int i = i0 + threadIdx.x;
      float x[16];
      T* to = nullptr;
      int at = 0;
      if (i < items) {
        const int th = i / tpt, t = th / a.G, g = th % a.G;
        at = (i % tpt) * 16;
        const long long tok = p0 - start + t, head_at = (long long)(h * a.G + g) * c.hd;
        const T* q = (const T*)a.q + (long long)b * a.q_robot + tok * a.q_token + head_at;
        Turned16<T> query;
        query.load(q, at, c.hd, a.q_vec, a.r);
        query.values(q, at, c.hd, a.r, cs + t * half, x);
        to = (T*)a.q_out + (long long)b * a.qo_robot + tok * a.qo_token + head_at;
      }
      __syncthreads();   // (blockDim.x is a whole number of heads: 16 threads per token, tpt to a head)
      if (to) store16(to, at, c.hd, a.q_vec, x);
    }
    return;
  }
  float kx[16], vx[16];
  if (fresh) {
    key.values(k, d, c.hd, a.r, cs + (pos - p0) * half, kx);
    value.values(vx);
  }
  const size_t head = (size_t)b * c.Hkv + h;
  store_block<0>(s, kx, vx, fresh, stay, blk * kCacheBlock < start, token, c, (head * c.T + pos) * c.hdp,
                 head * (c.T / kCacheBlock) + blk, d);
}

// Bandwidth-bound for many tokens, a launch and dependent loads for few: a thread takes 16
// values of a token's key row and of its value row.  Measured (one KV head of 256; alone / in a
// chain): 816 tokens of 16 robots, 20 MB, 6.8 / 5.4 us; 4096 of 64, 403 MB, 71 (5.7 TB/s).
template <typename T>
__global__ void __launch_bounds__(256) cache_read_kernel(ReadArgs a) {
  const CacheLayer& c = a.c;
  const int b = blockIdx.z, h = blockIdx.y;
  const int tpt = c.hdp / 16;
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  pdl_trigger();
  pdl_wait();
  const int i = (int)(idx / tpt), d = (int)(idx % tpt) * 16;
  if (i >= a.n || d >= c.hd) return;
  const int first = a.firsts ? a.firsts[b] : 0;
  const int length = a.lengths ? a.lengths[b] : a.max_tokens;
  const bool bad = first < 0 || length < 0 || length > a.max_tokens;
  if (bad && idx == 0 && h == 0) raise_error(a.err, ERR_SHAPE);
  const size_t head = (size_t)b * c.Hkv + h;
  float k[16], v[16];
  if (!bad && i < length - first) {
    const int pos = first + i;
    const size_t row = (head * c.T + pos) * c.hdp + d, block = head * (c.T / kCacheBlock) + pos / kCacheBlock;
    const uint4 kw = *(const uint4*)(c.k + row), vw = *(const uint4*)(c.v + row);
    e4m3x16_to_f32(kw, exp2i(c.ke[block]), k);
    e4m3x16_to_f32(vw, exp2i(c.ve[block]), v);
  } else {
#pragma unroll
    for (int q = 0; q < 16; ++q) k[q] = v[q] = 0.f;
  }
  const size_t out = (head * a.n + i) * c.hd;
  store16((T*)a.k + out, d, c.hd, a.vec, k);
  store16((T*)a.v + out, d, c.hd, a.vec, v);
}

// ---- eviction ---------------------------------------------------------------

constexpr int kSelThreads = 1024;
constexpr int kSelCluster = 8;      // CTAs of a head at most

__device__ __forceinline__ unsigned ld_cluster_u1(uint32_t a) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

// Order of masses as unsigned integers: ascending, -0 = +0, NaN above all.
__device__ __forceinline__ uint32_t mass_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// The tokens that one (robot, KV head) keeps: the key of the last one in by a radix
// selection over the middle's masses (up to four histograms of 8 bits), then one ordered
// pass that gives each kept token its place.  Ties go to the earlier tokens.  No order
// of arrival enters the result: the histograms count.
//
// A cluster per (robot, KV head), each of its CTAs with a run of the tokens; the
// histograms and the counts are added up through distributed shared memory.  The
// masses are read up to six times (four histograms, the counts of the runs before, the
// places), from L2 after the first: one CTA took 66 us for 65537 tokens, 64 dependent turns of
// the loop per pass.  Measured: 4 heads of 65537 tokens 22 us (latency: three to four passes of
// loads, cluster barrier, remote reads and scan at 4 us), 64 robots of 816 tokens 7.6 us.
__global__ void __launch_bounds__(kSelThreads) cache_select_kernel(EvictArgs a, int ctas) {
  __shared__ unsigned hist[2][256], sums[256];
  __shared__ uint32_t sel_bin, sel_left, sel_all;
  __shared__ unsigned totals[2][32];
  __shared__ unsigned kept_here[2], before_here[2];   // surely in, ties: of this CTA's run, of the runs before it
  const int h = blockIdx.x / ctas, rank = blockIdx.x % ctas, b = blockIdx.y, Hkv = a.from.Hkv;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_trigger();
  pdl_wait();
  int len = a.lengths[b];
  if (len < 0 || len > a.max_tokens || len > a.mass_stride) {
    if (tid == 0 && blockIdx.x == 0) raise_error(a.err, ERR_SHAPE);
    len = 0;
  }
  const int kept = min(len, a.keep);
  const size_t head = (size_t)b * Hkv + h;
  const float* mass = a.mass + head * a.mass_stride;
  int* index = a.index + head * a.keep;
  float* nm = a.new_mass ? a.new_mass + head * a.keep : nullptr;
  if (tid == 0 && blockIdx.x == 0) a.new_lengths[b] = kept;
  for (int i = kept + rank * kSelThreads + tid; i < a.keep; i += ctas * kSelThreads) {
    index[i] = -1;
    if (nm) nm[i] = 0.f;
  }
  if (len <= a.keep) {   // (all of the cluster)
    for (int i = rank * kSelThreads + tid; i < kept; i += ctas * kSelThreads) {
      index[i] = i;
      if (nm) nm[i] = mass[i];
    }
    return;
  }
  const int lo = a.sinks, hi = len - a.recent;   // the middle, longer than what stays of it
  const int run = ((len + ctas - 1) / ctas + kSelThreads - 1) / kSelThreads * kSelThreads;
  const int r0 = min(rank * run, len), r1 = min(r0 + run, len);
  const int m0 = max(lo, r0), m1 = min(hi, r1);   // the middle's part of this run
  uint32_t left = (uint32_t)(a.keep - a.sinks - a.recent);
  uint32_t prefix = 0xffffffffu;   // (nothing of the middle stays: no key is above, no tie taken)
  if (left > 0) {
    prefix = 0u;
    uint32_t mask = 0u;
    int buf = 0;
    for (int shift = 24; shift >= 0; shift -= 8, buf ^= 1) {
      // (two histograms in turn: a CTA may still read this one's while its neighbours are at the next)
      if (tid < 256) hist[buf][tid] = 0u;
      __syncthreads();
      auto count = [&](float m) {
        const uint32_t key = mass_key(m);
        if ((key & mask) == prefix) atomicAdd(&hist[buf][(key >> shift) & 255u], 1u);
      };
      int j = m0 + tid;
      for (; j + 7 * kSelThreads < m1; j += 8 * kSelThreads) {
        float x[8];   // (all on their way together)
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = mass[j + q * kSelThreads];
#pragma unroll
        for (int q = 0; q < 8; ++q) count(x[q]);
      }
      for (; j < m1; j += kSelThreads) count(mass[j]);
      if (ctas > 1) cluster_sync();
      else __syncthreads();
      if (tid < 256) {
        unsigned n = 0;
        if (ctas > 1) {
          const uint32_t at = smem_u32(&hist[buf][tid]);
          unsigned x[kSelCluster];   // (all on their way together)
#pragma unroll
          for (int q = 0; q < kSelCluster; ++q) x[q] = ld_cluster_u1(mapa_shared(at, (uint32_t)min(q, ctas - 1)));
#pragma unroll
          for (int q = 0; q < kSelCluster; ++q) n += q < ctas ? x[q] : 0u;
        } else {
          n = hist[buf][tid];
        }
        sums[tid] = n;
      }
      __syncthreads();
      if (warp == 0) {
        // lane i holds bins 255 - 8i .. 248 - 8i, from the heaviest down
        unsigned n[8], sum = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          n[q] = sums[255 - 8 * lane - q];
          sum += n[q];
        }
        unsigned before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned up = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += up;
        }
        before -= sum;   // tokens in heavier lanes' bins
        if (before < left && before + sum >= left) {
          bool found = false;
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            if (!found && before + n[q] >= left) {
              sel_bin = (uint32_t)(255 - 8 * lane - q);
              sel_left = left - before;
              sel_all = n[q];
              found = true;
            }
            before += n[q];
          }
        }
      }
      __syncthreads();
      prefix |= sel_bin << shift;
      mask |= 255u << shift;
      left = sel_left;
      if (sel_all == left && prefix > 0u) {   // the whole bin stays: its least key, and no ties
        --prefix;
        left = 0;
        break;
      }
    }
  }
  // which tokens are surely in (heavier, first, last), and which are ties
  auto load = [&](int j) { return j < r1 ? mass[j] : 0.f; };
  auto kind = [&](int j, float m, bool& in, bool& tie) {
    const uint32_t key = mass_key(m);
    const bool always = j < r1 && (j < lo || j >= hi), mid = j >= m0 && j < m1;
    in = always || (mid && key > prefix);
    tie = mid && key == prefix;
  };
  unsigned sure = 0, ties = 0;
  if (ctas > 1) {   // of the runs before this one
    if (tid < 2) kept_here[tid] = 0u;
    __syncthreads();
    unsigned n0 = 0, n1 = 0;
#pragma unroll 4
    for (int j = r0 + tid; j < r1; j += kSelThreads) {
      bool in, tie;
      kind(j, load(j), in, tie);
      n0 += in;
      n1 += tie;
    }
    n0 = __reduce_add_sync(0xffffffffu, n0);
    n1 = __reduce_add_sync(0xffffffffu, n1);
    if (lane == 0) {
      atomicAdd(&kept_here[0], n0);
      atomicAdd(&kept_here[1], n1);
    }
    cluster_sync();
    if (tid < 2) {
      unsigned n = 0, x[kSelCluster];
#pragma unroll
      for (int q = 0; q < kSelCluster; ++q) x[q] = ld_cluster_u1(mapa_shared(smem_u32(&kept_here[tid]), (uint32_t)min(q, ctas - 1)));
#pragma unroll
      for (int q = 0; q < kSelCluster; ++q) n += q < rank ? x[q] : 0u;
      before_here[tid] = n;
    }
    __syncthreads();
    sure = before_here[0];
    ties = before_here[1];
  }
  // kept before j: those surely in and as many ties as still fit
  int buf = 0;
  auto place = [&](int j, float m) {   // (every thread; j from r1 on: nothing)
    bool in, tie;
    kind(j, m, in, tie);
    const unsigned bi = __ballot_sync(0xffffffffu, in), bt = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) totals[buf][warp] = __popc(bi) | __popc(bt) << 16;
    __syncthreads();
    const unsigned own = totals[buf][lane];
    unsigned pre = own;   // both counts in one word: at most 1024 each
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned up = __shfl_up_sync(0xffffffffu, pre, o);
      if (lane >= o) pre += up;
    }
    const unsigned all = __shfl_sync(0xffffffffu, pre, 31);
    const unsigned warps = __shfl_sync(0xffffffffu, pre - own, warp);
    const unsigned below = (1u << lane) - 1u;
    const unsigned s0 = sure + (warps & 0xffffu) + __popc(bi & below), t0 = ties + (warps >> 16) + __popc(bt & below);
    if (in || (tie && t0 < left)) {
      const unsigned at = s0 + min(t0, left);
      index[at] = j;
      if (nm) nm[at] = m;
    }
    sure += all & 0xffffu;
    ties += all >> 16;
    buf ^= 1;
  };
  int base = r0;
  for (; base + 3 * kSelThreads < r1; base += 4 * kSelThreads) {
    float m[4];   // (loads ahead of the turns' barriers)
#pragma unroll
    for (int q = 0; q < 4; ++q) m[q] = load(base + q * kSelThreads + tid);
#pragma unroll
    for (int q = 0; q < 4; ++q) place(base + q * kSelThreads + tid, m[q]);
  }
  for (; base < r1; base += kSelThreads) place(base + tid, load(base + tid));
  if (ctas > 1) cluster_sync();   // nobody leaves while its counts are read
}

// Values on their way from cache to cache are 2^kMoveUp below what they stand for: a finite one
// near fp32's largest is held as 2^128, which fp32 is not.
constexpr int kMoveUp = 8;

// The kept rows into the other cache: a CTA per block of 16, as in append.  Bound by the
// dependent loads (index, block exponent, row): 256 of 816 tokens of 64 robots 7.8 us for 17 MB.
__global__ void __launch_bounds__(256) cache_move_kernel(EvictArgs a) {
  __shared__ BlockShared s;
  const CacheLayer &from = a.from, &to = a.to;
  const int b = blockIdx.z, h = blockIdx.y;
  pdl_trigger();
  pdl_wait();
  const int kept = a.new_lengths[b];
  if ((int)blockIdx.x * kCacheBlock >= kept) return;
  const int tpt = to.hdp / 16;
  const int token = threadIdx.x / tpt, d = (threadIdx.x % tpt) * 16;
  const int pos = blockIdx.x * kCacheBlock + token;
  const size_t head = (size_t)b * to.Hkv + h;
  float kx[16], vx[16];
  const bool fresh = pos < kept;
  if (fresh) {
    const int j = a.index[head * a.keep + pos];
    const size_t row = (head * from.T + j) * from.hdp + d, block = head * (from.T / kCacheBlock) + j / kCacheBlock;
    const uint4 kw = *(const uint4*)(from.k + row), vw = *(const uint4*)(from.v + row);
    e4m3x16_to_f32(kw, exp2i(from.ke[block] - kMoveUp), kx);
    e4m3x16_to_f32(vw, exp2i(from.ve[block] - kMoveUp), vx);
  }
  store_block<kMoveUp>(s, kx, vx, fresh, false, false, token, to, (head * to.T + pos) * to.hdp,
              head * (to.T / kCacheBlock) + blockIdx.x, d);
}

}  // namespace

cudaError_t launch_cache_append(const AppendArgs& a, Dtype dt, cudaStream_t st) {
  // a start inside a block needs one block more
  const dim3 grid((a.n + 2 * kCacheBlock - 2) / kCacheBlock, a.c.Hkv, a.batch);
  const Overlap overlap;
  return launch_kernel(dt == DT_BF16 ? cache_append_kernel<bf16> : cache_append_kernel<float>, grid, dim3(a.c.hdp), 0, st, 1, a);
}

cudaError_t launch_cache_append_rotary(const AppendRotaryArgs& a, Dtype dt, cudaStream_t st) {
  // Queries of few tokens in the same launch: a token of 64 robots (8 query heads on one of 256) 2.9 us, turned and
  // stored by two calls 3.7.  Of many in one that streams them: 816 tokens of 16 robots 31 us (46 in one launch;
  // two calls, whose keys are rounded to bf16 in between, 27).  One launch / two, n tokens of 16 robots, 8 heads on one of 256: 1
  // 2.7 / 4.5 us, 4 3.9 / 4.6, 8 6.0 / 5.2, 16 10.3 / 6.4, 32 11.0 / 6.7; of 64 robots 4 5.5 / 5.4, 16 15.6 / 9.0; 16 robots
  // with 16 heads on 4 of 64: 8 3.7 / 4.8, 16 5.7 / 5.6, 32 6.2 / 6.3, 64 6.8 / 9.4.  (16 is right for the latter, late by half for
  // heads of 256 that share one KV head.)  (A grid has 65535 rows of CTAs, a cache up to as many heads.)
  const bool apart = a.q && (a.n > 16 || a.c.Hkv > 65535 / 2);
  if (apart) {
    RotaryArgs r{a.r, a.q, a.q_out, a.q_robot, a.q_token, a.qo_robot, a.qo_token, a.batch, a.n, a.c.Hkv * a.G, a.c.hd,
                 a.starts, a.positions, a.counts, a.q_align, a.num_sms, a.max_tokens};
    const cudaError_t e = launch_rotary(r, dt, st);
    if (e != cudaSuccess) return e;
  }
  const dim3 grid((a.n + 2 * kCacheBlock - 2) / kCacheBlock, a.q && !apart ? 2 * a.c.Hkv : a.c.Hkv, a.batch);
  const Overlap overlap;
  return launch_kernel(dt == DT_BF16 ? cache_append_rotary_kernel<bf16> : cache_append_rotary_kernel<float>, grid, dim3(a.c.hdp), 0,
                       st, 1, a);
}

cudaError_t launch_cache_read(const ReadArgs& a, Dtype dt, cudaStream_t st) {
  const dim3 grid((unsigned)(((long long)a.n * (a.c.hdp / 16) + 255) / 256), a.c.Hkv, a.batch);
  const Overlap overlap;
  return launch_kernel(dt == DT_BF16 ? cache_read_kernel<bf16> : cache_read_kernel<float>, grid, dim3(256), 0, st, 1, a);
}

cudaError_t launch_cache_evict(const EvictArgs& a, cudaStream_t st) {
  // a CTA per 4096 tokens, up to a cluster of 8 (at 816 tokens a cluster's barriers take longer than they save)
  const int ctas = (int)std::min((long long)kSelCluster, std::max(1ll, std::min((long long)a.max_tokens, a.mass_stride) / 4096));
  const Overlap overlap;
  cudaError_t e = launch_kernel_cluster(cache_select_kernel, dim3(a.from.Hkv * ctas, a.batch), dim3(kSelThreads), 0, st,
                                        dim3(ctas, 1, 1), a, ctas);
  if (e != cudaSuccess) return e;
  const dim3 grid((a.keep + kCacheBlock - 1) / kCacheBlock, a.to.Hkv, a.batch);
  return launch_kernel(cache_move_kernel, grid, dim3(a.to.hdp), 0, st, 1, a);
}

}  // namespace ravel
