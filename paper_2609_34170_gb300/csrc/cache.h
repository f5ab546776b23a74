// Internal launch API of the 8-bit context cache (host side).  Every launcher
// enqueues on `st` and returns the launch's cudaError_t.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace ravel {

constexpr int kCacheBlock = 16;      // tokens that share an exponent
constexpr int kCacheRound = 128;     // capacities are whole multiples of this, so that tiles stay inside
constexpr int kCacheExpMin = -100;   // least exponent of a block

// One layer of a cache: rows of hdp bytes, [B][Hkv][T][hdp], exponents
// [B][Hkv][T / 16].  T: the capacity rounded up to kCacheRound.
struct CacheLayer {
  uint8_t *k, *v;
  int8_t *ke, *ve;
  int Hkv, hd, hdp, T;
};

struct AppendArgs {
  CacheLayer c;
  const void *k, *v;
  long long robot, token;   // strides in elements
  int batch, n, max_tokens;
  const int *starts, *counts;
  int vec;                  // rows are 16-byte aligned
  int* err;
};
cudaError_t launch_cache_append(const AppendArgs& a, Dtype dt, cudaStream_t st);

struct ReadArgs {
  CacheLayer c;
  int batch, n, max_tokens;
  const int *firsts, *lengths;
  void *k, *v;
  int vec;
  int* err;
};
cudaError_t launch_cache_read(const ReadArgs& a, Dtype dt, cudaStream_t st);

struct EvictArgs {
  CacheLayer from, to;
  int batch, keep, sinks, recent, max_tokens;
  const int* lengths;
  const float* mass;
  long long mass_stride;
  int *new_lengths, *index;
  float* new_mass;
  int* err;
};
cudaError_t launch_cache_evict(const EvictArgs& a, cudaStream_t st);

// A layer's codes as tensor maps (host memory): boxes for the tensor cores' tiles and for
// the units of the kernel for few rows.
struct CacheMaps {
  CUtensorMap k_tc, v_tc, k_rows, v_rows;
};
cudaError_t encode_layer(CacheMaps* m, const CacheLayer& c, int batch);

// Division by a number that stays the same over a launch, of n < 2^31: with 2^shift >= d and
// mul = 2^(31 + shift) / d rounded up, whose excess times n stays below 2^(31 + shift), the
// quotient is n * mul / 2^(31 + shift).  (An item of the prompts' kernel takes ten of them: as
// divisions, one of 64 bits among them, 2000 cycles.)
struct LaunchDiv {
  uint32_t d, mul;
  int shift;
  LaunchDiv() : LaunchDiv(1) {}
  explicit LaunchDiv(int by) : d((uint32_t)by), shift(0) {
    while ((1ull << shift) < d) ++shift;
    mul = (uint32_t)(((1ull << (31 + shift)) + d - 1) / d);
  }
#ifdef __CUDACC__
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return (uint32_t)((uint64_t)n * mul >> (31 + shift)); }
#endif
};

struct CacheAttnArgs {
  CacheLayer c;
  const CacheMaps* maps;
  const void* q;
  void* out;
  long long q_robot, q_token, out_robot, out_token;
  const int *lengths, *counts;
  int batch, n, G, max_length;
  LaunchDiv by_G, by_heads;   // by G, by the KV heads
  int causal, window, sinks;
  float scale_log2;         // softmax scale * log2(e)
  float* mass;
  long long mass_stride;
  int mass_add;
  int vec;                  // q rows are 16-byte aligned
  int num_sms;
  const int* clusters;      // clusters of that many (up to 8) tensor-core CTAs that the device holds at once
  // workspace
  float* part;              // [units * splits][rows of a tile x hdp] normalised partial outputs
  float2* part_ml;          // [units * splits][rows of a tile] (max, sum)
  unsigned* arrived;        // [units] splits that have finished (zero between launches)
  float2* row_ml;           // [B][Hkv][n * G] see row_weight, written where mass is wanted
  float* mass_ws;           // the mass's sums by chunk, or scores kept for it
  size_t mass_ws_bytes;
  uint8_t* q_ws;            // per SM, 128 bytes per row (of 128) and 64 dims: an item's laid out Q
  int* err;
  // chosen by the launcher
  int row_tiles, splits;
  LaunchDiv by_splits, by_group, by_last, by_pairs;   // tensor cores: of items, see there
  long long mass_pitch;     // tokens of a chunk's sums, or of a row's scores
  float* scores;            // few rows: scores kept for the mass, or null
  int b0, i0, i1;           // few rows: this launch's first robot, its queries i0 .. i1 - 1
  int group;                // tensor cores: (robot, KV head) pairs walked together
};
constexpr int kCacheSplitCtas = 608;   // row tiles (of 16) x splits of a launch that splits the tokens
constexpr int kCacheTcRows = 128;      // rows of a tile on the tensor cores: at most one such tile x split per SM
cudaError_t launch_cache_attend(const CacheAttnArgs& a, Dtype dt, cudaStream_t st);
cudaError_t launch_cache_attend_tc(const CacheAttnArgs& a, cudaStream_t st);   // bf16; not the mass
cudaError_t launch_cache_mass_tc(CacheAttnArgs a, cudaStream_t st);   // bf16, after the attention
// rows: query rows per KV head of which scores may be kept; G: query heads per KV head
size_t cache_mass_ws_bytes(int heads, int Hkv, int G, long long rows, int T, int num_sms);
cudaError_t init_cache_mass_tc_kernels();
cudaError_t init_cache_kernels();
cudaError_t init_cache_tc_kernels(int hdp, int* clusters);   // clusters: [9]

}  // namespace ravel
