// Internal launch API of what a decode step needs beside the context cache
// (host side): rotary positions, products with 4-bit weights, drawing tokens.
// Every launcher enqueues on `st` and returns the launch's cudaError_t.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "cache.h"
#include "kernels.h"

namespace ravel {

// Angles as whole numbers: `f` holds f_i / (2 pi) of a turn in units of 2^-64, so that
// position * f[i], modulo 2^64, is the fraction of a turn, whatever the position.
struct RotaryTable {
  const unsigned long long* f;   // device [dims / 2]
  int dims, interleaved;
  float amplitude;
};

struct RotaryArgs {
  RotaryTable r;
  const void* x;
  void* out;
  long long x_robot, x_token, out_robot, out_token;   // strides in elements
  int batch, n, heads, hd;
  const int *starts, *positions, *counts;
  int align;   // largest power of two, up to 16, that divides every row's address and stride in bytes
  int num_sms;
  int room;    // > 0: a robot whose count is not 0 .. n or whose tokens from starts on would pass `room` is left out
};
cudaError_t launch_rotary(const RotaryArgs& a, Dtype dt, cudaStream_t st);

struct AppendRotaryArgs {
  CacheLayer c;
  RotaryTable r;
  const void *q, *k, *v;
  void* q_out;
  long long q_robot, q_token, qo_robot, qo_token, k_robot, k_token, v_robot, v_token;
  int batch, n, G, max_tokens;
  const int *starts, *positions, *counts;
  int kv_vec, q_vec;   // rows of k and v, of q and q_out are 16-byte aligned
  int q_align, num_sms;   // as RotaryArgs, of q and q_out
  int* err;
};
cudaError_t launch_cache_append_rotary(const AppendRotaryArgs& a, Dtype dt, cudaStream_t st);

// A matrix of 4-bit weights in the order in which the tensor cores' fragments
// take it (w4.cu): tiles of 16 rows, blocks of 64 columns.
constexpr int kPadGroups = 8;
struct W4Matrix {
  uint4* codes;       // [tiles][kblocks][32 lanes]
  uint2* sz;          // [tiles][groups][8]: (scale, 128 + zero) of rows g and g + 8; kPadGroups groups of zeros behind
  int N, K, group;
  int tiles, kblocks, groups;   // tiles: an even number
  W4Matrix() = default;
  W4Matrix(int n, int k, int g)
      : codes(nullptr), sz(nullptr), N(n), K(k), group(g), tiles((n + 31) / 32 * 2), kblocks((k + 63) / 64), groups((k + g - 1) / g) {}
};
// Which kernel takes a product.
enum W4Kernel { W4_FEW = 0 /* up to 8 tokens */, W4_TILES = 1 /* tiles of 16 */, W4_TC = 2 /* tcgen05, tiles of 32 or 64 */ };
// What a test sets for its thread's products of more than 8 aligned tokens (ravel_debug_w4); -1: by the rule.
inline int& w4_forced() {
  static thread_local int kernel = -1;
  return kernel;
}
// Launches of the tcgen05 kernel by this thread that are left to run with its tokens withheld (ravel_debug_w4_withhold).
inline int& w4_withheld() {
  static thread_local int launches = 0;
  return launches;
}
struct W4Args {
  W4Matrix w;
  const void* x;
  void* out;
  const float* bias;
  int M, lda, ldo, epi, out_bf16;
  int vec;            // rows of x are 16-byte aligned
  int num_sms;
  int* err;
  int withhold = 0;   // fault injection (tests): no tokens are loaded, so that bounded waits run out
};
W4Kernel w4_kernel(const W4Args& a);
cudaError_t launch_w4_gemm(const W4Args& a, cudaStream_t st);
cudaError_t launch_w4_load(const W4Matrix& w, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, cudaStream_t st);
cudaError_t launch_w4_read(const W4Matrix& w, void* out, int ldo, Dtype dt, cudaStream_t st);
cudaError_t launch_w4_quantize(const void* W, int N, int K, int ldw, Dtype dt, int group, uint8_t* codes, uint16_t* scales,
                               uint8_t* zeros, cudaStream_t st);
cudaError_t launch_w4_tc(const W4Args& a, cudaStream_t st);   // aligned rows of tokens, any number
cudaError_t init_w4_kernels();
cudaError_t init_w4_tc_kernels();

struct DrawArgs {
  const void* logits;
  int batch, vocab;
  long long row;
  const float *u, *temperature, *top_p, *min_p;
  const int* top_k;
  int* tokens;
  float* log_probs;
  int num_sms;
};
cudaError_t init_draw_kernels();
cudaError_t launch_draw(const DrawArgs& a, Dtype dt, cudaStream_t st);

}  // namespace ravel
