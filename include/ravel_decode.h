/*
 * ravel_decode.h -- C ABI of what a VLM's decode step needs beside the context
 * cache (ravel_cache.h): rotary positions for queries and keys, on their own
 * or on the way into the cache, products of few rows with 4-bit weights, and
 * drawing a token from logits.
 *
 * Conventions beside those of ravel.h and ravel_cache.h:
 *  - Positions, counts and settings of a robot are device arrays, read by the
 *    kernels, so that calls can be captured into CUDA graphs.
 *  - Every call but the ones that create, destroy or load is enqueued on `stream`
 *    and returns.  Its launch may begin while the one before
 *    it on the stream ends, and waits for it before it reads or writes anything
 *    that is passed to the call.
 *  - A rotary table and loaded weights are not changed by the calls that use
 *    them, and these have no workspace: calls that share them may run at the same
 *    time, on several streams, from several threads and graphs.
 */
#ifndef RAVEL_DECODE_H_
#define RAVEL_DECODE_H_

#include "ravel.h"
#include "ravel_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions -------------------------------------------------------
 * Of the hd dims of a head the first `dims` turn in pairs, (i, i + dims / 2) or,
 * interleaved, (2i, 2i + 1), by the angle a = p f_i, p the token's position:
 *   (x, y) -> amplitude * (x cos a - y sin a, x sin a + y cos a)
 * The others stay.  p is any int32 (the transpose, which is also the gradient, is
 * the rotation by -p).  The table holds f_i / (2 pi), computed in 64-bit floats, and p times it is
 * reduced in 64-bit integers: an angle is off by no more than p times the table's rounding, f_i 2^-51 (of frequencies
 * between low and high their formula's): up to positions of 10^8 less than a rounding of fp32, in which everything else
 * is, 3e-7 at 2^31.  Results are rounded once.  Other rules for long contexts, a ramp over the dims' index say, are given as `frequencies`. */
typedef struct {
  int dims;             /* even, 2 to 256 */
  int interleaved;      /* 0: pairs (i, i + dims / 2); 1: pairs (2i, 2i + 1) */
  double base;          /* f_i = base^(-2i / dims); > 0 */
  double factor;        /* > 0: frequencies are divided by it (1: as they are) ... */
  double original_length; /* ... all of them (0), or with t = original_length f_i / (2 pi), the turns that a
                           frequency makes over that length: in full for t <= low, not at all for t >= high,
                           and in between f_i (g + (1 - g) / factor) with g = (t - low) / (high - low) */
  double low, high;     /* 0 <= low < high, read where original_length > 0 */
  double amplitude;     /* of the turned dims, finite in fp32 (1: lengths stay) */
  const double* frequencies; /* host [dims / 2] or NULL: the f_i themselves, in the place of base to high; given or made,
                           they are finite */
} ravel_rotary_config;

typedef struct ravel_rotary_ctx ravel_rotary_t;

/* Validate cfg and put the table of frequencies on `device`.  Synchronous. */
ravel_status ravel_rotary_create(const ravel_rotary_config* cfg, int device, ravel_rotary_t** out);

/* Free the table (after synchronising the device).  NULL is a no-op. */
void ravel_rotary_destroy(ravel_rotary_t* r);

/* Turn rows of heads.
 *   x, out     device [batch, n, heads, hd] of dtype; heads of a token are contiguous, token i of robot b
 *              begins at element b * robot_stride + i * token_stride.  out is x itself (with x's strides)
 *              or does not overlap it; its rows do not overlap each other: a robot's tokens lie before the next one's, or a
 *              token's robots before the next one's (rows that interleave in another way are refused).  Query and
 *              key heads that lie side by side are one call.
 *   batch, heads  up to 65535; n up to 2^30
 *   hd         dims to 256
 *   starts     device int32 [batch] or NULL (0): token i of robot b has position starts[b] + i ...
 *   positions  device int32 [batch, n] or NULL: ... or positions[b][i]
 *   counts     device int32 [batch] or NULL (n): tokens from counts[b] on are not written (a count below 0 is
 *              taken as 0, one above n as n) */
ravel_status ravel_rotary_apply(ravel_rotary_t* r, int batch, int n, int heads, int hd, int dtype, const void* x,
                                long long x_robot_stride, long long x_token_stride, void* out, long long out_robot_stride,
                                long long out_token_stride, const int* starts, const int* positions, const int* counts,
                                void* stream);

/* ravel_cache_append of keys turned to their positions, and the queries turned
 * with them, in one call.  Between a turned key and the cache nothing is rounded
 * but to the cache's own values.  (For prompts two calls, ravel_rotary_apply and ravel_cache_append, take less
 * time, 27 us for 816 tokens of 16 robots with 8 heads of 256 where this takes 31, and round keys to the cache's
 * type in between.)
 *   q, q_out   device [batch, n, Hq, hd] of the cache's dtype, or both NULL; q_out is q itself (with q's strides)
 *              or overlaps none of the others; its rows do not overlap each other (as above).  Hq * (hd rounded up to
 *              64) is at most 2^30
 *   k, v       as for ravel_cache_append, each with strides of its own; they are not written
 *   positions  device int32 [batch, n] or NULL: starts[b] + i
 *   starts, counts  as for ravel_cache_append; rows of q_out from counts[b] on are not written
 * The rotary table's dims are at most the cache's head_dim, its device is the cache's. */
ravel_status ravel_cache_append_rotary(ravel_cache_t* c, int layer, const ravel_rotary_t* r, int batch, int n, const void* q,
                                       long long q_robot_stride, long long q_token_stride, void* q_out,
                                       long long q_out_robot_stride, long long q_out_token_stride, const void* k,
                                       long long k_robot_stride, long long k_token_stride, const void* v,
                                       long long v_robot_stride, long long v_token_stride, const int* starts,
                                       const int* positions, const int* counts, void* stream);

/* ---- products with 4-bit weights -----------------------------------------------
 * Row n of a matrix W [N, K] holds for each k a code c of 0 .. 15 and for each group
 * of `group` ks a zero point z of 0 .. 15 and a bf16 scale s: w = (c - z) s.  Codes
 * come two to a byte (even k in the low nibble), [N, (K + 1) / 2]; scales and zeros
 * [N, (K + group - 1) / group].  Scales held in another type are rounded to bf16 by the caller: of an
 * fp16 scale that moves its group's weights by up to 2^-8 of their size, 0.06 of a step of the codes at most. */
typedef struct ravel_w4_ctx ravel_w4_t;

/* Allocate an N x K matrix (about N K / 2 + 4 N K / group bytes) on `device`, all zeros.
 * group is 32, 64 or 128; N and K are at least 1 and at most 2^24.  Synchronous. */
ravel_status ravel_w4_create(int N, int K, int group, int device, ravel_w4_t** out);

/* Free the matrix (after synchronising the device).  NULL is a no-op. */
void ravel_w4_destroy(ravel_w4_t* w);

/* Clear the error word of a matrix, after waiting for the device: a product of more than 8 rows in
 * which a bounded wait ran out (its output is not valid) makes later ones return RAVEL_ETIMEOUT. */
ravel_status ravel_w4_reset(ravel_w4_t* w);

/* Codes, scales and zeros (device, as above, contiguous) into the matrix, in the order
 * in which the products read them.  Scales are finite.  Waits until `stream` is done, because
 * products read weights ahead of their place on a stream; refused (RAVEL_EINVAL)
 * on a stream that is being captured.  No product may be running.  (20 us for 2560 x 1024, 72 for 8192 x 8192, 530 for
 * 65536 x 8192.) */
ravel_status ravel_w4_load(ravel_w4_t* w, const void* codes, const void* scales, const void* zeros, void* stream);

/* Nearest codes of a matrix: per row and group s = (max(w, 0) - min(w, 0)) / 15 in
 * bf16, z = -min(w, 0) / s and c = w / s + z, both rounded to nearest (ties to even)
 * and limited to 0 .. 15; a group of zeros has s = z = c = 0.  For values of
 * up to 3e38 (codes of a larger one may stand for more than fp32 holds).  (160 us for 8192 x 8192 in bf16.)
 *   W  device [N, ldw] of dtype, first K columns; codes, scales, zeros device, written
 * Enqueued on `stream` of the current device. */
ravel_status ravel_w4_quantize(const void* W, int N, int K, int ldw, int dtype, int group, void* codes, void* scales,
                               void* zeros, void* stream);

/* The matrix as values: out [N, ldo] of dtype, its first K columns written ((c - z) s in
 * fp32, which holds it exactly, or rounded to bf16), for example for ravel_gemm on
 * whole prompts.  Enqueued on `stream`.  (120 us for 8192 x 8192.) */
ravel_status ravel_w4_read(ravel_w4_t* w, void* out, int ldo, int dtype, void* stream);

/* out (op)= X W^T (+ bias), the epilogues of ravel_gemm:
 *   X    device bf16 [M, lda], first K columns (rows 16-byte aligned are faster, not required)
 *   epi  0: out = X W^T + bias     1: out = SiLU(X W^T + bias)
 *        2: out += X W^T + bias (float32 out)
 *        3: GeGLU (N % 128 == 0, bf16 out): W rows in 128-row blocks of 64 gate rows, then the 64
 *           matching up rows; out[m][f] = gelu_tanh(gate + bias) * (up + bias) for f < N / 2
 *   out  device [M, ldo], out_dtype RAVEL_FP32 or RAVEL_BF16; bias device float32 [N] or NULL
 * Codes are multiplied as whole numbers and sums kept in fp32, so that the result is that of the
 * weights held, not of weights rounded to bf16.  Meant for few rows, where the weights' bytes are
 * what a product costs; M up to 2^19 works, in tiles of 16 to 64 rows that each go through the matrix.
 * out must not overlap X. */
ravel_status ravel_w4_gemm(const ravel_w4_t* w, const void* X, int M, int lda, int epi, void* out, int ldo, int out_dtype,
                           const float* bias, void* stream);

/* ---- drawing a token -------------------------------------------------------------
 * Of each row of logits one token.  With w_i = exp((x_i - max x) / T), and tokens
 * ordered by their logit (equal ones by their index), of the row stay
 *   the first top_k tokens (top_k <= 0: all);
 *   of those the shortest run from the first on whose weights sum to at least
 *   top_p of their sum (top_p >= 1: all; <= 0: the first);
 *   of those the ones with w_i >= min_p (min_p above 1 counts as 1),
 * and the token is the lowest index for which the weights of what stays, summed in the
 * order of the index, exceed u times their sum.  T < 2^-20 (0, say): the first of the order.
 * Sums are of whole numbers (weights in units of 2^-43, computed to some 2^-42 whatever T), so that no order of summation enters
 * the result and ties are ties.
 *   logits       device [batch, row_stride] of dtype, vocab columns (vocab up to 2^20)
 *   u            device float32 [batch], 0 <= u < 1
 *   temperature  device float32 [batch] or NULL (1)
 *   top_k        device int32 [batch] or NULL (all)
 *   top_p, min_p device float32 [batch] or NULL (1; 0)
 *   tokens       device int32 [batch], written
 *   log_probs    device float32 [batch] or NULL, written: log of the token's share of what stays
 * A logit of -inf is never drawn.  A row without a finite logit, with a logit of NaN or +inf or
 * with a setting or u that is NaN or (u, T) out of range gets token -1 and log-probability -inf.
 * Enqueued on `stream` of the current device. */
ravel_status ravel_draw_tokens(const void* logits, int batch, int vocab, long long row_stride, int dtype, const float* u,
                               const float* temperature, const int* top_k, const float* top_p, const float* min_p,
                               int* tokens, float* log_probs, void* stream);

/* Text of the last error of a call of this header on this thread that has no cache to keep it (never NULL). */
const char* ravel_decode_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* RAVEL_DECODE_H_ */
