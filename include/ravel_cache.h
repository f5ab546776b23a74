/*
 * ravel_cache.h -- C ABI of the 8-bit context cache: the VLM side of the
 * rolling step.  A prompt's keys and values (and those of the tokens that a
 * robot decodes) are stored in 8 bits, attended to by single tokens, by the
 * slots of an action expert or by whole prompts, shrunk to a budget by the
 * attention mass that each token drew, and read back in the layout that
 * ravel_set_context takes.
 *
 * What a cache holds, per layer, robot and KV head:
 *  - keys and values in e4m3 (4 exponent bits, 3 mantissa bits), a row of
 *    head_dim values per token;
 *  - for each block of 16 tokens one exponent e for the keys and one for the
 *    values: the smallest e >= -100 for which the largest magnitude stored is
 *    at most 448 * 2^e.  A value x is held as x / 2^e rounded to e4m3 (nearest,
 *    ties to even); a power of two costs the format no precision and makes
 *    the division exact.  (Values above 248 * 2^120 = 3.3e38 are held as 2^128,
 *    which ravel_cache_read returns as infinity.)
 *  - Tokens that arrive in a block behind others never lower its e.  Where it
 *    rises, the tokens already there are rounded again.
 *  - A token that has a value that is not finite, in its key or its value row,
 *    is held as a key row of NaN and a value row of zeros: every query that
 *    sees it gets NaN, no other query is touched by it.
 *
 * Conventions beside those of ravel.h:
 *  - B robots, robots 0 .. batch - 1 of the cache; Hq query heads, query head h
 *    reads KV head h / (Hq / Hkv).
 *  - Positions, lengths and counts are device int32 arrays, read by the kernels,
 *    so that calls can be captured into CUDA graphs.  A robot whose values are
 *    out of range is left out (its outputs are zeros) and the device error word
 *    is raised: a later call returns RAVEL_EDEVICE until ravel_cache_reset.
 *  - Strides are in elements.  Heads of a token are contiguous, [heads, head_dim],
 *    so q, k and v may be columns of one projection's rows.  16-byte aligned
 *    pointers and strides are faster, not required beyond the type's own.
 *  - A cache is not thread-safe, and its attention calls share a workspace: calls
 *    on one cache must be serialised and must not overlap on the GPU.
 */
#ifndef RAVEL_CACHE_H_
#define RAVEL_CACHE_H_

#include "ravel.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RAVEL_CACHE_BLOCK 16

typedef struct {
  int layers;       /* L */
  int n_q_heads;    /* Hq, a multiple of n_kv_heads */
  int n_kv_heads;   /* Hkv */
  int head_dim;     /* hd, a multiple of 8, at most 256 (rows are held in 64, 128, 192 or 256 bytes) */
  int max_tokens;   /* tokens per robot; max_batch * n_kv_heads * max_tokens is below 2^31 - 2^16 */
  int max_batch;    /* robots */
  int max_queries;  /* largest n of ravel_cache_attend */
  int dtype;        /* RAVEL_BF16 or RAVEL_FP32: type of the keys, values, queries and outputs of every call.
                       RAVEL_FP32 results are fp32-accurate for the keys and values held.  RAVEL_BF16: weights have
                       11 bits; of more than 16 query rows per KV head, a query's elements below 2^-13 of its
                       largest are held to within 2^-21 of the largest */
} ravel_cache_config;

typedef struct ravel_cache_ctx ravel_cache_t;

/* Validate cfg and allocate the cache and the workspace on `device`: beside the
 * tokens about 30 MB at head_dim 256 and, for the attention mass, up to 64 MB
 * (more where one query's scores, or two sums per token, take more).
 * Synchronous.  On success *out owns all of it until ravel_cache_destroy. */
ravel_status ravel_cache_create(const ravel_cache_config* cfg, int device, ravel_cache_t** out);

/* Free everything (after synchronising the device).  NULL is a no-op. */
void ravel_cache_destroy(ravel_cache_t* c);

/* Clear the device error word, after waiting for the device.  What the cache
 * holds stays. */
ravel_status ravel_cache_reset(ravel_cache_t* c);

/* Store new tokens of one layer: token i < counts[b] of robot b goes to
 * position starts[b] + i; what lay there and behind it in its last block is no
 * longer meant to be read.
 *   k, v    device [batch, n, Hkv, hd] of the cache's dtype: token i of robot b
 *           begins at element b * robot_stride + i * token_stride
 *   starts  device int32 [batch]; NULL: 0 for every robot
 *   counts  device int32 [batch], 0 <= counts[b] <= n; NULL: n for every robot
 * Enqueued on `stream`. */
ravel_status ravel_cache_append(ravel_cache_t* c, int layer, int batch, int n, const void* k, const void* v,
                                long long robot_stride, long long token_stride, const int* starts, const int* counts,
                                void* stream);

/* Attention of n queries per robot over one layer's cached tokens.
 * Robot b has lengths[b] tokens and counts[b] queries; query i sits at
 * position p = lengths[b] - counts[b] + i and sees
 *   causal = 0: every token;  causal = 1: tokens j <= p, and with window > 0 of
 *   those the ones with j > p - window or j < sinks.
 * out = softmax(scale q k) v over what it sees.  Queries that see nothing and
 * queries from counts[b] on are zeros.
 *   q, out      device [batch, n, Hq, hd] of the cache's dtype, strides as for
 *               ravel_cache_append; out must not overlap q
 *   lengths     device int32 [batch], 0 <= lengths[b] <= max_length
 *   counts      device int32 [batch], 0 <= counts[b] <= n (causal: also
 *               <= lengths[b]); NULL: n for every robot
 *   max_length  host bound of the lengths, at most max_tokens.  Launches are planned
 *               for it, the lengths being on the device: one that is far above
 *               them costs time (one token of one robot over 816, 8 heads of 256:
 *               8 us with a bound of 816, 16 with 2048, 39 with 8192, 81 with 32768)
 *   scale       > 0, or 0 for 1 / sqrt(hd)
 *   mass        device float32 [batch, Hkv, mass_stride] or NULL: entry j of
 *               [b][h] receives (mass_add = 0; zeros from lengths[b] up to
 *               max_length) or is increased by (mass_add = 1) the sum of token
 *               j's softmax weights over robot b's queries and the query heads
 *               of KV head h.  mass_stride >= max_length.
 * A query that has a value that is not finite gets NaN.  Enqueued on `stream`. */
ravel_status ravel_cache_attend(ravel_cache_t* c, int layer, int batch, int n, const void* q, long long q_robot_stride,
                                long long q_token_stride, void* out, long long out_robot_stride,
                                long long out_token_stride, const int* lengths, const int* counts, int max_length,
                                int causal, int window, int sinks, float scale, float* mass, long long mass_stride,
                                int mass_add, void* stream);

/* Eviction: of each robot and KV head the `keep` tokens that stay, in their
 * order, go into layer to_layer of another cache `to` (another layer of the same
 * one will do), from position 0 on, rounded into blocks anew.  A robot of at
 * most `keep` tokens keeps them all; of a longer one stay the first `sinks`,
 * the last `recent` and of the rest those with the largest mass (ties: the
 * earlier token; NaN counts as the largest).
 *   lengths      device int32 [batch], 0 <= lengths[b] <= max_tokens
 *   mass         device float32 [batch, Hkv, mass_stride], as written by
 *                ravel_cache_attend; mass_stride >= the longest length
 *   new_lengths  device int32 [batch], written: min(lengths[b], keep)
 *   index        device int32 [batch, Hkv, keep], written: positions that stay, then -1
 *   new_mass     device float32 [batch, Hkv, keep] or NULL, written: their mass, then 0
 * sinks + recent <= keep <= max_tokens of `to`; the caches agree in Hkv, hd, and
 * device.  Enqueued on `stream`. */
ravel_status ravel_cache_evict(ravel_cache_t* c, int layer, ravel_cache_t* to, int to_layer, int batch,
                               const int* lengths, const float* mass, long long mass_stride, int keep, int sinks,
                               int recent, int* new_lengths, int* index, float* new_mass, void* stream);

/* What the cache holds, as values: tokens firsts[b] .. firsts[b] + n - 1 of one
 * layer, in the layout of a layer of ravel_set_context.
 *   n        at most max_tokens rounded up to a multiple of 128
 *   firsts   device int32 [batch], >= 0; NULL: 0 for every robot
 *   lengths  device int32 [batch] or NULL: tokens from lengths[b] on (and NULL:
 *            from max_tokens on) are zeros
 *   k, v     device [batch, Hkv, n, hd] of the cache's dtype, contiguous, written
 * (bf16 holds every value exactly.)  Enqueued on `stream`. */
ravel_status ravel_cache_read(ravel_cache_t* c, int layer, int batch, int n, const int* firsts, const int* lengths,
                              void* k, void* v, void* stream);

/* Per-cache text of the last error (never NULL). */
const char* ravel_cache_last_error(const ravel_cache_t* c);

#ifdef __cplusplus
}
#endif
#endif /* RAVEL_CACHE_H_ */
