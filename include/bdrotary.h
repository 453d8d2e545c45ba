/*
 * bdrotary: positions on the way into the caches, and the latent cache, on one
 * GB300 (sm_103a). The forward whose hidden states bd_commit_step reads turns
 * its queries and keys by their positions (the ones bdkv_tables gives) before
 * they meet in an attention; a model with latent attention keeps, for each
 * token, one latent vector for all heads and one turned key part.
 *
 *   bdrot_rotate            rows of queries or keys turned, or turned back
 *   bdrot_write             keys turned and stored with the values in the 8-bit
 *                           cache of bdcache.h, queries turned in the same call
 *   bdrot_latent_write      latents and turned key parts into the latent cache
 *   bdrot_latent_attention  attention of all heads over the latent cache
 *
 * Conventions are those of bdcache.h: caller-owned device memory, calls
 * asynchronous on the given stream (a cudaStream_t, NULL = legacy default),
 * arguments checked before any CUDA call, status codes of bd_status, nothing
 * traps or aborts, page numbers and slots outside a cache never dereferenced.
 */
#ifndef BDROTARY_H
#define BDROTARY_H

#include <stddef.h>
#include <stdint.h>

#include "bdcache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A rotation by positions. Pair p of a row's first `dim` elements,
 *   (x[p], x[p + dim / 2]), or interleaved (x[2 p], x[2 p + 1]),
 * becomes
 *   scale * (a cos t - b sin t, a sin t + b cos t),  t = position * f_p;
 * elements from `dim` on stay as they are.
 *   turns        [dim / 2] on the device, 16-byte aligned: f_p as a fraction of
 *                a turn, times 2^64, modulo 2^64 (f_p / 2 pi * 2^64 for f_p in
 *                radians a position). position * turns modulo 2^64 is then the
 *                angle without its whole turns, exact at any position.
 *   dim          a multiple of 16, 16..256
 *   scale        0, or from 2^-96 to what fp32 holds in magnitude; cosines and
 *                sines are multiplied by it (1, or the amplitude of a rotation
 *                stretched for long contexts)
 * Positions are int32 of any sign (one behind the last token, -1, turns its row
 * as any other). Sines and cosines are fp32, results rounded once. */
typedef struct {
  const uint64_t* turns;
  int32_t dim;
  int32_t interleaved; /* 0 or 1 */
  double scale;
} bdrot_rotary;

/* ------------------------------------------------------------------ rotate --
 * out[i, h] = x[i, h] turned by positions[i], for n_tokens rows of n_heads heads
 * of head_dim elements (a multiple of 16, 16..1024, rotary->dim at least).
 *   inverse   turned by -positions[i], with the same scale: the adjoint, which
 *             takes gradients of the result to gradients of x
 * out may be x (same pointer and strides; elements behind rotary->dim are then
 * not touched) or be apart from it: rows that lie on x otherwise are refused
 * (BD_ERR_ARG), as are rows of out on one another. Rows of x may share memory.
 * To turn the last elements of a head, pass the rows that begin there. */
int bdrot_rotate(const bdrot_rotary* rotary, const bdkv_rows* x, const bdkv_rows* out, int32_t n_heads,
                 int32_t head_dim, const int32_t* positions, int64_t n_tokens, int32_t inverse, void* stream);

/* ------------------------------------------------------------------- write --
 * bdkv_write of keys turned by positions[i], rounded to their type as
 * bdrot_rotate rounds them: the cache gets the codes and scales that those two
 * calls would give. rotary->dim is at most the cache's head_dim.
 *   q, q_out     queries of the same n_tokens tokens and their turned rows, as
 *                in bdrot_rotate, with n_q_heads heads of the cache's head_dim;
 *                both NULL: keys and values alone. Rows of every token are
 *                turned, also of those whose slot is skipped.
 * k and v are only read; q_out must not lie on them. */
int bdrot_write(const bdrot_rotary* rotary, const bdkv_cache* cache, const bdkv_rows* k, const bdkv_rows* v,
                const int64_t* slot_map, const int32_t* positions, int64_t n_tokens, const bdkv_rows* q,
                const bdkv_rows* q_out, int32_t n_q_heads, void* stream);

/* ------------------------------------------------------------ latent cache --
 * One layer: n_pages pages of page_size tokens, each a latent vector of
 * latent_dim elements, which is its value and the first part of its key, and
 * rope_dim elements, the key's last part. In the 16 bits of the model: the
 * vector is shared by all heads, so it is small as it is.
 *   latent, rope   element i of a token is [page * stride[0] + token * stride[1]
 *                  + i]. Pointers 16-byte aligned, strides multiples of 8 of at
 *                  least the elements they step over, below 2^38; the two may be
 *                  parts of the same rows.
 *   page_size      16, 32, 64, 128 or 256
 *   latent_dim     a multiple of 16, 16..512
 *   rope_dim       a multiple of 16, 16..64 */
typedef struct {
  void* latent;
  void* rope;
  int32_t dtype; /* bdkv_dtype */
  int32_t page_size;
  int64_t n_pages;
  int32_t latent_dim;
  int32_t rope_dim;
  int64_t latent_stride[2]; /* page, token */
  int64_t rope_stride[2];
} bdrot_latent;

/* Stores row i of latent [n_tokens, latent_dim] and rope [n_tokens, rope_dim]
 * (stride_head is not read) at slot slot_map[i] (page * page_size + offset;
 * negative or past the cache: skipped), rope turned by positions[i].
 *   rotary      rotary->dim = rope_dim; NULL: rope is stored as it is, and
 *               positions is not read
 * A token whose latent has an infinity or NaN is stored as a latent of zeros and
 * a key part of NaN: the queries that see it get NaN, and no others. The slots
 * of a call differ (of two rows for one slot either may stay, element by
 * element). The rows must not lie in the cache. */
int bdrot_latent_write(const bdrot_rotary* rotary, const bdrot_latent* cache, const bdkv_rows* latent,
                       const bdkv_rows* rope, const int64_t* slot_map, const int32_t* positions, int64_t n_tokens,
                       void* stream);

/* Attention over the latent cache. For request s with queries query_start[s] ..
 * query_start[s + 1] (the last of its kv_lens[s] cached tokens) and head h:
 *     S_t = scale * (q[0..latent_dim) . latent_t + q[latent_dim..) . rope_t)
 *     out = sum_t softmax_t(S) latent_t   over t < visible(i)
 *     lse = ln sum_t exp(S_t)             (optional)
 * The projections from and to the heads' own widths are products of the caller
 * (the absorbed form). Masks, lengths, query_start, rows that see nothing, rows
 * whose scores are all -inf, workspace and bounds are those of bdkv_attention;
 * lse is float32 [tokens, n_heads] contiguous, or NULL.
 *   q      rows [token, head, latent_dim + rope_dim] of the cache's type
 *   out    rows [token, head, latent_dim] of the same type, apart from q: rows
 *          of the first token that lie on its queries are refused (BD_ERR_ARG);
 *          how many tokens there are is on the device, so for the others the
 *          caller sees to it
 * Latents of tokens that are seen by some query of the call are finite (as
 * bdrot_latent_write stores them); what is behind a request's tokens in its last
 * page may be anything. Products of 16-bit elements are exact and summed in
 * fp32; statistics are fp32; softmax weights are rounded to the cache's type.
 * Scores are held times log2 e, so they are infinite from 2.35e38 on, and scale
 * times log2 e must be finite (BD_ERR_ARG). Weights are up to 2^15 before they
 * are divided by their sum: bf16 latents of 2^113 / kv_len and more can overflow.
 * Limits: n_heads 1..1024, n_seq at most 65535, max_kv_len at most 2^30,
 * max_q_len * n_heads at most 2^26. */
typedef struct {
  bdkv_rows q;
  bdkv_rows out;
  float* lse;
  const int32_t* block_table;
  int64_t table_stride;
  int32_t max_blocks;
  const int32_t* kv_lens;
  const int32_t* query_start;
  int32_t n_seq;
  int32_t n_heads;
  int32_t max_q_len;
  int32_t max_kv_len;
  int32_t mask_block;
  float scale;
  void* workspace;
  size_t workspace_bytes;
  void* stream;
} bdrot_latent_attention_args;

int bdrot_latent_attention(const bdrot_latent* cache, const bdrot_latent_attention_args* args);

/* Bytes of workspace a call with these arguments needs (0 where it needs none,
 * or the arguments are invalid). Depends on sizes and the device only. */
size_t bdrot_latent_attention_workspace(const bdrot_latent* cache, const bdrot_latent_attention_args* args);

/* As bdkv_get_device_status and bdkv_shutdown, for this library. */
int bdrot_get_device_status(void* stream);
int bdrot_shutdown(void);

#ifdef __cplusplus
}
#endif

#endif /* BDROTARY_H */
