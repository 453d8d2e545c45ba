/*
 * bdcache: the paged 8-bit key/value cache of the serving loop around the
 * commit step, on one GB300 (sm_103a). The forward whose hidden states
 * bd_commit_step reads attends over the cached tokens of each request and the
 * window of blocks behind them; the blocks that bd_commit_sweep commits stay
 * in the cache ("one-step cache writes", engine appendix of the paper).
 *
 *   bdkv_tables     pages for the tokens a forward adds or takes back: block
 *                   tables, slot map and positions from the requests' lengths
 *   bdkv_write      the forward's keys and values into the cache
 *   bdkv_attention  attention of the forward's queries over the cache
 *
 * Conventions are those of bdcommit.h: caller-owned device memory, calls
 * asynchronous on the given stream (a cudaStream_t, NULL = legacy default),
 * arguments checked before any CUDA call, status codes of bd_status, nothing
 * traps or aborts. A page number of a block table or slot map outside the
 * cache is never dereferenced (its tokens are skipped by a write and read as
 * zero codes by the attention).
 */
#ifndef BDCACHE_H
#define BDCACHE_H

#include <stddef.h>
#include <stdint.h>

#include "bdcommit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of queries, keys, values and outputs. */
typedef enum {
  BDKV_BF16 = 1, /* = BD_BF16 */
  BDKV_F16 = 16  /* IEEE binary16 */
} bdkv_dtype;

/* The cache of one layer: n_pages pages of page_size tokens, n_heads
 * key/value heads of head_dim elements.
 *   k, v            E4M3 codes (OCP "fn"); element (page, token, head, i) of k
 *                   is k[page * k_stride[0] + token * k_stride[1] +
 *                   head * k_stride[2] + i], of v alike. Pointers 16-byte
 *                   aligned, strides non-negative multiples of 16. A cache that
 *                   is only read may share memory between pages, tokens or
 *                   heads (a stride of 0); bdkv_write refuses it (BD_ERR_ARG),
 *                   and scales of pages that share memory.
 *   k_scale, v_scale  one E8M0 byte e for each page and head, at
 *                   [page * stride + head]: the element's value is
 *                   code * 2^(e - 127). A power of two decodes exactly, and a
 *                   page whose scale grows is scaled again without a second
 *                   rounding (but for codes that become subnormal). bdkv_write
 *                   stores e in 27..247; the attention takes 27..227, and
 *                   values that are not NaN (bdkv_write stores none: one in a
 *                   token may reach queries of the call that do not see it).
 *   page_size       16, 32, 64, 128 or 256
 *   head_dim        a multiple of 16, 16..128 */
typedef struct {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int64_t n_pages;
  int32_t page_size;
  int32_t n_heads;
  int32_t head_dim;
  int64_t k_stride[3];
  int64_t v_stride[3];
  int64_t k_scale_stride;
  int64_t v_scale_stride;
} bdkv_cache;

/* Rows [token, head, head_dim], head_dim contiguous; strides in elements,
 * multiples of 8; pointer 16-byte aligned. Rows that are read may share memory
 * (a stride of 0); rows that are written must not (BD_ERR_ARG where the
 * strides show that they do). */
typedef struct {
  void* data;
  int32_t dtype; /* bdkv_dtype */
  int64_t stride_token;
  int64_t stride_head;
} bdkv_rows;

/* ------------------------------------------------------------- page tables --
 * One forward's bookkeeping on the GPU, with no host round trip. Request s
 * holds lens[s] tokens (negative: none) in the pages block_table[s,
 * 0..ceil(lens[s] / page_size)) and adds new_tokens[s] tokens, or, where that
 * is negative, gives its last -new_tokens[s] tokens back (all of them at most).
 *
 * Free pages wait in a ring: free_pages[i mod ring_size] for pool_in[0] <= i <
 * pool_in[1] (head, tail). Pages are taken from the head, in the requests'
 * order; pages that a request no longer needs are put behind the tail, in the
 * requests' order and from its table's front. Pages given back in a call can
 * be taken from the next call on. pool_out receives the new (head, tail);
 * pool_in is not written, so a call repeated on the same inputs gives the same
 * outputs. The ring must have room for every page of the cache.
 *
 * A request that is not served adds nothing, but its added tokens count in
 * query_start all the same (so that rows keep their places): what an attention
 * computes for those rows, whose tokens are not in the cache, means nothing and
 * must not be used.
 *
 * status[s]: 0 = served; 1 = too few free pages (the request, and every later
 * one that needs a page, keeps its length); 2 = it would need more than
 * max_blocks pages (it keeps its length and takes no page).
 *   kv_lens[s]      the length after the call (lens[s] where status is not 0)
 *   query_start     [n_seq + 1] exclusive sums of max(new_tokens, 0)
 *   slot_map[i]     for added token i: page * page_size + offset in the page;
 *                   -1 for a request not served and behind the last added token
 *   positions[i]    its position in the request; -1 behind the last
 *   block_table     entries of pages taken are written, others left alone
 * slot_map and positions have max_tokens entries, all written; tokens past
 * them are not (their pages are taken all the same). query_start counts them: an
 * attention of such a forward needs rows for all of them.
 * Limits: n_seq 0..8192; page_size as in bdkv_cache; sums of lengths below 2^31. */
typedef struct {
  int32_t n_seq;
  int32_t page_size;
  int32_t max_blocks;  /* columns of block_table */
  int32_t max_tokens;  /* entries of slot_map and positions */
  int64_t table_stride; /* elements between rows of block_table */
  int64_t ring_size;
  const int32_t* lens;
  const int32_t* new_tokens;
  int32_t* block_table;
  int32_t* free_pages;
  const int64_t* pool_in;
  int64_t* pool_out; /* must not be pool_in */
  int32_t* kv_lens;  /* must not be lens */
  int32_t* query_start;
  int64_t* slot_map;
  int32_t* positions;
  int32_t* status;
} bdkv_tables_args;

int bdkv_tables(const bdkv_tables_args* args, void* stream);

/* ------------------------------------------------------------------ writes --
 * Quantises n_tokens rows of keys and values into the cache. Row i goes to
 * slot slot_map[i] (page * page_size + offset; negative or past the cache:
 * skipped). Rows whose slots follow one another in a page form a run; the rows
 * of a page in one call must form one run (as bdkv_tables lays them out), and
 * a page belongs to one request.
 *   - A run that begins at offset 0 starts its page afresh: the scale of a head
 *     is the smallest power of two that brings the run's largest magnitude of
 *     that head to at most 448 (2^-100 at least).
 *   - A run that begins at offset a > 0 keeps the a tokens before it: the scale
 *     is the larger of the page's and the run's own, and where it grows those
 *     tokens' codes are scaled by the (power of two) ratio, to the nearest
 *     code, ties to even.
 *   Tokens of the page behind the run hold nothing afterwards. What they and
 *   tokens before them have done to the page's scale stays: a window that is
 *   written and taken back leaves a page that is not begun afresh with the
 *   largest scale it has needed. With E4M3's four bits an element is then off
 *   by at most 2^-4 of it and 2^-9 * 2^(e - 127), e the page's scale: only
 *   elements below 2^-13 of the largest that the page has held are coarser
 *   than 2^-4.
 *   - code = e4m3(x * 2^(127 - e)), to nearest, ties to even.
 *   - A token with an infinity or NaN in its key or value of a head is stored,
 *     for that head, as a key of NaN codes and a value of zeros, and does not
 *     count for the scales: the queries that see it get NaN, and no others. */
int bdkv_write(const bdkv_cache* cache, const bdkv_rows* k, const bdkv_rows* v, const int64_t* slot_map,
               int64_t n_tokens, void* stream);

/* --------------------------------------------------------------- attention --
 * For request s with queries query_start[s] .. query_start[s + 1] (q_len of
 * them, the last q_len of its kv_lens[s] cached tokens) and query head h, which
 * reads key/value head h / (n_q_heads / n_heads):
 *     out = sum_t softmax_t(scale * q . k_t) v_t    over t < visible(i)
 *     lse = ln sum_t exp(scale * q . k_t)           (optional)
 * query_start is ascending, from 0 or more, and q, out and lse have at least
 * query_start[n_seq] rows (it is on the device: nothing checks it).
 *   mask_block 0: visible(i) = kv_len
 *   mask_block B >= 1: causal by blocks of B queries,
 *       visible(i) = kv_len - q_len + min(q_len, (i / B + 1) * B);
 *     B = 1 is causal, B = the engine's block length its block-causal mask.
 * A query that sees no token (an empty cache, or kv_len < q_len) gives 0 and
 * lse -inf; one whose scores are all -inf (an infinity in q) gives NaN and lse
 * -inf, as the formula does. Products of 16-bit by decoded 8-bit elements are
 * exact (of bf16 queries: elements down to 2^-31 of their row's largest;
 * smaller ones are off by at most 2^-39 of it) and summed in fp32; statistics
 * are fp32; the softmax weights are rounded to f16, scaled so that weights down
 * to 2^-22 of a row's largest keep 11 bits (smaller ones 2^-33 of it).
 *   max_q_len, max_kv_len  upper bounds of the q_len and kv_lens (a longer one
 *                   is cut there); max_kv_len <= max_blocks * page_size.
 *                   They size the launch: tight bounds launch less.
 *   lse             float32 [tokens, n_q_heads] contiguous, or NULL
 *   workspace       bdkv_attention_workspace bytes, 256-byte aligned; NULL = a
 *                   library-owned buffer of the current device, grown on demand
 *                   (not inside graph capture). One workspace must not be used
 *                   by calls that can run at the same time.
 * Limits: n_q_heads a multiple of n_heads, at most 64 times it; n_seq at most
 * 65535; max_kv_len at most 2^30. Rows of `out` past query_start[n_seq] are
 * left alone. */
typedef struct {
  bdkv_rows q;
  bdkv_rows out; /* dtype = q.dtype */
  float* lse;
  const int32_t* block_table;
  int64_t table_stride;
  int32_t max_blocks;
  const int32_t* kv_lens;
  const int32_t* query_start;
  int32_t n_seq;
  int32_t n_q_heads;
  int32_t max_q_len;
  int32_t max_kv_len;
  int32_t mask_block;
  float scale;
  void* workspace;
  size_t workspace_bytes;
  void* stream;
} bdkv_attention_args;

int bdkv_attention(const bdkv_cache* cache, const bdkv_attention_args* args);

/* Bytes of workspace a call with these arguments needs (0 where it needs none,
 * or the arguments are invalid). Depends on sizes only. */
size_t bdkv_attention_workspace(const bdkv_cache* cache, const bdkv_attention_args* args);

/* Synchronises `stream`, then returns and clears the library's device status
 * on the current device: BD_OK, or BD_ERR_TIMEOUT if a bounded device-side
 * wait gave up since the last call (that call's outputs are invalid). */
int bdkv_get_device_status(void* stream);

/* Frees the library-owned workspaces. No call may be in flight. */
int bdkv_shutdown(void);

#ifdef __cplusplus
}
#endif

#endif /* BDCACHE_H */
