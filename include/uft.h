/*
 * uft.h -- C ABI of the token operators: a paged cache of tokens, attention over
 * it under a sliding window with sinks (prompts, single tokens, trees of drafted
 * tokens), and the same attention of whole sequences with its gradient.
 *
 * They stand beside the chunk window of uf.h, whose pinned first chunk and
 * oldest-first eviction they repeat at the granularity of tokens, and follow its
 * conventions: bf16 as raw bit patterns, head_dim 128, d_* device pointers owned by
 * the caller, work enqueued on `stream` without synchronisation or allocation,
 * status codes of uf.h (uf_last_error has the text), handles not thread-safe.
 *
 * Visibility.  Positions count from 0 in each sequence.  The query at position i
 * sees the key at position j iff
 *     j <= i  and  (window == 0  or  i - j < window  or  j < sinks),
 * and, in the cache, j's page is there (uft_trim).  For each query and head
 *     O = sum_j softmax_j(scale q.k_j) v_j over the keys it sees,
 *     LSE = natural log of sum_j exp(scale q.k_j);
 * a query that sees nothing gets O = 0 and LSE = -inf.  Query head n reads key
 * head n / (q_heads / kv_heads).  Scores, weights' sums and accumulators are fp32;
 * weights are rounded to bf16 for their product with V.  A key or value that is not
 * finite reaches the queries that see it and no others, and in the gradients the rows
 * that they take part in and no others, Q and dO alike (where there is one, the rows
 * beside it are formed key by key, which is slow: a backward of 2 ms takes 40).  Memory
 * past a sequence's end, padding and pages of others are never read.
 */
#ifndef UFT_H
#define UFT_H

#include "uf.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct uft_cache uft_cache; /* opaque host-side handle: page tables and use counts */

/* A cache of at most max_seqs sequences of at most max_tokens tokens each, in
 * n_pages pages of page_tokens tokens.  A page holds its tokens of every layer:
 * `layers` pools of the same pages, one page table.  flags: UF_F_DRYRUN or 0. */
typedef struct {
  int32_t layers;      /* 1 .. 65535 */
  int32_t kv_heads;    /* 1 .. 4096 */
  int32_t head_dim;    /* must be 128 */
  int32_t page_tokens; /* 64 or 128 */
  int32_t n_pages;     /* >= 1 */
  int32_t max_seqs;    /* 1 .. 65535; sequences are named 0 .. max_seqs-1 */
  int32_t max_tokens;  /* 1 .. 2^30 */
  uint32_t flags;
} uft_desc;

typedef struct {
  int32_t free_pages;  /* pages that no sequence holds */
  int32_t step_seqs;   /* sequences of the last uft_extend, 0 if it no longer holds (see there) */
  int32_t step_tokens; /* its new tokens */
  int32_t step_longest;/* the most new tokens of one of its sequences */
} uft_info;

/* Elements between neighbours along each axis; the head dimension is contiguous.
 * Multiples of 8, at most 2^24 from token to token and 2^30 from head to head; batch
 * is not read where there is none. */
typedef struct {
  int64_t batch, token, head;
} uft_stride;

/* Bytes of the pool, [layers][n_pages][K, V][kv_heads][page_tokens][head_dim] bf16,
 * and of the device tables.  Errors: UF_ERR_ARG, UF_ERR_UNSUPPORTED. */
int uft_pool_bytes(const uft_desc* desc, size_t* bytes);
int uft_table_bytes(const uft_desc* desc, size_t* bytes);

/* Create a handle over a caller-owned pool and table (256-byte aligned), which must
 * outlive it; neither needs to be cleared.  Errors: UF_ERR_ARG,
 * UF_ERR_UNSUPPORTED, UF_ERR_CAPACITY (a buffer is too small). */
int uft_create(const uft_desc* desc, void* d_pool, size_t pool_bytes, void* d_table, size_t table_bytes,
               uft_cache** out);
int uft_destroy(uft_cache* cache); /* NULL is accepted */

/* Begin a step: sequence seqs[i] grows by counts[i] >= 0 tokens (an empty one
 * begins).  Pages are taken lowest free number first, sequence by sequence; a
 * partly filled last page that other sequences share is copied into a page of its
 * own first (all layers).  The new tokens' rows are written by uft_write and
 * attended by uft_attn, layer by layer; both act on the last step, in whose order
 * tokens are counted: sequence by sequence.  A step no longer holds once one of
 * its sequences is kept or freed, or trimmed of the step's own tokens.  A sequence
 * appears once.  A captured graph of uft_write and uft_attn reads the step from the
 * tables when it is replayed: it may be replayed after any later step of as many
 * sequences with the same counts.
 * Errors: UF_ERR_ARG, UF_ERR_CAPACITY (no free pages, or longer than max_tokens),
 * UF_ERR_HIP. */
int uft_extend(uft_cache* cache, int32_t n, const int32_t* seqs, const int32_t* counts, void* stream);

/* Write the step's keys and values of one layer: d_k, d_v [step tokens, kv_heads,
 * head_dim] bf16, 16-byte aligned.  Errors: UF_ERR_ARG, UF_ERR_EMPTY (no step),
 * UF_ERR_HIP. */
int uft_write(const uft_cache* cache, int32_t layer, const void* d_k, const uft_stride* k_stride, const void* d_v,
              const uft_stride* v_stride, void* stream);

/* Sequences dst[i], empty before, become continuations of src[i]: they share its
 * pages until one of them grows (uft_extend).  Errors: UF_ERR_ARG (a dst twice, or
 * not empty), UF_ERR_EMPTY (src has no token), UF_ERR_HIP. */
int uft_fork(uft_cache* cache, int32_t n, const int32_t* src, const int32_t* dst, void* stream);

/* The same with pages of their own: rows of src are copied as they are (all layers;
 * those of a step that is not written yet may hold anything).
 * Errors: as uft_fork, and UF_ERR_CAPACITY. */
int uft_copy(uft_cache* cache, int32_t n, const int32_t* src, const int32_t* dst, void* stream);

/* Keep chosen tokens: sequence seqs[i] keeps its first starts[i] tokens, then the
 * tokens whose positions are the next counts[i] entries of d_index (int32, device
 * memory, any order, all of the sequence), moved to positions starts[i], ...; the
 * rest leaves.  counts[i] = 0 cuts the sequence to starts[i] tokens (d_index may be
 * NULL where all are 0).  starts[i] + counts[i] is at most the sequence's length; a
 * position outside the sequence, or trimmed, gives a row of zeros.  Up to 16 tokens are moved in place,
 * if no other sequence shares the pages they go to; otherwise fresh pages are
 * taken, lowest free number first, sequence by sequence, from the page of
 * starts[i] on, before the old ones are given back.  A sequence appears once.
 * Errors: UF_ERR_ARG (also: pages from starts[i] on were trimmed),
 * UF_ERR_CAPACITY, UF_ERR_HIP. */
int uft_keep(uft_cache* cache, int32_t n, const int32_t* seqs, const int32_t* starts, const int32_t* counts,
             const int32_t* d_index, void* stream);

/* Give back the pages of sequences that no query of a later step sees under this
 * window (>= 1) and these sinks: whole pages of positions j with sinks <= j <=
 * length - window.  Queries attended after the call, of a wider window and of the
 * present step too, see nothing there; positions do not change.  So it belongs
 * behind a step's last layer; a step some of whose own tokens lie in those pages
 * no longer holds.  Errors: UF_ERR_ARG, UF_ERR_HIP. */
int uft_trim(uft_cache* cache, int32_t n, const int32_t* seqs, int32_t window, int32_t sinks, void* stream);

/* Empty the sequences; pages that no other sequence shares become free (their
 * rows stay until they are taken again).  Host metadata only.  Errors: UF_ERR_ARG. */
int uft_free(uft_cache* cache, int32_t n, const int32_t* seqs);

/* Move pages so that those in use are numbered 0 .. used-1 (the highest into the
 * lowest free, all layers).  used_pages may be NULL.  Errors: UF_ERR_ARG, UF_ERR_HIP. */
int uft_pack(uft_cache* cache, int32_t* used_pages, void* stream);

/* State.  uft_seq_pages writes the page of each page_tokens tokens of a sequence,
 * -1 where it was trimmed, at most `cap`, and gives their number.  Errors:
 * UF_ERR_ARG. */
int uft_get_info(const uft_cache* cache, uft_info* info);
int uft_seq_tokens(const uft_cache* cache, int32_t seq, int32_t* tokens);
int uft_seq_pages(const uft_cache* cache, int32_t seq, int32_t* pages, int32_t cap, int32_t* n);

/* Attention of the step's tokens over their sequences.  d_q [step tokens, q_heads,
 * head_dim] bf16 (16-byte aligned, strided), d_o the same, contiguous; d_lse
 * [step tokens, q_heads] fp32 or NULL.
 *
 * d_tree, NULL or int64 [step tokens] (device): the new tokens of each sequence, at
 * most 64, are nodes of a tree over its earlier tokens.  Bit u of node t's word
 * says that t sees node u (its ancestors and itself; others are possible; bits of
 * no node are not read).  The node's position is that of the first new token + the
 * number of nodes it sees - 1 (at least the first new token's); earlier tokens are
 * seen by the window rule from there.  window must be 0 or at least the nodes of
 * every sequence.
 *
 * Where the step has too few rows for n_cu compute units (n_cu = 0: never) a row's
 * keys are cut into slices that leave partial results in d_work (16-byte aligned,
 * >= uft_attn_work_bytes for the same step, q_heads and desc; 0 bytes: may be NULL),
 * joined by a second launch.  A call's work may not be shared with a call that
 * runs at the same time.  scale: positive and finite, scale*log2(e) a normal float.
 * Errors: UF_ERR_ARG, UF_ERR_UNSUPPORTED (a tree of more than 64 nodes),
 * UF_ERR_EMPTY (no step), UF_ERR_HIP. */
typedef struct {
  int32_t q_heads; /* a multiple of kv_heads */
  int32_t window;  /* >= 0; 0: all earlier tokens */
  int32_t sinks;   /* >= 0 */
  int32_t n_cu;    /* >= 0 */
  float scale;
  uft_stride q;
} uft_attn_desc;
int uft_attn_work_bytes(const uft_cache* cache, const uft_attn_desc* desc, size_t* bytes);
int uft_attn(const uft_cache* cache, int32_t layer, const uft_attn_desc* desc, const void* d_q, const int64_t* d_tree,
             void* d_o, float* d_lse, void* d_work, size_t work_bytes, void* stream);

/* The same attention of whole sequences, without a cache: d_q [batch, tokens,
 * q_heads, head_dim], d_k, d_v [batch, tokens, kv_heads, head_dim] bf16 (16-byte
 * aligned, strided), d_o [batch, tokens, q_heads, head_dim] bf16 contiguous, d_lse
 * [batch, q_heads, tokens] fp32 or NULL.  d_lengths, NULL or int32 [batch] (device):
 * tokens from d_lengths[b] on are padding: no key, not read, and their rows get
 * O = 0, LSE = -inf and zero gradients.  q.head times the query heads of a key head
 * is at most 2^30; scale as for uft_attn, and at least 2^-100.  Errors: UF_ERR_ARG, UF_ERR_HIP.
 *
 * Backward: d_o and d_lse as the forward of the same call left them (a row's weights,
 * exp(scale q.k - LSE), are taken to sum to 1), d_do [batch, tokens, q_heads,
 * head_dim] bf16 contiguous; outputs d_dq (as q) and d_dk, d_dv (as k) bf16,
 * contiguous, fully overwritten; gradients of a key head add over its query heads
 * in fp32.  The weights are rounded to bf16 for dV, the scores' gradients for dK (from
 * weights in fp16, scaled) and, in two parts, for dQ; everything else is fp32.  d_work
 * (16-byte aligned, >= uft_window_bwd_work_bytes) is scratch.  No atomics: results are
 * reproducible. */
typedef struct {
  int32_t batch, tokens, q_heads, kv_heads, head_dim;
  int32_t window, sinks;
  float scale;
  uft_stride q, k, v;
} uft_window_desc;
int uft_window_fwd(const uft_window_desc* desc, const void* d_q, const void* d_k, const void* d_v,
                   const int32_t* d_lengths, void* d_o, float* d_lse, void* stream);
int uft_window_bwd_work_bytes(const uft_window_desc* desc, size_t* bytes);
int uft_window_bwd(const uft_window_desc* desc, const void* d_q, const void* d_k, const void* d_v, const void* d_o,
                   const float* d_lse, const void* d_do, const int32_t* d_lengths, void* d_dq, void* d_dk, void* d_dv,
                   void* d_work, size_t work_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* UFT_H */
