/*
 * ufs.h -- C ABI of the state operators: linear attention with a decay for each
 * head (whole sequences with their gradient; prompts, pieces of prompts and single
 * tokens over states that a cache holds), the reordering of those states, and the
 * selection of a beam search.
 *
 * They stand beside the token operators of uft.h: where a token cache keeps what a
 * window sees, a state keeps all of the past in one matrix a head.  Conventions are
 * those of uf.h and uft.h: bf16 as raw bit patterns, head_dim 128, d_* device pointers
 * owned by the caller, work enqueued on `stream` without synchronisation or
 * allocation, status codes of uf.h (uf_last_error has the text), handles not
 * thread-safe.
 *
 * Linear attention.  Key head h has a log decay g_h (float32, a constant: no gradient;
 * at most 0 in earnest, 0 forgets nothing, -inf all), L = exp(g_h).  Over the tokens t
 * of a sequence, from a state S_-1 (zero where none is given),
 *     S_t = L S_{t-1} + k_t v_t^T          [128 (of k), 128 (of v)], float32
 *     o_t = scale S_t^T q_t   =   scale ( sum_{j <= t} L^{t-j} (q_t.k_j) v_j + L^{t+1} S_-1^T q_t ).
 * Query head n reads key head n / (q_heads / kv_heads).  Scores, states and
 * accumulators are fp32; weights and states enter their products in two bf16 parts (in
 * steps of few tokens in fp32), what is added to a state in three (backwards in two where
 * d_dstate is not wanted, and for dq's walks always: their states are no results), and every
 * bf16 result is rounded once.  A value that is not finite reaches its own token and those
 * after it (gradients: dk and dv before it), and no others.
 */
#ifndef UFS_H
#define UFS_H

#include "uf.h"
#include "uft.h" /* uft_stride */

#ifdef __cplusplus
extern "C" {
#endif

/* ---- whole sequences -------------------------------------------------------- */

/* d_q [batch, tokens, q_heads, head_dim], d_k, d_v [batch, tokens, kv_heads,
 * head_dim] bf16 (16-byte aligned, strided), d_decay [kv_heads] fp32, d_o [batch,
 * tokens, q_heads, head_dim] bf16 contiguous.  d_lengths, NULL or int32 [batch]
 * (device): tokens from d_lengths[b] on (brought into 0 .. tokens) are padding: not read,
 * and their rows get zeros, in o and in the gradients.  d_state, NULL (zeros) or fp32
 * [batch, kv_heads, head_dim, head_dim]: the states before the first token; d_final, NULL
 * or the same: those behind the last one (d_final may be d_state; outputs overlap nothing
 * else).
 *
 * Sequences are cut into parts where that fills the GPU; the states between them lie
 * in d_work (16-byte aligned, >= ufs_linear_work_bytes; 0 bytes: may be NULL).  A part of
 * a sequence's key head is a workgroup, of which there are at most 2^23 - 1 (else
 * UF_ERR_ARG, of the sizes' queries too).  scale: finite.  Errors: UF_ERR_ARG,
 * UF_ERR_UNSUPPORTED (head_dim), UF_ERR_HIP.
 *
 * Backward: d_do [batch, tokens, q_heads, head_dim] bf16 contiguous; d_dfinal, NULL
 * (zeros) or the gradient of the final states, fp32; outputs d_dq (as q) and d_dk, d_dv
 * (as k) bf16, contiguous, fully overwritten, and d_dstate, NULL or the gradient of
 * d_state, fp32 (also where that is NULL).  Gradients of a key head add over its query
 * heads in fp32.  No atomics: results are reproducible.  A call's work may not be shared
 * with a call that runs at the same time. */
typedef struct {
  int32_t batch, tokens, q_heads, kv_heads, head_dim;
  float scale;
  uft_stride q, k, v;
} ufs_linear_desc;
int ufs_linear_work_bytes(const ufs_linear_desc* desc, size_t* bytes);
int ufs_linear_fwd(const ufs_linear_desc* desc, const void* d_q, const void* d_k, const void* d_v, const float* d_decay,
                   const int32_t* d_lengths, const float* d_state, void* d_o, float* d_final, void* d_work,
                   size_t work_bytes, void* stream);
int ufs_linear_bwd_work_bytes(const ufs_linear_desc* desc, size_t* bytes);
int ufs_linear_bwd(const ufs_linear_desc* desc, const void* d_q, const void* d_k, const void* d_v, const void* d_do,
                   const float* d_decay, const int32_t* d_lengths, const float* d_state, const float* d_dfinal,
                   void* d_dq, void* d_dk, void* d_dv, float* d_dstate, void* d_work, size_t work_bytes, void* stream);

/* ---- states that a cache holds ----------------------------------------------- */

typedef struct ufs_cache ufs_cache; /* opaque host-side handle: what each sequence holds */

/* States of at most max_seqs sequences in `layers` layers.  flags: UF_F_DRYRUN or 0. */
typedef struct {
  int32_t layers;   /* 1 .. 65535 */
  int32_t kv_heads; /* 1 .. 4096 */
  int32_t head_dim; /* must be 128 */
  int32_t max_seqs; /* 1 .. 65535; sequences are named 0 .. max_seqs-1 */
  uint32_t flags;
} ufs_desc;

typedef struct {
  int32_t step_seqs;    /* sequences of the last ufs_extend, 0 if it no longer holds (see there) */
  int32_t step_tokens;  /* its new tokens */
  int32_t step_longest; /* the most new tokens of one of its sequences */
} ufs_info;

/* Bytes of the pool, [layers][max_seqs][kv_heads][head_dim (of k)][head_dim (of v)]
 * fp32, and of the device table.  Errors: UF_ERR_ARG, UF_ERR_UNSUPPORTED. */
int ufs_pool_bytes(const ufs_desc* desc, size_t* bytes);
int ufs_table_bytes(const ufs_desc* desc, size_t* bytes);

/* Create a handle over a caller-owned pool and table (256-byte aligned), which must
 * outlive it; neither needs to be cleared: a sequence that holds no token has the
 * state zero, whatever lies in its place.  Errors: UF_ERR_ARG, UF_ERR_UNSUPPORTED,
 * UF_ERR_CAPACITY (a buffer is too small). */
int ufs_create(const ufs_desc* desc, void* d_pool, size_t pool_bytes, void* d_table, size_t table_bytes, ufs_cache** out);
int ufs_destroy(ufs_cache* cache); /* NULL is accepted */

/* Begin a step: sequence seqs[i] grows by counts[i] >= 0 tokens (an empty one
 * begins).  Each layer then takes the new tokens by one ufs_attn, which moves its
 * states past them; tokens are counted sequence by sequence.  A step no longer
 * holds once one of its sequences is reordered or freed.  A sequence appears once.  A
 * captured graph of ufs_attn reads the step from the table when it is replayed: it may
 * be replayed after any later step of as many sequences with the same counts (after
 * another it stays within its buffers, and some sequences are left out).
 * Errors: UF_ERR_ARG (also: a sequence of more than 2^31 - 1 tokens), UF_ERR_HIP (no
 * sequence has grown; the step before may no longer hold). */
int ufs_extend(ufs_cache* cache, int32_t n, const int32_t* seqs, const int32_t* counts, void* stream);

/* Linear attention of the step's tokens: d_q [step tokens, q_heads, head_dim], d_k, d_v
 * [step tokens, kv_heads, head_dim] bf16 (16-byte aligned, strided; batch strides are
 * not read), d_decay [kv_heads] fp32, d_o [step tokens, q_heads, head_dim] bf16
 * contiguous.  The layer's states of the step's sequences are replaced by those behind
 * their new tokens: a second call in the same step would take the tokens once more (and a
 * sequence that begins would begin again).  d_work (16-byte aligned, >=
 * ufs_attn_work_bytes for the same step; 0 bytes: may be NULL) holds states between parts of
 * long sequences; a call's work may not be shared with a call that runs at the same
 * time.  Errors: UF_ERR_ARG, UF_ERR_EMPTY (no step), UF_ERR_HIP. */
typedef struct {
  int32_t q_heads; /* a multiple of kv_heads */
  float scale;
  uft_stride q, k, v;
} ufs_attn_desc;
int ufs_attn_work_bytes(const ufs_cache* cache, size_t* bytes);
int ufs_attn(const ufs_cache* cache, int32_t layer, const ufs_attn_desc* desc, const void* d_q, const void* d_k,
             const void* d_v, const float* d_decay, void* d_o, void* d_work, size_t work_bytes, void* stream);

/* Sequences dst[i], empty before, become continuations of src[i]: states are copied,
 * all layers, as they are (so: behind a step's layers, as in ufs_reorder).  Errors:
 * UF_ERR_ARG (a dst twice, or not empty), UF_ERR_EMPTY (src has no token), UF_ERR_HIP. */
int ufs_fork(ufs_cache* cache, int32_t n, const int32_t* src, const int32_t* dst, void* stream);

/* Reorder states, all layers: the sequences seqs[g * beams + i], i = 0 .. beams-1, of
 * each group g go on from the states that seqs[g * beams + d_parents[g][i]] of the same
 * group had before the call; d_parents int32 [groups, beams] (device).  A parent that
 * is none of 0 .. beams-1 leaves its sequence as it is.  The sequences of a group hold
 * the same number of tokens, at least one; a sequence appears once; beams is 1 .. 64.
 * Errors: UF_ERR_ARG, UF_ERR_EMPTY (a sequence has no token), UF_ERR_HIP (the first
 * groups may be reordered). */
int ufs_reorder(ufs_cache* cache, int32_t groups, int32_t beams, const int32_t* seqs, const int32_t* d_parents, void* stream);

/* Empty the sequences.  Host metadata only.  Errors: UF_ERR_ARG. */
int ufs_free(ufs_cache* cache, int32_t n, const int32_t* seqs);

int ufs_get_info(const ufs_cache* cache, ufs_info* info);
int ufs_seq_tokens(const ufs_cache* cache, int32_t seq, int32_t* tokens);

/* ---- the selection of a beam search ------------------------------------------- */

/* Each of `groups` requests has `beams` hypotheses with scores (sums of log
 * probabilities; -inf: not in use) and logits over a vocabulary.  Continuation (w, t) has
 * the score
 *     score_w + (logit_wt - lse_w),   lse_w = log sum_t exp(logit_wt),
 * each step rounded to fp32.  lse_w comes of fp32 exponentials: before its rounding it is off
 * by at most 2^-19 + 2^-22 m, m the mean of the row's largest logit less each, by the row's
 * probabilities; rows of the same logits have the same bits of it.  A finished hypothesis (d_done, NULL or one byte each, not 0)
 * has the one continuation (w, end) with score_w itself, and its logits are not read.  A
 * continuation whose score is NaN or -inf is none.
 *
 * Selected are the k best of each request, best first, equal scores by the lowest
 * (w, t): d_best fp32, d_parents and d_tokens int32 [groups, k]; where there are fewer,
 * the places left get -inf, -1 and -1.
 *
 * d_logits [groups, beams, vocab], contiguous along the vocabulary, with strides in
 * elements; aligned to its type.  d_scores [groups, beams] fp32, d_done [groups, beams].
 * groups * beams <= 2^20, beams <= 64, vocab <= 2^24, k <= 64.  d_work (16-byte aligned,
 * >= ufs_select_work_bytes) is scratch; a call's work may not be shared with a call
 * that runs at the same time.  Errors: UF_ERR_ARG, UF_ERR_UNSUPPORTED (the type),
 * UF_ERR_HIP. */
#define UFS_BF16 0
#define UFS_FP16 1
#define UFS_FP32 2
typedef struct {
  int32_t groups, beams, vocab, k;
  int32_t type;                     /* of the logits */
  int32_t end;                      /* 0 .. vocab-1; not read without d_done */
  int64_t group_stride, beam_stride; /* >= 0, at most 2^40 */
} ufs_select_desc;
int ufs_select_work_bytes(const ufs_select_desc* desc, size_t* bytes);
int ufs_select(const ufs_select_desc* desc, const void* d_logits, const float* d_scores, const uint8_t* d_done,
               float* d_best, int32_t* d_parents, int32_t* d_tokens, void* d_work, size_t work_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* UFS_H */
