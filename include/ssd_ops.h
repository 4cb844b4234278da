/*
 * ssd_ops.h — operators of libssd for training a draft on its oracle.
 *
 * Staged speculative decoding (Sec. 2.3, 3.2 of arXiv 2308.04623) is only as
 * fast as its draft agrees with the oracle.  A draft is brought nearer by
 * sampling a batch of continuations of one prompt from the oracle, and fitting
 * the draft's distribution to the oracle's on them.  The operators here are what
 * that takes beside the verification pass and the top-k of ssd.h, for a draft
 * whose layers between embedding and logits have their gradients elsewhere (or
 * are none, as a bigram model's); attention has no backward pass:
 *   ssd_prefix_attn      attention of a batch of sequences over the keys and
 *                        values of a prompt they share and over their own;
 *   ssd_distill_*        the divergence of the draft's logits from the
 *                        oracle's top logits, and its gradient;
 *   ssd_embed, ssd_embed_grad
 *                        scaled embedding rows, and the table's gradient.
 *
 * The conventions of ssd.h hold: device pointers are the caller's, work goes
 * onto the caller's stream, nothing synchronises the host, every argument
 * check runs on the host before anything is enqueued.  No call allocates:
 * those that need scratch take a workspace of the size their _workspace
 * function gives, whose contents do not matter before and after a call; calls
 * that share one are ordered by the caller (one stream, or events).  All can be
 * captured into a HIP graph.  Results are bitwise the same from run to run.
 */
#ifndef SSD_OPS_H
#define SSD_OPS_H

#include "ssd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Shapes and strides of ssd_prefix_attn.  Strides count elements; the
 * head_dim elements of a head's row lie side by side.
 *   q, out             element (b, t, h, i) at b q_seq + t q_row + h q_head + i
 *   k_prefix, v_prefix element (g, j, i) at g prefix_head + j prefix_row + i
 *   k_own, v_own       element (b, g, j, i) at b own_seq + g own_head + j own_row + i
 * with b < n_seq, t < n_query, h < n_head, g < n_kv_head. */
typedef struct {
  ssd_dtype dtype; /* of q, keys, values and out */
  int32_t n_seq, n_query, n_head, n_kv_head, head_dim;
  int32_t prefix_len; /* rows of k_prefix and v_prefix */
  int32_t own_rows;   /* rows of k_own and v_own for each sequence and head */
  float scale;        /* of the scores, e.g. 1 / sqrt(head_dim) */
  int64_t q_seq, q_row, q_head;
  int64_t out_seq, out_row, out_head;
  int64_t prefix_head, prefix_row;
  int64_t own_seq, own_head, own_row;
} ssd_prefix_attn_desc;

/* Bytes of workspace for a call with these shapes (0 < *bytes).  Errors:
 * as ssd_prefix_attn for the shapes. */
ssd_status ssd_prefix_attn_workspace(const ssd_prefix_attn_desc *a, size_t *bytes);

/* Attention of n_seq sequences that share a prefix.  Sequence b's queries are
 * its last n_query positions: its own rows 0 .. own_len[b]-1 (device; their
 * keys and values are written already) end with them.  Query t of sequence b
 * sees every prefix row and own rows j <= own_len[b] - n_query + t; head h
 * reads the keys and values of head h / (n_head / n_kv_head).  out is the
 * softmax of scale q.k over the seen rows times their values; rows that are
 * not seen are never looked at and may hold anything.  A query that sees no
 * row gives 0, and so do the queries of a sequence with own_len[b] < 0 (an
 * unused slot of the batch); lengths past own_rows count as own_rows.  A row whose
 * score is -infinity counts as one that is not seen; a score of NaN makes the
 * query's out and lse NaN.
 * lse, if not NULL: float32 [n_seq][n_query][n_head], the log of the sum of
 * exponentials of the seen scores (-infinity where there are none).
 *   dtype SSD_F32 or SSD_BF16; head_dim 32, 64 or 128; n_head a multiple of
 * n_kv_head and at most 1024; 1 <= n_seq <= 4096, 1 <= n_query <= 64, prefix_len,
 * own_rows >= 0 and below 2^30.  Pointers are 16-byte aligned and strides multiples
 * of 16 bytes, not negative; out's rows do not overlap, nor does out share an
 * element with an input (it may lie between its rows, heads or tokens, where a
 * step that divides the larger ones of both tells them apart).  k_prefix and v_prefix may be NULL when prefix_len is 0,
 * k_own and v_own when own_rows is 0.  Scores and sums are float32: q.k and |scale| q.k have to lie below 2^127 in size, and are infinite
 * beyond.  bfloat16 calls round the weights exp(x - max) to bfloat16 for the
 * product with the values.
 * Errors: SSD_E_INVALID_ARG, SSD_E_CAPACITY (workspace too small, or queries and
 * chunks of rows for 2^24 workgroups), SSD_E_UNSUPPORTED (head_dim, alignment),
 * SSD_E_DEVICE. */
ssd_status ssd_prefix_attn(const ssd_prefix_attn_desc *a, const void *q, const void *k_prefix, const void *v_prefix,
                           const void *k_own, const void *v_own, const int32_t *own_len, void *out, float *lse,
                           void *workspace, size_t workspace_bytes, void *stream);

/* Divergence of a student's logits from a teacher's top logits.  Row n's
 * teacher tokens are ids[n][k] with the logits vals[n][k] (as ssd_topk
 * gives them); a slot is left out when its id is outside [0, vocab) or its
 * logit is -infinity.  With T the temperature,
 *   p = softmax(vals[n] / T) over the row's slots,
 *   q = softmax(logits[n] / T) over the vocabulary,
 *   loss[n]    = weight[n] sum_j p_j (log p_j - log q(id_j)),
 *   lse[n]     = log sum_i exp(logits[n][i] / T),
 *   dlogits[n] = weight[n] / T (q - p), rounded once to the logits' type.
 * Slots that name one token twice each count.  weight may be NULL (all 1); a
 * row whose weight is 0 or whose slots are all left out has loss and dlogits
 * 0, whatever its logits hold (its lse is still the logits').  All arithmetic
 * is float32.
 *   logits, dlogits: [n_rows][vocab] of dtype, ld and ld_d elements from row to
 * row; any alignment of the element's.  dlogits may be logits itself (with the
 * same row stride) and overlaps it in no other way.  ids, vals: [n_rows][k].
 * n_rows >= 0, 1 <= vocab <= 2^24, 1 <= k <= 128, temperature and
 * log2(e) / temperature positive and finite.
 * Errors: SSD_E_INVALID_ARG, SSD_E_DEVICE. */
ssd_status ssd_distill_forward(ssd_dtype dtype, const void *logits, int64_t ld, int32_t n_rows, int32_t vocab,
                               const int32_t *ids, const float *vals, int32_t k, const float *weight,
                               float temperature, float *loss, float *lse, void *stream);
/* The gradient from lse as ssd_distill_forward left it; weight[n] is the
 * derivative of the objective with respect to row n's unweighted divergence.
 * (q is exp(logits / T - lse) here and carries lse's rounding, 2^-24 |lse| of itself.) */
ssd_status ssd_distill_backward(ssd_dtype dtype, const void *logits, int64_t ld, int32_t n_rows, int32_t vocab,
                                const int32_t *ids, const float *vals, int32_t k, const float *lse,
                                const float *weight, float temperature, void *dlogits, int64_t ld_d, void *stream);
/* Both at once, for weights known beforehand: the logits are read once where a
 * row fits the registers of a compute unit (float32: 98,304 entries, bfloat16:
 * 196,608). */
ssd_status ssd_distill_step(ssd_dtype dtype, const void *logits, int64_t ld, int32_t n_rows, int32_t vocab,
                            const int32_t *ids, const float *vals, int32_t k, const float *weight, float temperature,
                            float *loss, float *lse, void *dlogits, int64_t ld_d, void *stream);

/* out[n] = scale table[tokens[n]], rounded once to out's type; a token outside
 * [0, vocab) gives a row of zeros.  table [vocab][d], ld_table elements from
 * row to row; out [n][d], ld_out.  Any alignment of the element's.  n >= 0,
 * 1 <= vocab <= 2^24, 1 <= d <= 65536.  Errors: SSD_E_INVALID_ARG,
 * SSD_E_DEVICE. */
ssd_status ssd_embed(ssd_dtype table_dtype, ssd_dtype out_dtype, const int32_t *tokens, int32_t n, const void *table,
                     int64_t ld_table, int32_t vocab, int32_t d, float scale, void *out, int64_t ld_out,
                     void *stream);

/* Gradient of ssd_embed with respect to the table:
 *   dtable[v] = scale sum of grad[n] over the n with tokens[n] = v,
 * 0 for a token that does not occur; with accumulate != 0 the sum is added to
 * dtable (the gradient of a tied LM head, say) and other rows are left alone.
 * Tokens outside [0, vocab) add nothing.  A row's terms are added in float32 in
 * an order that the tokens alone decide, and rounded once to dtable's type.
 * Sizes as ssd_embed, n <= 2^24.  Errors: SSD_E_INVALID_ARG, SSD_E_CAPACITY
 * (workspace too small, or a workspace that is not 16-byte aligned), SSD_E_DEVICE. */
ssd_status ssd_embed_grad_workspace(int32_t n, int32_t vocab, int32_t d, size_t *bytes);
ssd_status ssd_embed_grad(ssd_dtype grad_dtype, ssd_dtype table_dtype, const int32_t *tokens, int32_t n,
                          const void *grad, int64_t ld_grad, int32_t vocab, int32_t d, float scale,
                          int32_t accumulate, void *dtable, int64_t ld_table, void *workspace,
                          size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
