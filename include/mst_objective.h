/*
 * mst_objective.h -- C ABI of the LM head's other objectives (in libmst_lmhead, hand-written HIP for gfx950 / MI355X).
 *
 * mst_lmhead_ce_fwd / _bwd (mst_lmhead.h) give the mean cross-entropy of logits Z = H W^T.  The calls here give, in the same
 * mini-sequences, with the same tiles and likewise without logits in memory, two objectives that training needs beside it:
 *
 *   wce      cross-entropy of capped logits, with a weight for each token, a penalty on the log-sum-exp and every token's loss
 *   distill  divergence from a teacher of which the largest logits of each token were kept, and cross-entropy beside it
 *
 * Of row s with logits z (float32):
 *   y_v   = softcap * tanh(z_v / softcap), or z_v where softcap is 0
 *   lse   = log sum_v exp(y_v),   nll = lse - y_label                     where the row has a label
 *   wce:      l_s = weight_s * (nll + z_coef * lse^2)                     where the row has a label, else 0
 *   distill:  l_s = weight_s * (label_coef * nll + teacher_coef * T^2 * kd)      each term where the row has a label, a teacher
 *   loss  = sum_s l_s / n,   n = rows that have a label or a teacher, or `divisor` where that is not 0 (the tokens of a whole
 *           step that is made of several calls, say); 0 where no row has either
 *
 * The teacher gives row s up to K entries, vocabulary indices v_k with logits t_k.  With T the temperature, and with
 * teacher_lse_s = log sum over the teacher's whole vocabulary of exp(t / T), or NULL:
 *   q_k   = exp(t_k / T - teacher_lse_s)  and  rest = max(0, 1 - sum_k q_k)      where teacher_lse is given
 *   q     = softmax of t / T over the entries,  rest = 0                         where it is NULL
 *   p     = softmax of y / T over the whole vocabulary,  p_rest = the sum of p over all v that are no entry of the row
 *   kd    = sum_k q_k (log q_k - log p_{v_k}) + rest (log rest - log p_rest)     (0 log 0 = 0)
 * so rest is compared with what the student leaves to all other vocabulary entries together.  p_rest is summed up itself, not
 * formed as a difference from 1.  Where a row's entries are the whole vocabulary, rest counts as 0.
 *
 * Gradients (by y; by z times 1 - (y / softcap)^2):
 *   at the entries       label terms + teacher_coef T weight (p_v (Q + rest) - q_v),  Q = sum_k q_k
 *   at all others        label terms + teacher_coef T weight (p_v (Q + rest) - rest p_v / p_rest)
 *   label terms          label_coef weight (softmax(y)_v - [v == label]), wce: + 2 z_coef weight lse softmax(y)_v
 *
 * Conventions: those of mst_lmhead.h (device pointers, streams, graphs, errors, M, shapes, alignment), and
 *   - labels equal to ignore_index have no loss; a row whose entries are all missing, or have a logit of -infinity (or one of
 *     -5e29 or less, as masks of a type's lowest value) all of them with teacher_lse NULL, has no teacher; one NaN among them makes kd
 *     and the loss NaN;
 *   - an index below 0 is no entry (rows with fewer than K entries, in any place); an index that comes twice in a row counts
 *     once, with the logit it has first;
 *   - a label outside [0, V) that is not ignore_index, or an index of V or more, never causes an out-of-range access: *loss is
 *     then NaN, *n_valid -1, and the backward call fills dH and dW with NaN;
 *   - a row of weight 0 adds nothing to the loss and has no gradient; it counts in n;
 *   - `saved` carries what the backward call needs from the forward call (mst_objective_bytes): per row 16 bytes, distill 24 and
 *     8 for each of K entries.  The backward call takes softcap, temperature, coefficients, weights, labels and the teacher from
 *     it; H, W, S, d, V and K have to be those of the forward call, M need not be.  NULL where no backward call follows;
 *   - M is the largest number of mini-sequences: the calls make fewer, longer ones as long as the fp32 logits of one are at most
 *     512 MiB and its rows x d below 2^30, and their workspace is that of these, whatever larger M is given;
 *   - arithmetic: that of mst_lmhead.h; a capped logit within 8 half steps of float32 of its value, at any cap; the loss and the
 *     rows' outputs float32 (sums over rows in 64 bits); the gradient of the logits rounded to bf16 before the two products, without
 *     grad_loss / n and without what all rows have in common: the labels' coefficient but for a power of 2, with label_coef 0 or no
 *     labels teacher_coef * temperature (a factor that all weights have is better given as grad_loss).  Everything in a fixed order,
 *     without atomics: repeated calls give the same bits;
 *   - no output and neither `saved` nor the workspace may overlap another argument (MST_ERR_BAD_ARGUMENT);
 *   - mst_profile_collect counts the launches under the kinds of the plain calls' that they stand for: sorting a teacher's entries under the
 *     label scan, putting them into the logits' gradient and adding up dW's parts under dH's reduce.
 */
#ifndef MST_OBJECTIVE_H
#define MST_OBJECTIVE_H

#include "mst_lmhead.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MST_MAX_ENTRIES 256       /* largest K */

/*
 * Bytes of the forward's and the backward's workspace and of `saved` (host, pure; each pointer may be NULL).  K: 0 for wce.
 * The backward's workspace is that of mst_lmhead_ce_bwd, one mini-sequence (see M above) of fp32 logits; the forward's that of
 * mst_lmhead_ce_fwd and 8 bytes a row, for distill also 6 bytes for each pair that is kept there and 12 K + 4 bytes for each row of
 * a group of mini-sequences; small calls up to 0.2 MB more.
 */
mst_status mst_objective_bytes(int64_t S, int64_t d, int64_t V, int32_t M, int32_t K, size_t* fwd_bytes, size_t* bwd_bytes, size_t* saved_bytes);

/*
 *   H        bf16 [S, d];  W bf16 [V, d];  labels int32 [S]
 *   weights  fp32 [S], or NULL: all 1
 *   softcap  0 (none), or 0.001 to 1e6;  z_coef finite;  divisor >= 0
 *   loss     out, fp32 scalar
 *   nll, lse out, fp32 [S] each, each may be NULL: of every row; nll is 0 where the row has no label
 *   n_valid  out, int64 scalar, may be NULL: rows with a label
 */
mst_status mst_lmhead_wce_fwd(const void* H, const void* W, const int32_t* labels, const float* weights,
                              int64_t S, int64_t d, int64_t V, int32_t ignore_index, int32_t M,
                              float softcap, float z_coef, int64_t divisor,
                              void* workspace, size_t workspace_bytes, void* saved, size_t saved_bytes,
                              float* loss, float* nll, float* lse, int64_t* n_valid, void* stream);

/* dH bf16 [S, d] and dW fp32 [V, d], both fully overwritten; grad_loss: upstream gradient of the loss (host value). */
mst_status mst_lmhead_wce_bwd(const void* H, const void* W, int64_t S, int64_t d, int64_t V, int32_t M, float grad_loss,
                              const void* saved, size_t saved_bytes, void* workspace, size_t workspace_bytes,
                              void* dH, float* dW, void* stream);

/*
 *   labels   int32 [S], or NULL: the teacher alone (label_coef 0, nll NULL)
 *   teacher_index  int32 [S, K];  teacher_logits [S, K] of teacher_type (0: bf16, 1: fp32);  teacher_lse fp32 [S] or NULL
 *   K        1 to MST_MAX_ENTRIES, and S * max(K, 64) below 2^32;  label_coef, teacher_coef finite;  temperature 0.01 to 100
 *   nll, kd  out, fp32 [S] each, each may be NULL: 0 where the row has no label, no teacher
 *   n_valid  out, int64 scalar, may be NULL: rows with a label or a teacher
 */
mst_status mst_lmhead_distill_fwd(const void* H, const void* W, const int32_t* labels, const float* weights,
                                  const int32_t* teacher_index, const void* teacher_logits, int32_t teacher_type, const float* teacher_lse,
                                  int64_t S, int64_t d, int64_t V, int32_t K, int32_t ignore_index, int32_t M,
                                  float softcap, float label_coef, float teacher_coef, float temperature, int64_t divisor,
                                  void* workspace, size_t workspace_bytes, void* saved, size_t saved_bytes,
                                  float* loss, float* nll, float* kd, int64_t* n_valid, void* stream);

mst_status mst_lmhead_distill_bwd(const void* H, const void* W, int64_t S, int64_t d, int64_t V, int32_t K, int32_t M, float grad_loss,
                                  const void* saved, size_t saved_bytes, void* workspace, size_t workspace_bytes,
                                  void* dH, float* dW, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MST_OBJECTIVE_H */
