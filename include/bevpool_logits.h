/*
 * bevpool_logits.h -- operators over rows of logits: what a model answers with
 * and learns from, over vocabularies as over depth bins.
 *
 *   logprobs   log probabilities of given tokens, the distribution's log-sum-exp
 *              and entropy, and its k best alternatives; the logits' gradient
 *   distill    divergence from a teacher's k alternatives; the logits' gradient,
 *              by itself or with the loss
 *
 * A row of logits x (V of them, of element type dtype) stands for the
 * distribution p = softmax(scale x), scale > 0 an inverse temperature (scale log2 e
 * has to be finite in float32: up to 2.35e38).  Values beyond float32 are infinite,
 * the difference of two logits among them.
 *
 * Conventions are those of bevpool_rows.h (device pointers owned by the caller,
 * nothing allocated or synchronised, arguments validated before any HIP call,
 * float32 sums rounded once, a fixed order of operations, bitwise reproducible
 * results, a matrix with a stride has that many elements between its rows,
 * pointers aligned to their element, rows may be 0), and:
 *   - ids outside [0, V) are dropped, not errors: a position without a token, an
 *     alternative that the student does not know;
 *   - a logit of -inf has probability 0.  A row of nothing else has no
 *     distribution: its log probabilities and lse are -inf, its entropy 0, its
 *     alternatives -1, its gradient 0;
 *   - a NaN or +inf in a row makes that row's values NaN, but for those of
 *     dropped ids;
 *   - a row whose outgoing gradients are zero or belong to dropped ids (padding)
 *     has a gradient of zeros whatever it holds;
 *   - in gradients, an element of a token with an outgoing gradient of its own, or
 *     of one that is taught, may be stored twice: with its vector and, after that,
 *     with its value;
 *   - limits: rows < 2^31, V <= 2^20, k <= V, and k <= 64 in logprobs, <= 256 in
 *     distill.
 */
#ifndef BEVPOOL_LOGITS_H
#define BEVPOOL_LOGITS_H

#include "bevpool_rows.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Log probabilities.  For every row t:
 *   stats[2 t], stats[2 t + 1]  the largest logit m (NaN not counted; -inf where
 *                 there is none, and beside a NaN for float32's lowest number)
 *                 and S = sum_v e^(scale (x_v - m)) (0 for a row without a
 *                 distribution, NaN for one that holds a NaN or +inf);
 *   logprob[t]    scale (x_id - m) - log S for ids[t] (of key_type), 0 for an id
 *                 outside [0, V);
 *   lse[t]        scale m + log S;
 *   entropy[t]    -sum_v p_v log p_v;
 *   top, top_ids  (rows x k) the k largest logits, equal ones by the lower
 *                 index: their log probabilities and indices, in that order.  NaN
 *                 and -inf are never chosen; where fewer than k can be, the rest
 *                 are -inf and -1.
 * stats is always written.  logprob (and ids), lse and entropy may be NULL; top
 * and top_ids are not used where k is 0.  The workspace is scratch of
 * bevpool_logprobs_workspace_size bytes (may be NULL when that is 0).
 *
 * bevpool_logprobs_backward: with the outgoing gradients g of logprob, lse,
 * entropy and top (each NULL where there is none)
 *   grad[v] = scale (p_v (g_lse - g_logprob - sum_j g_top_j - g_entropy (log p_v + H))
 *                    + [v = id] g_logprob + sum_j [v = top_ids_j] g_top_j)
 * from the forward's stats, entropy H (read with grad_entropy only) and top_ids
 * (with grad_top).  grad_logits is rows x V, dense, of dtype.
 */
int bevpool_logprobs_workspace_size(int64_t rows, int64_t V, int32_t k, int dtype, size_t* bytes);
int bevpool_logprobs_forward(int64_t rows, int64_t V, int32_t k, int dtype, const void* logits,
                             int64_t logits_stride, float scale, int key_type, const void* ids,
                             float* stats, float* logprob, float* lse, float* entropy, float* top,
                             int32_t* top_ids, void* workspace, size_t workspace_bytes,
                             void* stream);
int bevpool_logprobs_backward(int64_t rows, int64_t V, int32_t k, int dtype, const void* logits,
                              int64_t logits_stride, float scale, int key_type, const void* ids,
                              const float* stats, const float* entropy, const int32_t* top_ids,
                              const float* grad_logprob, const float* grad_lse,
                              const float* grad_entropy, const float* grad_top, void* grad_logits,
                              void* stream);

/*
 * Distillation.  A teacher's k alternatives of every row: ids (rows x k, of
 * key_type) and their log probabilities teacher (rows x k, float32).  Slots
 * whose id is dropped have no part, whatever their log probability, nor have
 * slots of log probability -inf.  With q_j = e^teacher_j, over the sum of the
 * row's kept slots where renormalise != 0,
 *   loss[t] = sum_j q_j (log q_j - log p_id_j)
 * over the slots with q_j > 0 (0 where there are none); an id that occurs more
 * than once counts each time.  Renormalised, what is added to all of a row's
 * teacher has no part.  A NaN in a kept slot (renormalised, +inf too) makes the
 * row's loss and gradient NaN.  stats as above.
 *
 * bevpool_distill_backward: grad[v] = grad_loss scale (Q p_v - sum_j [v = id_j] q_j),
 * Q = sum_j q_j, from the forward's stats; grad_logits as above.
 * bevpool_distill_step forms both, for callers whose grad_loss does not depend
 * on the loss.  Forward and step share bevpool_distill_workspace_size.
 */
int bevpool_distill_workspace_size(int64_t rows, int64_t V, int32_t k, int dtype, size_t* bytes);
int bevpool_distill_forward(int64_t rows, int64_t V, int32_t k, int dtype, const void* logits,
                            int64_t logits_stride, float scale, int key_type, const void* ids,
                            const float* teacher, int renormalise, float* loss, float* stats,
                            void* workspace, size_t workspace_bytes, void* stream);
int bevpool_distill_backward(int64_t rows, int64_t V, int32_t k, int dtype, const float* grad_loss,
                             const void* logits, int64_t logits_stride, float scale, int key_type,
                             const void* ids, const float* teacher, int renormalise,
                             const float* stats, void* grad_logits, void* stream);
int bevpool_distill_step(int64_t rows, int64_t V, int32_t k, int dtype, const float* grad_loss,
                         const void* logits, int64_t logits_stride, float scale, int key_type,
                         const void* ids, const float* teacher, int renormalise, float* loss,
                         float* stats, void* grad_logits, void* workspace, size_t workspace_bytes,
                         void* stream);

#ifdef __cplusplus
} /* extern "C" */
#endif

#endif /* BEVPOOL_LOGITS_H */
