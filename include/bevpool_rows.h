/*
 * bevpool_rows.h -- row operators of libbevpool.so: the moves of the pooling
 * path (a stable sort by key, rows read through the sorted trace, weighted
 * sums of rows and their gradients) for keys that are expert ids or row ids
 * instead of voxels.
 *
 *   sort_keys   stable order of n keys, the analogue of bevpool_prepare
 *   route       router: softmax weights of the k best experts of each token
 *   dispatch    token rows in the order of their experts
 *   combine     weighted sum of each token's expert rows
 *   expert_layer  router weights to output in one call, for a few tokens
 *   embed       lookup of table rows with a scale; its gradient sums the rows
 *               of each id through the sorted order, without atomics
 *
 * Conventions are those of bevpool.h (device pointers owned by the caller,
 * nothing allocated or synchronised, arguments validated before any HIP call,
 * negative bevpool_status, the stream as void*, float32 accumulation rounded
 * once to the output type, every output element written with one value, no
 * atomics on floating-point values, bitwise reproducible results), and:
 *   - a row is moved in vectors of 16 bytes; where its length is not a multiple
 *     of them, the last one ends with the row and repeats elements of the one
 *     before, which are then stored twice, with the same value;
 *   - element types are BEVPOOL_F32, BEVPOOL_F16 and BEVPOOL_BF16.  Where a
 *     call has an in_dtype and an out_dtype, they are equal or out_dtype is
 *     F32;
 *   - a matrix argument marked with a stride has that many elements between
 *     its rows (0 for one row repeated); within a row elements are
 *     neighbours.  Other arrays are dense.  Pointers need the alignment of
 *     their element only;
 *   - keys outside [0, n_keys) are dropped, not errors (as bevpool_prepare
 *     drops points outside the grid): padding, or a token past an expert's
 *     capacity.  Dropped slots sort behind all kept ones;
 *   - row counts may be 0 (the pointers of empty arrays may be NULL);
 *   - outputs must not alias inputs or each other;
 *   - kernels bounds-check every place and id they read;
 *   - limits: n = rows * k < 2^31, n_keys < 2^31 - 1, C <= 2^20,
 *     n_experts <= 1024 and k <= 64 in route; in expert_layer n_experts <= 1024,
 *     rows k <= 1024, C and F <= 2^16.
 */
#ifndef BEVPOOL_ROWS_H
#define BEVPOOL_ROWS_H

#include "bevpool.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A third element type (bfloat16), accepted by the calls of this header. */
#define BEVPOOL_BF16 2

enum bevpool_key_type {
  BEVPOOL_KEY_I32 = 0, /* int32 keys */
  BEVPOOL_KEY_I64 = 1  /* int64 keys */
};

/*
 * Stable sort of n keys.  Writes
 *   order[n]            the slots (indices of keys) in ascending key, ties in
 *                       ascending slot, dropped slots last;
 *   position[n]         the place of each slot: position[order[q]] = q;
 *   offsets[n_keys + 1] offsets[v] = number of kept keys below v, so key v's
 *                       slots are order[offsets[v] .. offsets[v + 1]) and
 *                       offsets[n_keys] is the number of kept slots.
 * The workspace is scratch of bevpool_sort_keys_workspace_size bytes (may be
 * NULL when that is 0).
 */
int bevpool_sort_keys_workspace_size(int64_t n, int64_t n_keys, size_t* bytes);
int bevpool_sort_keys(int64_t n, int64_t n_keys, int key_type, const void* keys, int32_t* order,
                      int32_t* position, int32_t* offsets, void* workspace,
                      size_t workspace_bytes, void* stream);

/*
 * Router.  For every row of logits (rows x n_experts): the k largest logits,
 * equal ones by the lower index; -inf (and NaN) logits are never chosen.
 * ids (rows x k, descending logit) holds the chosen experts, weights (rows x
 * k, float32) exp(logit - m) over the sum of that term over the chosen
 * experts (renormalise != 0) or over all experts (0), m the row's largest
 * logit.  Where fewer than k experts can be chosen the remaining ids are -1
 * and their weights 0.  A row that holds a NaN gets NaN for all k weights.
 *
 * bevpool_route_backward gives the logits' gradient (rows x n_experts, dtype,
 * dense) from the weights' gradient, the logits, and the forward's weights
 * and ids:
 *   renormalise: grad[id_j] = w_j (g_j - s), 0 elsewhere;
 *   else:        grad[e] = p_e (G_e - s), p the softmax over all experts and
 *                G_{id_j} = g_j, 0 elsewhere;  s = sum_j w_j g_j.
 * Slots whose id names no expert (-1, or outside [0, n_experts)) have no
 * gradient and no part in s.  The logits are only read when
 * renormalise is 0 (else they may be NULL).
 */
int bevpool_route_forward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                          const void* logits, int64_t logits_stride, int renormalise,
                          float* weights, int32_t* ids, void* stream);
int bevpool_route_backward(int64_t rows, int32_t n_experts, int32_t k, int dtype,
                           const float* grad_weights, const void* logits, int64_t logits_stride,
                           const float* weights, const int32_t* ids, int renormalise,
                           void* grad_logits, void* stream);

/*
 * Dispatch: x (rows x C), each row with k slots.
 *   out[position[t k + j]] = x[t]        for a kept slot,
 *   out[position[t k + j]] = 0           for a dropped one,
 * so the rows of expert e are out[offsets[e] .. offsets[e + 1]) and the rows
 * behind offsets[n_keys] are zero.  bevpool_dispatch_forward sorts the ids
 * (rows x k) itself and writes order, position and offsets as
 * bevpool_sort_keys does (its workspace is that call's);
 * bevpool_dispatch_rows moves the rows by an order at hand, `kept` pointing
 * at offsets[n_keys].
 *
 * bevpool_dispatch_backward: grad_x[t] = sum over the kept slots j of t of
 * grad_out[position[t k + j]].
 */
int bevpool_dispatch_forward(int64_t rows, int32_t k, int64_t C, int64_t n_keys, int dtype,
                             const void* x, int64_t x_stride, int key_type, const void* ids,
                             int32_t* order, int32_t* position, int32_t* offsets, void* out,
                             void* workspace, size_t workspace_bytes, void* stream);
int bevpool_dispatch_rows(int64_t rows, int32_t k, int64_t C, int dtype, const void* x,
                          int64_t x_stride, const int32_t* position, const int32_t* kept,
                          void* out, void* stream);
int bevpool_dispatch_backward(int64_t rows, int32_t k, int64_t C, int dtype, const void* grad_out,
                              int64_t grad_stride, const int32_t* position, const int32_t* kept,
                              void* grad_x, void* stream);

/*
 * Combine: out[t] = sum over the kept slots j of t of
 *   weights[t k + j] * in[position[t k + j]],
 * in (rows k x C) the experts' outputs in dispatch order, weights of
 * weight_dtype (F32 or in_dtype).  Rows behind *kept are not used.
 *
 * bevpool_combine_backward:
 *   grad_in[position[t k + j]]  = weights[t k + j] * grad_out[t], 0 for a
 *                                 dropped slot;
 *   grad_weights[t k + j]       = <grad_out[t], in[position[t k + j]]>, 0 for
 *                                 a dropped slot (weight_dtype).
 * grad_out has out_dtype, grad_in in_dtype.  Either output may be NULL and is
 * then not formed (in may be NULL without grad_weights, weights without
 * grad_in).
 */
int bevpool_combine_forward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                            int weight_dtype, const void* in, int64_t in_stride,
                            const void* weights, const int32_t* position, const int32_t* kept,
                            void* out, void* stream);
int bevpool_combine_backward(int64_t rows, int32_t k, int64_t C, int in_dtype, int out_dtype,
                             int weight_dtype, const void* grad_out, int64_t grad_stride,
                             const void* in, int64_t in_stride, const void* weights,
                             const int32_t* position, const int32_t* kept, void* grad_in,
                             void* grad_weights, void* stream);

/*
 * Expert layer of a few tokens, without an order: with slot s = t k + j of
 * expert e = ids[s],
 *   hidden[s, f] = silu(<x[t], up[e, f]>) <x[t], up[e, F + f]>,  silu(a) = a / (1 + e^-a)
 *   out[t]       = sum over the kept slots j of t of weights[s] down[e] hidden[s],
 * up (n_experts x 2F x C) and down (n_experts x C x F) dense, x, up, down and out
 * of dtype, weights (rows x k) of weight_dtype (F32 or dtype), ids int32 as
 * bevpool_route_forward writes them (those outside [0, n_experts) are dropped;
 * experts without a slot are not read).  Sums and hidden are float32, whatever
 * dtype.  A token whose slots are all dropped is zeros.
 */
int bevpool_expert_layer_workspace_size(int64_t rows, int32_t k, int64_t C, int64_t F,
                                        int32_t n_experts, int dtype, size_t* bytes);
int bevpool_expert_layer_forward(int64_t rows, int32_t k, int64_t C, int64_t F, int32_t n_experts,
                                 int dtype, int weight_dtype, const void* x, int64_t x_stride,
                                 const void* up, const void* down, const void* weights,
                                 const int32_t* ids, void* out, void* workspace,
                                 size_t workspace_bytes, void* stream);

/*
 * Embedding: out[i] = scale * table[ids[i]], zeros for an id outside
 * [0, table_rows); ids of key_type, n of them, table (table_rows x C).
 *
 * bevpool_embed_backward: grad_table[v] = scale * sum over ids[i] = v of
 * grad_out[i], zeros where v does not occur; the table's gradient is written
 * in full.  grad_out has in_dtype, grad_table out_dtype (equal, or one of the
 * two F32).  The ids are sorted
 * within the call; the workspace holds that order and the partial sums of
 * ids that occur often (bevpool_embed_backward_workspace_size bytes).
 */
int bevpool_embed_forward(int64_t n, int64_t table_rows, int64_t C, int in_dtype, int out_dtype,
                          const void* table, int64_t table_stride, int key_type, const void* ids,
                          float scale, void* out, void* stream);
int bevpool_embed_backward_workspace_size(int64_t n, int64_t table_rows, int64_t C, size_t* bytes);
int bevpool_embed_backward(int64_t n, int64_t table_rows, int64_t C, int in_dtype, int out_dtype,
                           const void* grad_out, int64_t grad_stride, int key_type,
                           const void* ids, float scale, void* grad_table, void* workspace,
                           size_t workspace_bytes, void* stream);

#ifdef __cplusplus
} /* extern "C" */
#endif

#endif /* BEVPOOL_ROWS_H */
