/*
 * tq_seq.h -- C ABI of the operators of sequence models over measurement
 * records, part of libtq.
 *
 * A measurement record is a sequence of bitstrings that tq_sample drew: ids
 * below a vocabulary of V rows (the 2^n bitstrings of n qubits and whatever
 * further ids a program adds, such as a start token).  A recurrent model of
 * such records looks the ids up in a table (tq_embed), runs a gated linear
 * recurrence over time (tq_gated_scan), normalises its states
 * (tq_layer_norm) and is trained by the cross entropy of the next bitstring
 * (tq_softmax_xent); each comes with its gradient.
 *
 * Conventions, beside those of tq.h
 * ---------------------------------
 *  - Every array is a DEVICE pointer owned by the caller, `stream` a
 *    hipStream_t.  Calls validate on the host, then only enqueue; they
 *    allocate nothing and clear nothing with memory-set calls, so that they
 *    may be captured into a graph.  Scratch memory is the caller's too: a
 *    call with a `workspace` needs as many bytes as its *_workspace function
 *    says, 256-byte aligned, its contents arbitrary before and after.
 *  - `type`, a tq_dtype, is the type of the arrays declared `void`; everything
 *    else has the type it is declared with.  Rows are contiguous along their last
 *    axis; a leading dimension or stride counts elements.  Arrays need the
 *    alignment of their element only.
 *  - Sums, recurrent states and softmax statistics are kept in 32 bits; an
 *    output of a 16-bit type is rounded to it once, after that.  What is rounded
 *    on the way stands at the call (tq_softmax_xent_grad).  No sum is formed
 *    with floating-point atomics: every output is bitwise reproducible.
 *  - Ids are uint64 as tq_sample writes them.  An id >= V, such as the marker
 *    2^64 - 1 of a missing shot, is no error: it has an embedding of zeros and
 *    no loss, and no gradient comes from it.
 *  - Inputs and outputs of a call must not overlap except where said.
 */
#ifndef TQ_SEQ_H
#define TQ_SEQ_H

#include "tq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { TQ_F32 = 0, TQ_BF16 = 1, TQ_F16 = 2 } tq_dtype;

/* out[i, :] = scale * table[tokens[i], :] for i < N, formed in fp32; zeros
 * where tokens[i] >= V.  table [V, D] with rows ld_table apart, out [N, D] with
 * rows ld_out apart.  TQ_E_INVALID for negative sizes, ld < D, a NULL pointer
 * with work to do; TQ_E_UNSUPPORTED for N or V >= 2^31. */
tq_status tq_embed(const void *table, int64_t ld_table, int32_t type, int64_t V, int64_t D, const uint64_t *tokens,
                   int64_t N, float scale, void *out, int64_t ld_out, void *stream);

/* Gradient of tq_embed with respect to its table: grad[v, :] = scale * sum of
 * grad_out[i, :] over the i with tokens[i] = v, in the order of i within
 * fixed pieces; every row of grad [V, D] is written.  TQ_E_UNSUPPORTED for
 * D > 2^20. */
tq_status tq_embed_grad_workspace(int64_t V, int64_t D, int64_t N, size_t *bytes);
tq_status tq_embed_grad(const void *grad_out, int64_t ld_grad_out, int32_t type, int64_t V, int64_t D,
                        const uint64_t *tokens, int64_t N, float scale, void *grad, int64_t ld_grad, void *workspace,
                        size_t workspace_bytes, void *stream);

/* The gated linear recurrence over time of B records of T steps and D
 * channels: with a_t = sigmoid(g_t),
 *     h_t = a_t h_{t-1} + (1 - a_t) x_t      (h_{-1} = h0[b], zeros if NULL)
 * for t < lengths[b] (clamped to [0, T]; NULL: all T), y_t = h_t; past its
 * length a record keeps its state and y is zero, and x and g are not looked
 * at.  x[b, t, :] lies at x + b * batch stride + t * step stride, g and y
 * likewise.  h_last [B, D], the last state, may be h0 itself, and
 * may be NULL; for a single step (T = 1) such calls advance the records'
 * states in place.  states, when not NULL, receives the states that
 * tq_gated_scan_grad starts from: float [B, ceil(T / TQ_SCAN_PIECE), D], the
 * state before step j * TQ_SCAN_PIECE (steps past a record's length: not
 * written).
 * h0, h_last and states are contiguous.  Once a channel's state is infinite or
 * NaN its later ones are infinite or NaN too; which of the two is not fixed
 * (gates multiplied together may be zero where none of them is).
 * TQ_E_UNSUPPORTED for D > 2^20 or B ceil(D / 64) ceil(T / 64) >= 2^31. */
#define TQ_SCAN_PIECE 64
tq_status tq_gated_scan_workspace(int64_t B, int64_t T, int64_t D, size_t *bytes);
tq_status tq_gated_scan(int32_t type, int64_t B, int64_t T, int64_t D, const void *x, int64_t x_batch, int64_t x_step,
                        const void *g, int64_t g_batch, int64_t g_step, const float *h0, const int32_t *lengths,
                        void *y, int64_t y_batch, int64_t y_step, float *h_last, float *states, void *workspace,
                        size_t workspace_bytes, void *stream);

/* Gradients of tq_gated_scan from dy, the gradient of y, and dh_last (NULL:
 * zeros), that of h_last: with l_t = dy_t + a_{t+1} l_{t+1} (dh_last added at
 * the record's last step),
 *     dx_t = (1 - a_t) l_t,  dg_t = a_t (1 - a_t) (h_{t-1} - x_t) l_t,
 * zeros past the record's length, and dh0 = a_0 l_0 (NULL: not wanted;
 * dh_last for an empty record).  `states` are the ones tq_gated_scan wrote
 * for the same x, g, h0 and lengths.  dy, dx and dg have batch and step
 * strides of their own. */
tq_status tq_gated_scan_grad(int32_t type, int64_t B, int64_t T, int64_t D, const void *x, int64_t x_batch,
                             int64_t x_step, const void *g, int64_t g_batch, int64_t g_step, const float *states,
                             const int32_t *lengths, const void *dy, int64_t dy_batch, int64_t dy_step,
                             const float *dh_last, void *dx, int64_t dx_batch, int64_t dx_step, void *dg,
                             int64_t dg_batch, int64_t dg_step, float *dh0, void *workspace, size_t workspace_bytes,
                             void *stream);

/* Layer norm of N rows of D values: y = (x - mean) rstd * weight + bias with
 * rstd = (variance + eps)^{-1/2}, the variance the mean of (x - mean)^2.
 * weight and bias [D] have x's type; bias may be NULL.  mean and rstd, float
 * [N], are written when not NULL (both or neither); the gradient needs them.
 * eps >= 0. */
tq_status tq_layer_norm(const void *x, int64_t ld_x, int32_t type, int64_t N, int64_t D, const void *weight,
                        const void *bias, float eps, void *y, int64_t ld_y, float *mean, float *rstd, void *stream);

/* Gradients of tq_layer_norm: with u = dy * weight and xh = (x - mean) rstd,
 *     dx = rstd (u - mean(u) - xh mean(u xh)),
 * dweight = sum over rows of dy xh and dbias = sum over rows of dy, [D] in x's
 * type (dbias may be NULL). */
tq_status tq_layer_norm_grad_workspace(int64_t N, int64_t D, size_t *bytes);
tq_status tq_layer_norm_grad(const void *x, int64_t ld_x, int32_t type, int64_t N, int64_t D, const void *weight,
                             const float *mean, const float *rstd, const void *dy, int64_t ld_dy, void *dx,
                             int64_t ld_dx, void *dweight, void *dbias, void *workspace, size_t workspace_bytes,
                             void *stream);

/* Softmax cross entropy of N rows over a vocabulary of V >= 1, from hidden
 * [N, D] and weight [V, D]: with logits z = hidden weight^T, formed piece by
 * piece of the vocabulary and not kept,
 *     lse[i] = log sum_v exp z[i, v],   loss[i] = lse[i] - z[i, targets[i]],
 * loss[i] = 0 where targets[i] >= V.  loss and lse are float [N].  Products of
 * 16-bit inputs are exact and summed in fp32; fp32 inputs are split into
 * pairs of 16-bit numbers that hold 22 of their 24 bits, products summed in
 * fp32.  A row of infinities or NaN gives NaN for that row.  TQ_E_UNSUPPORTED
 * for D > 2^20, and where ceil(N / 128) ceil(V / 128), or either times
 * ceil(D / 128), reaches 2^27. */
tq_status tq_softmax_xent_workspace(int32_t type, int64_t N, int64_t V, int64_t D, size_t *bytes);
tq_status tq_softmax_xent(const void *hidden, int64_t ld_hidden, int32_t type, int64_t N, int64_t V, int64_t D,
                          const void *weight, int64_t ld_weight, const uint64_t *targets, float *loss, float *lse,
                          void *workspace, size_t workspace_bytes, void *stream);

/* Gradient of sum_i upstream[i] loss[i], float upstream[N]: with
 * p = softmax(z) - onehot(target), dhidden[i, :] = upstream[i] p[i, :] weight
 * and dweight = (upstream p)^T hidden, both in the inputs' type; rows without
 * a target (>= V) have zero dhidden and add nothing to dweight, whatever they
 * hold.  loss and lse, the outputs of tq_softmax_xent, come from the same
 * call.  For 16-bit types p is formed in 32 bits and enters both products
 * rounded to 16; hidden times upstream enters dweight's product as two 16-bit
 * numbers, which hold what a single one would lose, unless all upstreams that
 * are not zero are the same up to powers of two.  In f16 a token's part of
 * dweight is resolved to 2^-25 of the largest upstream times one.  For fp32 the
 * numbers that a sum over rows is formed of have their 22 bits at the largest row
 * and less below it: dhidden's terms are resolved to 2^-38 of the largest weight
 * times one, dweight's to 2^-38 of the largest hidden times upstream.  For f16 and
 * fp32 p is resolved to 2^-40 at least. */
tq_status tq_softmax_xent_grad_workspace(int32_t type, int64_t N, int64_t V, int64_t D, size_t *bytes);
tq_status tq_softmax_xent_grad(const void *hidden, int64_t ld_hidden, int32_t type, int64_t N, int64_t V, int64_t D,
                               const void *weight, int64_t ld_weight, const uint64_t *targets, const float *upstream,
                               void *dhidden, int64_t ld_dhidden, void *dweight, int64_t ld_dweight, float *loss,
                               float *lse, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TQ_SEQ_H */
