/*
 * tq_model.h -- C ABI of the operators of selective models of measurement
 * records, part of libtq: beside the operators of tq_seq.h, whose conventions
 * hold here too.
 *
 * A selective model of records mixes a few neighbouring steps of a record
 * (tq_causal_conv) and carries a state along it whose decay and whose input
 * depend on each step (tq_selective_scan); both advance by single steps where
 * records are extended.  Its gradients are clipped together (tq_clip_grad_norm), and
 * a beam search answers with the most likely records: tq_beam_select chooses the
 * beams' continuations, tq_beam_reorder gathers the states that go with them.
 */
#ifndef TQ_MODEL_H
#define TQ_MODEL_H

#include "tq_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The selective state space scan over time of B records of T steps, D channels
 * and S states (1 <= S <= 64) per channel: with
 *     d_t = softplus(dt_t + dt_bias)                                  [D]
 *     h_t = exp(d_t A) h_{t-1} + d_t x_t B_t   (h_{-1} = h0[b])       [D, S]
 *     y_t = (sum_s C_t[s] h_t[:, s] + skip x_t) silu(z_t)             [D]
 * for t < lengths[b] (clamped to [0, T]; NULL: all T).  Past its length a record
 * keeps its state, y is zero and x, dt, B, C and z are not looked at.  x, dt, z
 * and y are [B, T, D], Bm and Cm (the B_t and C_t) [B, T, S], each with a batch
 * and a step stride of its own; A is float [D, S], skip and dt_bias float [D].
 * NULL stands for zeros in h0, skip and dt_bias; a NULL z leaves the factor
 * silu(z) out.  h_last float [B, D, S], the last state, may be h0 itself and may
 * be NULL: a call with T = 1 then advances the records' states in place.
 * states, when not NULL, receives what tq_selective_scan_grad starts from: float
 * [B, ceil(T / TQ_STATES_PIECE), S, D], the state before every step that is a
 * multiple of TQ_STATES_PIECE (past a record's length: not written).
 * TQ_E_UNSUPPORTED for S > 64, D > 2^20 or B ceil(D / 64) ceil(T / 64) >= 2^31
 * (T = 0 counts as 1). */
#define TQ_STATES_PIECE 16
tq_status tq_selective_scan_workspace(int64_t B, int64_t T, int64_t D, int64_t S, size_t *bytes);
tq_status tq_selective_scan(int32_t type, int64_t B, int64_t T, int64_t D, int64_t S, const void *x, int64_t x_batch,
                            int64_t x_step, const void *dt, int64_t dt_batch, int64_t dt_step, const float *A,
                            const void *Bm, int64_t B_batch, int64_t B_step, const void *Cm, int64_t C_batch,
                            int64_t C_step, const float *skip, const void *z, int64_t z_batch, int64_t z_step,
                            const float *dt_bias, const float *h0, const int32_t *lengths, void *y, int64_t y_batch,
                            int64_t y_step, float *h_last, float *states, void *workspace, size_t workspace_bytes,
                            void *stream);

/* Gradients of tq_selective_scan from dy, the gradient of y, and dh_last (NULL:
 * zeros), that of h_last.  With q_t = dy_t silu(z_t), a_t = exp(d_t A) and
 * l_t = C_t q_t + a_{t+1} l_{t+1} (dh_last in place of a l at the record's last step),
 *     dx_t = d_t sum_s B_t l_t + skip q_t,       dskip = sum_bt q_t x_t,
 *     dC_t = sum_d q_t h_t,                      dB_t = sum_d d_t x_t l_t,
 *     dd_t = sum_s (A a_t h_{t-1} + B_t x_t) l_t,  ddt_t = dd_t sigmoid(dt_t + dt_bias),
 *     dA = sum_bt d_t a_t h_{t-1} l_t,           ddt_bias = sum_bt ddt_t,
 *     dz_t = dy_t (sum_s C_t h_t + skip x_t) silu'(z_t),  dh0 = a_0 l_0;
 * dx, ddt, dz, dB and dC are zero past the record's length.  dx, ddt, dz [B, T, D]
 * and dB, dC [B, T, S] have the inputs' type and strides of their own; dA, dskip,
 * ddt_bias and dh0 are float as the tensors that they belong to.  dz goes with z;
 * dskip, ddt_bias and dh0 may be NULL: not wanted.  `states` are the ones that
 * tq_selective_scan wrote for the same inputs.  For D = 0 nothing is enqueued: dB and
 * dC, sums over no channels, are the caller's to clear. */
tq_status tq_selective_scan_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t S, size_t *bytes);
tq_status tq_selective_scan_grad(int32_t type, int64_t B, int64_t T, int64_t D, int64_t S, const void *x,
                                 int64_t x_batch, int64_t x_step, const void *dt, int64_t dt_batch, int64_t dt_step,
                                 const float *A, const void *Bm, int64_t B_batch, int64_t B_step, const void *Cm,
                                 int64_t C_batch, int64_t C_step, const float *skip, const void *z, int64_t z_batch,
                                 int64_t z_step, const float *dt_bias, const float *states, const int32_t *lengths,
                                 const void *dy, int64_t dy_batch, int64_t dy_step, const float *dh_last, void *dx,
                                 int64_t dx_batch, int64_t dx_step, void *ddt, int64_t ddt_batch, int64_t ddt_step,
                                 void *dz, int64_t dz_batch, int64_t dz_step, void *dB, int64_t dB_batch,
                                 int64_t dB_step, void *dC, int64_t dC_batch, int64_t dC_step, float *dA, float *dskip,
                                 float *ddt_bias, float *dh0, void *workspace, size_t workspace_bytes, void *stream);

/* The short causal convolution over time, channel by channel, of B records of T
 * steps with K taps (1 <= K <= 8):
 *     u_t = bias + sum_k weight[k] x_{t - K + 1 + k},   y_t = silu ? u_t sigmoid(u_t) : u_t
 * for t < lengths[b] (clamped to [0, T]; NULL: all T); past it y is zero and x is
 * not looked at.  x and y are [B, T, D] with strides of their own, weight [K, D],
 * bias [D] (NULL: zeros), all of `type`.  state [B, K - 1, D] (NULL: zeros) holds
 * the inputs before the first step, the latest one last, and last [B, K - 1, D]
 * (NULL: not wanted) receives the inputs before the step after the record's last
 * one; it may be `state` itself: records are then extended in place.
 * TQ_E_UNSUPPORTED for K > 8, D > 2^20 or B ceil(T / 8) ceil(D / 4) >= 2^31
 * (for D < 8: B ceil(T / 8) D). */
tq_status tq_causal_conv(int32_t type, int64_t B, int64_t T, int64_t D, int64_t K, const void *x, int64_t x_batch,
                         int64_t x_step, const void *weight, const void *bias, const void *state,
                         const int32_t *lengths, int32_t silu, void *y, int64_t y_batch, int64_t y_step, void *last,
                         void *stream);

/* Gradients of tq_causal_conv from dy, the gradient of y, and dlast (NULL:
 * zeros), that of last: with g_t = dy_t silu'(u_t) (or dy_t),
 *     dx_t = sum_k weight[k] g_{t + K - 1 - k}, dlast added to the record's last K - 1 inputs,
 *     dweight[k] = sum_bt g_t x_{t - K + 1 + k},   dbias = sum_bt g_t,
 * and dstate, the same as dx for the inputs that `state` holds; dx is zero past the
 * record's length.  All have the inputs' type; dbias and dstate may be NULL: not
 * wanted. */
tq_status tq_causal_conv_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t K, size_t *bytes);
tq_status tq_causal_conv_grad(int32_t type, int64_t B, int64_t T, int64_t D, int64_t K, const void *x, int64_t x_batch,
                              int64_t x_step, const void *weight, const void *bias, const void *state,
                              const int32_t *lengths, int32_t silu, const void *dy, int64_t dy_batch, int64_t dy_step,
                              const void *dlast, void *dx, int64_t dx_batch, int64_t dx_step, void *dweight,
                              void *dbias, void *dstate, void *workspace, size_t workspace_bytes, void *stream);

/* The norm of n tensors together, and the tensors cut to a largest one: with
 *     norm = scale (sum over all elements of grads[i]^2)^{1/2},
 *     outs[i] = grads[i] scale (norm <= max_norm ? 1 : max_norm / norm).
 * grads, outs, counts, types and out_types are HOST arrays of n entries, read
 * during the call: device pointers, numbers of elements and tq_dtypes.  outs[i] may
 * be grads[i] where both have one type, but no other one of them (a tensor that is
 * listed twice cannot be cut in place).  Squares are summed in 64 bits; norm, float on
 * the device, is written always, infinite where the norm is past the range of fp32;
 * the factor is formed from the norm in 64 bits.  An infinite norm above max_norm gives
 * zeros for finite elements and NaN for infinite ones, a norm of NaN gives NaN.
 * max_norm >= 0 (infinite: nothing is cut, the factor is `scale` for an infinite norm
 * too), scale > 0 and finite (1 over the factor that a loss was scaled by).
 * TQ_E_UNSUPPORTED for n >= 2^20 or a tensor of 2^40 elements. */
tq_status tq_clip_grad_norm_workspace(int64_t n, const int64_t *counts, size_t *bytes);
tq_status tq_clip_grad_norm(int64_t n, const void *const *grads, const int64_t *counts, const int32_t *types,
                            float max_norm, float scale, void *const *outs, const int32_t *out_types, float *norm,
                            void *workspace, size_t workspace_bytes, void *stream);

/* One step of a beam search over R records with W beams each (1 <= W <= 64) and
 * logits [R * W, V], rows ld_logits apart: a candidate is a beam w and the id v that
 * it goes on with, its score
 *     scores[r, w] + logits[r, w, v] - log sum_u exp logits[r, w, u],
 * formed in 64 bits.  The K best (1 <= K <= 64, K <= W V) of a record's W V
 * candidates are given, best first: out_scores float [R, K], parents int32 [R, K]
 * (w) and tokens [R, K] (v).  Candidates of one beam rank by their logits, those of
 * different beams by their scores; ties go to the lower beam, then the lower id.
 *  - `last` [R, W] (NULL: no beam has ended) holds the beams' latest ids: a beam whose
 *    latest id is `end` goes on with `end` at its present score and with nothing else;
 *    its logits are not looked at.  end < V where last is given.
 *  - A score that is not below infinity (NaN among them) counts as -infinity.  A beam
 *    whose score is -infinity is out of use: at the start of a search all but one.
 *    Candidates at -infinity, such as ids that a logit of -infinity rules out, are
 *    given only where there are no others; they rank by beam and id, those of a
 *    beam that has others by id behind these.
 * TQ_E_UNSUPPORTED for W or K > 64 or R W ceil(V / 2048) >= 2^31. */
tq_status tq_beam_select_workspace(int32_t type, int64_t R, int64_t W, int64_t V, int64_t K, size_t *bytes);
tq_status tq_beam_select(int32_t type, int64_t R, int64_t W, int64_t V, int64_t K, const void *logits,
                         int64_t ld_logits, const float *scores, const uint64_t *last, uint64_t end, float *out_scores,
                         int32_t *parents, uint64_t *tokens, void *workspace, size_t workspace_bytes, void *stream);

/* The states of the beams that a search goes on with, n tensors in one call:
 * outs[i][r, k] = ins[i][r, parents[r, k]] for rows of row_bytes[i] bytes, ins[i]
 * [R, W] and outs[i] [R, K] of them; zeros where a parent is not in [0, W).  ins,
 * outs and row_bytes are HOST arrays of n entries, read during the call; parents
 * int32 [R, K] lies on the device.  No outs[i] may be any of ins.  TQ_E_UNSUPPORTED
 * for n >= 2^20, R K >= 2^31, rows of 2^40 bytes or R K ceil(row_bytes / 8192) >= 2^33. */
tq_status tq_beam_reorder(int64_t n, const void *const *ins, void *const *outs, const int64_t *row_bytes, int64_t R,
                          int64_t W, int64_t K, const int32_t *parents, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TQ_MODEL_H */
