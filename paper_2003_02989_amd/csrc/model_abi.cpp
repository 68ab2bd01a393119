// model_abi.cpp -- the extern "C" entry points of tq_model.h: every argument is
// checked here, on the host, before anything is enqueued.
#include <algorithm>
#include <cmath>
#include <utility>
#include <vector>

#include "abi_checks.h"
#include "model.h"

using namespace tq;

namespace {

constexpr int64_t kMaxStates = 64, kMaxTaps = 8, kMaxBeams = 64;

void check_select(const char *call, int type, int64_t B, int64_t T, int64_t D, int64_t S)
{
    check_type(call, type);
    check_size(call, "B", B);
    check_size(call, "T", T);
    check_size(call, "D", D);
    if (S < 1) fail(TQ_E_INVALID, text(call, "a channel needs one state at least"));
    if (S > kMaxStates) fail(TQ_E_UNSUPPORTED, text(call, "S must be at most 64"));
    if (D > kMaxWidth) fail(TQ_E_UNSUPPORTED, text(call, "D must be at most 2^20"));
    // in doubles: the product of three sizes; records of no steps have their states
    if ((double)B * (double)((D + 63) / 64) * (double)((std::max<int64_t>(T, 1) + 63) / 64) > kMaxIndex)
        fail(TQ_E_UNSUPPORTED, text(call, "B * ceil(D / 64) * ceil(T / 64) must be below 2^31"));
}

void check_steps(const char *call, const char *name, int64_t B, int64_t T, int64_t D, const Steps &s, size_t align)
{
    check_strides(call, name, B, T, D, s.batch, s.step, false);
    check_array(call, name, s.p, align);
}

void check_steps(const char *call, const char *name, int64_t B, int64_t T, int64_t D, const StepsOut &s, size_t align)
{
    check_strides(call, name, B, T, D, s.batch, s.step, true);
    check_array(call, name, s.p, align);
}

void check_conv(const char *call, int type, int64_t B, int64_t T, int64_t D, int64_t K)
{
    check_type(call, type);
    check_size(call, "B", B);
    check_size(call, "T", T);
    check_size(call, "D", D);
    if (K < 1) fail(TQ_E_INVALID, text(call, "a convolution needs one tap at least"));
    if (K > kMaxTaps) fail(TQ_E_UNSUPPORTED, text(call, "K must be at most 8"));
    if (D > kMaxWidth) fail(TQ_E_UNSUPPORTED, text(call, "D must be at most 2^20"));
    if (conv_items(B, T, D) > kMaxIndex || conv_items(B, 1, D) > kMaxIndex)
        fail(TQ_E_UNSUPPORTED, text(call, "B * ceil(T / 8) * ceil(D / 4), for D < 8 times D, must be below 2^31"));
}

void check_list(const char *call, int64_t n)
{
    if (n < 0) fail(TQ_E_INVALID, text(call, "n must not be negative"));
    if (n >= 1 << 20) fail(TQ_E_UNSUPPORTED, text(call, "n must be below 2^20"));
}

void check_counts(const char *call, const char *name, int64_t n, const int64_t *counts)
{
    if (n && !counts) fail(TQ_E_INVALID, text(call, name) + " is NULL");
    for (int64_t i = 0; i < n; i++) {
        if (counts[i] < 0) fail(TQ_E_INVALID, text(call, name) + " must not be negative");
        if (counts[i] >= (int64_t)1 << 40) fail(TQ_E_UNSUPPORTED, text(call, name) + " must be below 2^40");
    }
}

// Outputs may be their own inputs at most: one that is another entry's input is
// written while that is read.
void check_own(const char *call, int64_t n, const void *const *ins, void *const *outs, const int64_t *sizes)
{
    std::vector<std::pair<const void *, int64_t>> at;
    at.reserve(n);
    for (int64_t i = 0; i < n; i++)
        if (sizes[i]) at.emplace_back(ins[i], i);
    std::sort(at.begin(), at.end());
    for (int64_t i = 0; i < n; i++) {
        if (sizes[i] == 0) continue;
        auto k = std::lower_bound(at.begin(), at.end(), std::pair<const void *, int64_t>(outs[i], 0));
        for (; k != at.end() && k->first == outs[i]; ++k)
            if (k->second != i) fail(TQ_E_INVALID, text(call, "an output is another entry's input"));
    }
}

void check_beam(const char *call, int type, int64_t R, int64_t W, int64_t V, int64_t K)
{
    check_type(call, type);
    check_size(call, "R", R);
    check_size(call, "V", V);
    if (W < 1 || K < 1 || V < 1) fail(TQ_E_INVALID, text(call, "W, V and K must be positive"));
    if (W > kMaxBeams || K > kMaxBeams) fail(TQ_E_UNSUPPORTED, text(call, "W and K must be at most 64"));
    if (K > W * V) fail(TQ_E_INVALID, text(call, "there are fewer than K candidates"));
    if ((double)R * (double)W * (double)((V + 2047) / 2048) > kMaxIndex)
        fail(TQ_E_UNSUPPORTED, text(call, "R * W * ceil(V / 2048) must be below 2^31"));
}

} // namespace

extern "C" {

tq_status tq_selective_scan_workspace(int64_t B, int64_t T, int64_t D, int64_t S, size_t *bytes)
{
    return guarded([&] {
        check_select("selective_scan_workspace", TQ_F32, B, T, D, S);
        give(bytes, B && D ? select_workspace(B, T, D, S) : 0);
    });
}

tq_status tq_selective_scan_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t S, size_t *bytes)
{
    return guarded([&] {
        check_select("selective_scan_grad_workspace", TQ_F32, B, T, D, S);
        give(bytes, D ? select_grad_workspace(B, T, D, S) : 0);
    });
}

tq_status tq_selective_scan(int32_t type, int64_t B, int64_t T, int64_t D, int64_t S, const void *x, int64_t x_batch,
                            int64_t x_step, const void *dt, int64_t dt_batch, int64_t dt_step, const float *A,
                            const void *Bm, int64_t B_batch, int64_t B_step, const void *Cm, int64_t C_batch,
                            int64_t C_step, const float *skip, const void *z, int64_t z_batch, int64_t z_step,
                            const float *dt_bias, const float *h0, const int32_t *lengths, void *y, int64_t y_batch,
                            int64_t y_step, float *h_last, float *states, void *workspace, size_t workspace_bytes,
                            void *stream)
{
    return guarded([&] {
        const char *call = "selective_scan";
        check_select(call, type, B, T, D, S);
        if (B == 0 || D == 0) return;
        const size_t e = size_of(type);
        SelectArgs a{};
        a.B = B, a.T = T, a.D = D, a.S = (int)S;
        a.x = {x, x_batch, x_step}, a.dt = {dt, dt_batch, dt_step}, a.z = {z, z_batch, z_step};
        a.Bm = {Bm, B_batch, B_step}, a.Cm = {Cm, C_batch, C_step}, a.y = {y, y_batch, y_step};
        if (T) {
            check_steps(call, "x", B, T, D, a.x, e);
            check_steps(call, "dt", B, T, D, a.dt, e);
            check_steps(call, "B", B, T, S, a.Bm, e);
            check_steps(call, "C", B, T, S, a.Cm, e);
            if (z) check_steps(call, "z", B, T, D, a.z, e);
            check_steps(call, "y", B, T, D, a.y, e);
            check_array(call, "A", A, 4);
        }
        check_maybe("skip", skip, 4);
        check_maybe("dt_bias", dt_bias, 4);
        check_maybe("h0", h0, 4);
        check_maybe("lengths", lengths, 4);
        check_maybe("h_last", h_last, 4);
        check_maybe("states", states, 4);
        check_space(call, workspace, workspace_bytes, select_workspace(B, T, D, S));
        a.A = A, a.skip = skip, a.dt_bias = dt_bias, a.h0 = h0, a.lengths = lengths;
        a.h_last = h_last, a.states = states, a.ws = workspace;
        hip_check(launch_select(type, a, as_stream(stream)), "selective scan launch");
    });
}

tq_status tq_selective_scan_grad(int32_t type, int64_t B, int64_t T, int64_t D, int64_t S, const void *x,
                                 int64_t x_batch, int64_t x_step, const void *dt, int64_t dt_batch, int64_t dt_step,
                                 const float *A, const void *Bm, int64_t B_batch, int64_t B_step, const void *Cm,
                                 int64_t C_batch, int64_t C_step, const float *skip, const void *z, int64_t z_batch,
                                 int64_t z_step, const float *dt_bias, const float *states, const int32_t *lengths,
                                 const void *dy, int64_t dy_batch, int64_t dy_step, const float *dh_last, void *dx,
                                 int64_t dx_batch, int64_t dx_step, void *ddt, int64_t ddt_batch, int64_t ddt_step,
                                 void *dz, int64_t dz_batch, int64_t dz_step, void *dB, int64_t dB_batch,
                                 int64_t dB_step, void *dC, int64_t dC_batch, int64_t dC_step, float *dA, float *dskip,
                                 float *ddt_bias, float *dh0, void *workspace, size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "selective_scan_grad";
        check_select(call, type, B, T, D, S);
        if (D == 0) return;
        const size_t e = size_of(type);
        SelectArgs a{};
        a.B = B, a.T = T, a.D = D, a.S = (int)S;
        a.x = {x, x_batch, x_step}, a.dt = {dt, dt_batch, dt_step}, a.z = {z, z_batch, z_step};
        a.Bm = {Bm, B_batch, B_step}, a.Cm = {Cm, C_batch, C_step}, a.dy = {dy, dy_batch, dy_step};
        a.dx = {dx, dx_batch, dx_step}, a.ddt = {ddt, ddt_batch, ddt_step}, a.dz = {dz, dz_batch, dz_step};
        a.dB = {dB, dB_batch, dB_step}, a.dC = {dC, dC_batch, dC_step};
        if (B && T) {
            check_steps(call, "x", B, T, D, a.x, e);
            check_steps(call, "dt", B, T, D, a.dt, e);
            check_steps(call, "B", B, T, S, a.Bm, e);
            check_steps(call, "C", B, T, S, a.Cm, e);
            if (!z != !dz) fail(TQ_E_INVALID, text(call, "dz goes with z"));
            if (z) check_steps(call, "z", B, T, D, a.z, e);
            if (z) check_steps(call, "dz", B, T, D, a.dz, e);
            check_steps(call, "dy", B, T, D, a.dy, e);
            check_steps(call, "dx", B, T, D, a.dx, e);
            check_steps(call, "ddt", B, T, D, a.ddt, e);
            check_steps(call, "dB", B, T, S, a.dB, e);
            check_steps(call, "dC", B, T, S, a.dC, e);
            check_array(call, "A", A, 4);
            check_array(call, "states", states, 4);
        }
        check_array(call, "dA", dA, 4);
        check_maybe("skip", skip, 4);
        check_maybe("dt_bias", dt_bias, 4);
        check_maybe("lengths", lengths, 4);
        check_maybe("dh_last", dh_last, 4);
        check_maybe("dskip", dskip, 4);
        check_maybe("ddt_bias", ddt_bias, 4);
        check_maybe("dh0", dh0, 4);
        check_space(call, workspace, workspace_bytes, select_grad_workspace(B, T, D, S));
        a.A = A, a.skip = skip, a.dt_bias = dt_bias, a.states_in = states, a.lengths = lengths, a.dh_last = dh_last;
        a.dA = dA, a.dskip = dskip, a.ddt_bias = ddt_bias, a.dh0 = dh0, a.ws = workspace;
        hip_check(launch_select_grad(type, a, as_stream(stream)), "selective scan gradient launch");
    });
}

tq_status tq_causal_conv(int32_t type, int64_t B, int64_t T, int64_t D, int64_t K, const void *x, int64_t x_batch,
                         int64_t x_step, const void *weight, const void *bias, const void *state,
                         const int32_t *lengths, int32_t silu, void *y, int64_t y_batch, int64_t y_step, void *last,
                         void *stream)
{
    return guarded([&] {
        const char *call = "causal_conv";
        check_conv(call, type, B, T, D, K);
        if (B == 0 || D == 0) return;
        const size_t e = size_of(type);
        ConvArgs a{};
        a.B = B, a.T = T, a.D = D, a.K = K;
        a.x = {x, x_batch, x_step}, a.y = {y, y_batch, y_step};
        check_array(call, "weight", weight, e);
        if (T) {
            check_steps(call, "x", B, T, D, a.x, e);
            check_steps(call, "y", B, T, D, a.y, e);
        }
        check_maybe("bias", bias, e);
        check_maybe("state", state, e);
        check_maybe("lengths", lengths, 4);
        check_maybe("last", last, e);
        a.weight = weight, a.bias = bias, a.state = state, a.lengths = lengths, a.silu = silu != 0, a.last = last;
        hip_check(launch_conv(type, a, as_stream(stream)), "causal convolution launch");
    });
}

tq_status tq_causal_conv_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t K, size_t *bytes)
{
    return guarded([&] {
        check_conv("causal_conv_grad_workspace", TQ_F32, B, T, D, K);
        give(bytes, D ? conv_grad_workspace(B, T, D, K) : 0);
    });
}

tq_status tq_causal_conv_grad(int32_t type, int64_t B, int64_t T, int64_t D, int64_t K, const void *x, int64_t x_batch,
                              int64_t x_step, const void *weight, const void *bias, const void *state,
                              const int32_t *lengths, int32_t silu, const void *dy, int64_t dy_batch, int64_t dy_step,
                              const void *dlast, void *dx, int64_t dx_batch, int64_t dx_step, void *dweight,
                              void *dbias, void *dstate, void *workspace, size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "causal_conv_grad";
        check_conv(call, type, B, T, D, K);
        if (D == 0) return;
        const size_t e = size_of(type);
        ConvArgs a{};
        a.B = B, a.T = T, a.D = D, a.K = K;
        a.x = {x, x_batch, x_step}, a.dy = {dy, dy_batch, dy_step}, a.dx = {dx, dx_batch, dx_step};
        check_array(call, "weight", weight, e);
        check_array(call, "dweight", dweight, e);
        if (B && T) {
            check_steps(call, "x", B, T, D, a.x, e);
            check_steps(call, "dy", B, T, D, a.dy, e);
            check_steps(call, "dx", B, T, D, a.dx, e);
        }
        check_maybe("bias", bias, e);
        check_maybe("state", state, e);
        check_maybe("lengths", lengths, 4);
        check_maybe("dlast", dlast, e);
        check_maybe("dbias", dbias, e);
        check_maybe("dstate", dstate, e);
        check_space(call, workspace, workspace_bytes, conv_grad_workspace(B, T, D, K));
        a.weight = weight, a.bias = bias, a.state = state, a.lengths = lengths, a.silu = silu != 0, a.dlast = dlast;
        a.dweight = dweight, a.dbias = dbias, a.dstate = dstate, a.ws = workspace;
        hip_check(launch_conv_grad(type, a, as_stream(stream)), "causal convolution gradient launch");
    });
}

tq_status tq_clip_grad_norm_workspace(int64_t n, const int64_t *counts, size_t *bytes)
{
    return guarded([&] {
        const char *call = "clip_grad_norm_workspace";
        check_list(call, n);
        check_counts(call, "counts", n, counts);
        give(bytes, clip_workspace(n, counts));
    });
}

tq_status tq_clip_grad_norm(int64_t n, const void *const *grads, const int64_t *counts, const int32_t *types,
                            float max_norm, float scale, void *const *outs, const int32_t *out_types, float *norm,
                            void *workspace, size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "clip_grad_norm";
        check_list(call, n);
        check_counts(call, "counts", n, counts);
        if (!(max_norm >= 0.f)) fail(TQ_E_INVALID, text(call, "max_norm must not be negative"));
        if (!(scale > 0.f && std::isfinite(scale))) fail(TQ_E_INVALID, text(call, "scale must be positive and finite"));
        if (n && (!grads || !types || !outs || !out_types)) fail(TQ_E_INVALID, text(call, "a list is NULL"));
        for (int64_t i = 0; i < n; i++) {
            check_type(call, types[i]);
            check_type(call, out_types[i]);
            if (counts[i] == 0) continue;
            check_array(call, "grads", grads[i], size_of(types[i]));
            check_array(call, "outs", outs[i], size_of(out_types[i]));
            if (grads[i] == outs[i] && types[i] != out_types[i])
                fail(TQ_E_INVALID, text(call, "a tensor in place keeps its type"));
        }
        check_own(call, n, grads, outs, counts);
        check_array(call, "norm", norm, 4);
        check_space(call, workspace, workspace_bytes, clip_workspace(n, counts));
        hip_check(launch_clip({n, grads, outs, counts, types, out_types, max_norm, scale, norm, workspace},
                              as_stream(stream)),
                  "gradient clipping launch");
    });
}

tq_status tq_beam_select_workspace(int32_t type, int64_t R, int64_t W, int64_t V, int64_t K, size_t *bytes)
{
    return guarded([&] {
        check_beam("beam_select_workspace", type, R, W, V, K);
        give(bytes, beam_workspace(type, R, W, V, K));
    });
}

tq_status tq_beam_select(int32_t type, int64_t R, int64_t W, int64_t V, int64_t K, const void *logits,
                         int64_t ld_logits, const float *scores, const uint64_t *last, uint64_t end, float *out_scores,
                         int32_t *parents, uint64_t *tokens, void *workspace, size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "beam_select";
        check_beam(call, type, R, W, V, K);
        if (R == 0) return;
        check_ld(call, "ld_logits", ld_logits, V);
        check_array(call, "logits", logits, size_of(type));
        check_array(call, "scores", scores, 4);
        check_maybe("last", last, 8);
        if (last && end >= (uint64_t)V) fail(TQ_E_INVALID, text(call, "end must be an id below V"));
        check_array(call, "out_scores", out_scores, 4);
        check_array(call, "parents", parents, 4);
        check_array(call, "tokens", tokens, 8);
        check_space(call, workspace, workspace_bytes, beam_workspace(type, R, W, V, K));
        BeamArgs a{};
        a.R = R, a.W = W, a.V = V, a.K = K, a.logits = logits, a.ld = ld_logits, a.scores = scores, a.last = last;
        a.end = end, a.out_scores = out_scores, a.parents = parents, a.tokens = tokens, a.ws = workspace;
        hip_check(launch_beam(type, a, as_stream(stream)), "beam selection launch");
    });
}

tq_status tq_beam_reorder(int64_t n, const void *const *ins, void *const *outs, const int64_t *row_bytes, int64_t R,
                          int64_t W, int64_t K, const int32_t *parents, void *stream)
{
    return guarded([&] {
        const char *call = "beam_reorder";
        check_list(call, n);
        check_counts(call, "row_bytes", n, row_bytes);
        check_size(call, "R", R);
        check_size(call, "W", W);
        check_size(call, "K", K);
        if ((double)R * (double)K > kMaxIndex) fail(TQ_E_UNSUPPORTED, text(call, "R * K must be below 2^31"));
        if (n == 0 || R == 0 || K == 0) return;
        if (!ins || !outs) fail(TQ_E_INVALID, text(call, "a list is NULL"));
        for (int64_t i = 0; i < n; i++) {
            if (row_bytes[i] == 0) continue;
            if ((double)R * (double)K * (double)((row_bytes[i] + 8191) / 8192) >= (double)((int64_t)1 << 33))
                fail(TQ_E_UNSUPPORTED, text(call, "R * K * ceil(row_bytes / 8192) must be below 2^33"));
            if (W) check_array(call, "ins", ins[i], 1);
            check_array(call, "outs", outs[i], 1);
            if (ins[i] == outs[i]) fail(TQ_E_INVALID, text(call, "rows are not reordered in place"));
        }
        if (W) check_own(call, n, ins, outs, row_bytes);
        check_array(call, "parents", parents, 4);
        hip_check(launch_reorder({n, R, W, K, ins, outs, row_bytes, parents}, as_stream(stream)), "beam reorder launch");
    });
}

} // extern "C"
