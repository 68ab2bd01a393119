// seq_abi.cpp -- the extern "C" entry points of tq_seq.h: every argument is
// checked here, on the host, before anything is enqueued.
#include <algorithm>

#include "abi_checks.h"
#include "seq.h"

using namespace tq;

namespace {

void check_scan(const char *call, int type, int64_t B, int64_t T, int64_t D)
{
    check_type(call, type);
    check_size(call, "B", B);
    check_size(call, "T", T);
    check_size(call, "D", D);
    if (D > kMaxWidth) fail(TQ_E_UNSUPPORTED, text(call, "D must be at most 2^20"));
    // rows x segments of 64 steps, in doubles: the product of three sizes
    if ((double)B * (double)((D + 63) / 64) * (double)((T + 63) / 64) > kMaxIndex ||
        scan_items(B, T, D) > kMaxIndex)
        fail(TQ_E_UNSUPPORTED, text(call, "B * ceil(D / 64) * ceil(T / 64) must be below 2^31"));
}

} // namespace

extern "C" {

tq_status tq_embed(const void *table, int64_t ld_table, int32_t type, int64_t V, int64_t D, const uint64_t *tokens,
                   int64_t N, float scale, void *out, int64_t ld_out, void *stream)
{
    return guarded([&] {
        const char *call = "embed";
        check_type(call, type);
        check_size(call, "V", V);
        check_size(call, "D", D);
        check_size(call, "N", N);
        if (N == 0 || D == 0) return;
        check_ld(call, "ld_table", ld_table, D);
        check_ld(call, "ld_out", ld_out, D);
        if (V) check_array(call, "table", table, size_of(type));
        check_array(call, "tokens", tokens, 8);
        check_array(call, "out", out, size_of(type));
        hip_check(launch_embed(type, {table, ld_table, V, D, tokens, N, scale, out, ld_out}, as_stream(stream)),
                  "embed launch");
    });
}

tq_status tq_embed_grad_workspace(int64_t V, int64_t D, int64_t N, size_t *bytes)
{
    return guarded([&] {
        const char *call = "embed_grad_workspace";
        check_size(call, "V", V);
        check_size(call, "D", D);
        check_size(call, "N", N);
        if (D > kMaxWidth) fail(TQ_E_UNSUPPORTED, text(call, "D must be at most 2^20"));
        give(bytes, V && D ? embed_grad_workspace(V, D, N) : 0);
    });
}

tq_status tq_embed_grad(const void *grad_out, int64_t ld_grad_out, int32_t type, int64_t V, int64_t D,
                        const uint64_t *tokens, int64_t N, float scale, void *grad, int64_t ld_grad, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "embed_grad";
        check_type(call, type);
        check_size(call, "V", V);
        check_size(call, "D", D);
        check_size(call, "N", N);
        if (D > kMaxWidth) fail(TQ_E_UNSUPPORTED, text(call, "D must be at most 2^20"));
        if (V == 0 || D == 0) return;
        check_ld(call, "ld_grad", ld_grad, D);
        check_array(call, "grad", grad, size_of(type));
        if (N) {
            check_ld(call, "ld_grad_out", ld_grad_out, D);
            check_array(call, "grad_out", grad_out, size_of(type));
            check_array(call, "tokens", tokens, 8);
        }
        check_space(call, workspace, workspace_bytes, embed_grad_workspace(V, D, N));
        hip_check(launch_embed_grad(type, {grad_out, ld_grad_out, V, D, tokens, N, scale, grad, ld_grad, workspace},
                                    as_stream(stream)),
                  "embed gradient launch");
    });
}

tq_status tq_gated_scan_workspace(int64_t B, int64_t T, int64_t D, size_t *bytes)
{
    return guarded([&] {
        check_scan("gated_scan_workspace", TQ_F32, B, T, D);
        give(bytes, B && D ? scan_workspace(B, T, D) : 0);
    });
}

tq_status tq_gated_scan(int32_t type, int64_t B, int64_t T, int64_t D, const void *x, int64_t x_batch, int64_t x_step,
                        const void *g, int64_t g_batch, int64_t g_step, const float *h0, const int32_t *lengths,
                        void *y, int64_t y_batch, int64_t y_step, float *h_last, float *states, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "gated_scan";
        check_scan(call, type, B, T, D);
        if (B == 0 || D == 0) return;
        const size_t e = size_of(type);
        if (T) {
            check_strides(call, "x", B, T, D, x_batch, x_step, false);
            check_strides(call, "g", B, T, D, g_batch, g_step, false);
            check_strides(call, "y", B, T, D, y_batch, y_step, true);
            check_array(call, "x", x, e);
            check_array(call, "g", g, e);
            check_array(call, "y", y, e);
        }
        check_maybe("h0", h0, 4);
        check_maybe("lengths", lengths, 4);
        check_maybe("h_last", h_last, 4);
        check_maybe("states", states, 4);
        check_space(call, workspace, workspace_bytes, scan_workspace(B, T, D));
        ScanArgs a{};
        a.B = B, a.T = T, a.D = D;
        a.x = x, a.xb = x_batch, a.xs = x_step;
        a.g = g, a.gb = g_batch, a.gs = g_step;
        a.y = y, a.yb = y_batch, a.ys = y_step;
        a.h0 = h0, a.lengths = lengths, a.h_last = h_last, a.states = states, a.ws = workspace;
        hip_check(launch_scan(type, a, as_stream(stream)), "gated scan launch");
    });
}

tq_status tq_gated_scan_grad(int32_t type, int64_t B, int64_t T, int64_t D, const void *x, int64_t x_batch,
                             int64_t x_step, const void *g, int64_t g_batch, int64_t g_step, const float *states,
                             const int32_t *lengths, const void *dy, int64_t dy_batch, int64_t dy_step,
                             const float *dh_last, void *dx, int64_t dx_batch, int64_t dx_step, void *dg,
                             int64_t dg_batch, int64_t dg_step, float *dh0, void *workspace, size_t workspace_bytes,
                             void *stream)
{
    return guarded([&] {
        const char *call = "gated_scan_grad";
        check_scan(call, type, B, T, D);
        if (B == 0 || D == 0) return;
        const size_t e = size_of(type);
        if (T) {
            check_strides(call, "x", B, T, D, x_batch, x_step, false);
            check_strides(call, "g", B, T, D, g_batch, g_step, false);
            check_strides(call, "dy", B, T, D, dy_batch, dy_step, false);
            check_strides(call, "dx", B, T, D, dx_batch, dx_step, true);
            check_strides(call, "dg", B, T, D, dg_batch, dg_step, true);
            check_array(call, "x", x, e);
            check_array(call, "g", g, e);
            check_array(call, "dy", dy, e);
            check_array(call, "dx", dx, e);
            check_array(call, "dg", dg, e);
            check_array(call, "states", states, 4);
        }
        check_maybe("lengths", lengths, 4);
        check_maybe("dh_last", dh_last, 4);
        check_maybe("dh0", dh0, 4);
        check_space(call, workspace, workspace_bytes, scan_workspace(B, T, D));
        ScanArgs a{};
        a.B = B, a.T = T, a.D = D;
        a.x = x, a.xb = x_batch, a.xs = x_step;
        a.g = g, a.gb = g_batch, a.gs = g_step;
        a.dy = dy, a.dyb = dy_batch, a.dys = dy_step;
        a.dx = dx, a.dxb = dx_batch, a.dxs = dx_step;
        a.dg = dg, a.dgb = dg_batch, a.dgs = dg_step;
        a.states_in = states, a.lengths = lengths, a.dh_last = dh_last, a.dh0 = dh0, a.ws = workspace;
        hip_check(launch_scan_grad(type, a, as_stream(stream)), "gated scan gradient launch");
    });
}

tq_status tq_layer_norm(const void *x, int64_t ld_x, int32_t type, int64_t N, int64_t D, const void *weight,
                        const void *bias, float eps, void *y, int64_t ld_y, float *mean, float *rstd, void *stream)
{
    return guarded([&] {
        const char *call = "layer_norm";
        check_type(call, type);
        check_size(call, "N", N);
        check_size(call, "D", D);
        if (!(eps >= 0.f)) fail(TQ_E_INVALID, text(call, "eps must not be negative"));
        if (!mean != !rstd) fail(TQ_E_INVALID, text(call, "mean and rstd are kept together"));
        if (N == 0 || D == 0) return;
        const size_t e = size_of(type);
        check_ld(call, "ld_x", ld_x, D);
        check_ld(call, "ld_y", ld_y, D);
        check_array(call, "x", x, e);
        check_array(call, "weight", weight, e);
        check_maybe("bias", bias, e);
        check_array(call, "y", y, e);
        check_maybe("mean", mean, 4);
        check_maybe("rstd", rstd, 4);
        NormArgs a{};
        a.x = x, a.ld_x = ld_x, a.N = N, a.D = D, a.weight = weight, a.bias = bias, a.eps = eps;
        a.y = y, a.ld_y = ld_y, a.mean = mean, a.rstd = rstd;
        hip_check(launch_norm(type, a, as_stream(stream)), "layer norm launch");
    });
}

tq_status tq_layer_norm_grad_workspace(int64_t N, int64_t D, size_t *bytes)
{
    return guarded([&] {
        const char *call = "layer_norm_grad_workspace";
        check_size(call, "N", N);
        check_size(call, "D", D);
        give(bytes, norm_grad_workspace(N, D));
    });
}

tq_status tq_layer_norm_grad(const void *x, int64_t ld_x, int32_t type, int64_t N, int64_t D, const void *weight,
                             const float *mean, const float *rstd, const void *dy, int64_t ld_dy, void *dx,
                             int64_t ld_dx, void *dweight, void *dbias, void *workspace, size_t workspace_bytes,
                             void *stream)
{
    return guarded([&] {
        const char *call = "layer_norm_grad";
        check_type(call, type);
        check_size(call, "N", N);
        check_size(call, "D", D);
        if (D == 0) return;
        const size_t e = size_of(type);
        check_array(call, "weight", weight, e);
        check_array(call, "dweight", dweight, e);
        check_maybe("dbias", dbias, e);
        if (N) {
            check_ld(call, "ld_x", ld_x, D);
            check_ld(call, "ld_dy", ld_dy, D);
            check_ld(call, "ld_dx", ld_dx, D);
            check_array(call, "x", x, e);
            check_array(call, "dy", dy, e);
            check_array(call, "dx", dx, e);
            check_array(call, "mean", mean, 4);
            check_array(call, "rstd", rstd, 4);
        }
        check_space(call, workspace, workspace_bytes, norm_grad_workspace(N, D));
        NormArgs a{};
        a.x = x, a.ld_x = ld_x, a.N = N, a.D = D, a.weight = weight, a.mean_in = mean, a.rstd_in = rstd;
        a.dy = dy, a.ld_dy = ld_dy, a.dx = dx, a.ld_dx = ld_dx, a.dweight = dweight, a.dbias = dbias;
        a.ws = workspace;
        hip_check(launch_norm_grad(type, a, as_stream(stream)), "layer norm gradient launch");
    });
}

static void check_xent(const char *call, int type, int64_t N, int64_t V, int64_t D)
{
    check_type(call, type);
    check_size(call, "N", N);
    check_size(call, "V", V);
    check_size(call, "D", D);
    if (N && V == 0) fail(TQ_E_INVALID, text(call, "a vocabulary needs one row at least"));
    if (D > kMaxWidth) fail(TQ_E_UNSUPPORTED, text(call, "D must be at most 2^20"));
    // tiles of 128 x 128 of the logits and of the gradients
    const auto tiles = [](int64_t n) { return (n + 127) / 128; };
    if (tiles(N) * tiles(V) > kMaxIndex / 16 || std::max(tiles(N), tiles(V)) * tiles(D) > kMaxIndex / 16)
        fail(TQ_E_UNSUPPORTED, text(call, "ceil(N / 128) * ceil(V / 128), and either times ceil(D / 128), must be below 2^27"));
}

tq_status tq_softmax_xent_workspace(int32_t type, int64_t N, int64_t V, int64_t D, size_t *bytes)
{
    return guarded([&] {
        check_xent("softmax_xent_workspace", type, N, V, D);
        give(bytes, N ? xent_workspace(type, N, V, D, false) : 0);
    });
}

tq_status tq_softmax_xent_grad_workspace(int32_t type, int64_t N, int64_t V, int64_t D, size_t *bytes)
{
    return guarded([&] {
        check_xent("softmax_xent_grad_workspace", type, N, V, D);
        give(bytes, V ? xent_workspace(type, N, V, D, true) : 0);
    });
}

tq_status tq_softmax_xent(const void *hidden, int64_t ld_hidden, int32_t type, int64_t N, int64_t V, int64_t D,
                          const void *weight, int64_t ld_weight, const uint64_t *targets, float *loss, float *lse,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "softmax_xent";
        check_xent(call, type, N, V, D);
        if (N == 0) return;
        const size_t e = size_of(type);
        if (D) {
            check_ld(call, "ld_hidden", ld_hidden, D);
            check_ld(call, "ld_weight", ld_weight, D);
            check_array(call, "hidden", hidden, e);
            check_array(call, "weight", weight, e);
        }
        check_array(call, "targets", targets, 8);
        check_array(call, "loss", loss, 4);
        check_array(call, "lse", lse, 4);
        check_space(call, workspace, workspace_bytes, xent_workspace(type, N, V, D, false));
        XentArgs a{};
        a.hidden = hidden, a.ld_hidden = ld_hidden, a.weight = weight, a.ld_weight = ld_weight;
        a.N = N, a.V = V, a.D = D, a.targets = targets, a.loss = loss, a.lse = lse, a.ws = workspace;
        hip_check(launch_xent(type, a, false, as_stream(stream)), "softmax cross entropy launch");
    });
}

tq_status tq_softmax_xent_grad(const void *hidden, int64_t ld_hidden, int32_t type, int64_t N, int64_t V, int64_t D,
                               const void *weight, int64_t ld_weight, const uint64_t *targets, const float *upstream,
                               void *dhidden, int64_t ld_dhidden, void *dweight, int64_t ld_dweight, float *loss,
                               float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    return guarded([&] {
        const char *call = "softmax_xent_grad";
        check_xent(call, type, N, V, D);
        if (V == 0) return;
        const size_t e = size_of(type);
        if (D) {
            check_ld(call, "ld_weight", ld_weight, D);
            check_ld(call, "ld_dweight", ld_dweight, D);
            check_array(call, "weight", weight, e);
            check_array(call, "dweight", dweight, e);
        }
        if (N) {
            check_array(call, "targets", targets, 8);
            check_array(call, "upstream", upstream, 4);
            check_array(call, "loss", loss, 4);
            check_array(call, "lse", lse, 4);
            if (D) {
                check_ld(call, "ld_hidden", ld_hidden, D);
                check_ld(call, "ld_dhidden", ld_dhidden, D);
                check_array(call, "hidden", hidden, e);
                check_array(call, "dhidden", dhidden, e);
            }
        }
        check_space(call, workspace, workspace_bytes, xent_workspace(type, N, V, D, true));
        XentArgs a{};
        a.hidden = hidden, a.ld_hidden = ld_hidden, a.weight = weight, a.ld_weight = ld_weight;
        a.N = N, a.V = V, a.D = D, a.targets = targets, a.loss = loss, a.lse = lse, a.ws = workspace;
        a.upstream = upstream, a.dhidden = dhidden, a.ld_dhidden = ld_dhidden;
        a.dweight = dweight, a.ld_dweight = ld_dweight;
        hip_check(launch_xent(type, a, true, as_stream(stream)), "softmax cross entropy gradient launch");
    });
}

} // extern "C"
