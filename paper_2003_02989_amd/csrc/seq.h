// seq.h -- launchers of the sequence kernels; arguments are checked by the
// callers (seq_abi.cpp).
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/tq_seq.h"

namespace tq {

// Workspaces are carved from one allocation in 256-byte steps.
struct Carver {
    size_t used = 0;
    size_t take(size_t bytes)
    {
        const size_t at = used;
        used += (bytes + 255) & ~(size_t)255;
        return at;
    }
};

struct EmbedArgs {
    const void *table;
    int64_t ld_table, V, D;
    const uint64_t *tokens;
    int64_t N;
    float scale;
    void *out;
    int64_t ld_out;
};
hipError_t launch_embed(int32_t type, const EmbedArgs &a, hipStream_t s);

struct EmbedGradArgs {
    const void *dout;
    int64_t ld_dout, V, D;
    const uint64_t *tokens;
    int64_t N;
    float scale;
    void *grad;
    int64_t ld_grad;
    void *ws;
};
size_t embed_grad_workspace(int64_t V, int64_t D, int64_t N);
hipError_t launch_embed_grad(int32_t type, const EmbedGradArgs &a, hipStream_t s);

struct ScanArgs {
    int64_t B, T, D;
    const void *x, *g, *dy;
    void *y, *dx, *dg;
    int64_t xb, xs, gb, gs, yb, ys, dyb, dys, dxb, dxs, dgb, dgs;
    const float *h0, *dh_last;
    float *h_last, *states, *dh0;
    const float *states_in;
    const int32_t *lengths;
    void *ws;
};
// workgroups of a scan (below 2^31), whatever the type
int64_t scan_items(int64_t B, int64_t T, int64_t D);
size_t scan_workspace(int64_t B, int64_t T, int64_t D);
hipError_t launch_scan(int32_t type, const ScanArgs &a, hipStream_t s);
hipError_t launch_scan_grad(int32_t type, const ScanArgs &a, hipStream_t s);

struct NormArgs {
    const void *x, *weight, *bias, *dy;
    int64_t ld_x, ld_y, ld_dy, ld_dx, N, D;
    float eps;
    void *y, *dx, *dweight, *dbias;
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    void *ws;
};
size_t norm_grad_workspace(int64_t N, int64_t D);
hipError_t launch_norm(int32_t type, const NormArgs &a, hipStream_t s);
hipError_t launch_norm_grad(int32_t type, const NormArgs &a, hipStream_t s);

struct XentArgs {
    const void *hidden, *weight;
    int64_t ld_hidden, ld_weight, N, V, D;
    const uint64_t *targets;
    const float *upstream;
    void *dhidden, *dweight;
    int64_t ld_dhidden, ld_dweight;
    float *loss, *lse;
    void *ws;
};
size_t xent_workspace(int32_t type, int64_t N, int64_t V, int64_t D, bool grad);
hipError_t launch_xent(int32_t type, const XentArgs &a, bool grad, hipStream_t s);

} // namespace tq
