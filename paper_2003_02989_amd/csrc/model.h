// model.h -- launchers of the kernels of selective models; arguments are checked
// by the callers (model_abi.cpp).
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/tq_model.h"

namespace tq {

// An array of steps: element c of step t of record b at p + b batch + t step + c.
struct Steps {
    const void *p;
    int64_t batch, step;
};
struct StepsOut {
    void *p;
    int64_t batch, step;
};

struct SelectArgs {
    int64_t B, T, D;
    int S;
    Steps x, dt, Bm, Cm, z, dy;
    const float *A, *skip, *dt_bias, *h0, *dh_last, *states_in;
    const int32_t *lengths;
    StepsOut y, dx, ddt, dz, dB, dC;
    float *h_last, *states, *dA, *dskip, *ddt_bias, *dh0;
    void *ws;
};
size_t select_workspace(int64_t B, int64_t T, int64_t D, int64_t S);
size_t select_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t S);
hipError_t launch_select(int32_t type, const SelectArgs &a, hipStream_t s);
hipError_t launch_select_grad(int32_t type, const SelectArgs &a, hipStream_t s);

struct ConvArgs {
    int64_t B, T, D, K;
    Steps x, dy;
    StepsOut y, dx;
    const void *weight, *bias, *state, *dlast;  // [K, D], [D], [B, K - 1, D]
    const int32_t *lengths;
    bool silu;
    void *last, *dweight, *dbias, *dstate;
    void *ws;
};
int64_t conv_items(int64_t B, int64_t T, int64_t D);  // threads of a call at most
size_t conv_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t K);
hipError_t launch_conv(int32_t type, const ConvArgs &a, hipStream_t s);
hipError_t launch_conv_grad(int32_t type, const ConvArgs &a, hipStream_t s);

struct ClipArgs {
    int64_t n;
    // host arrays, read during the call
    const void *const *in;
    void *const *out;
    const int64_t *counts;
    const int32_t *types, *out_types;
    float max_norm, scale;
    float *norm;
    void *ws;
};
size_t clip_workspace(int64_t n, const int64_t *counts);
hipError_t launch_clip(const ClipArgs &a, hipStream_t s);

struct BeamArgs {
    int64_t R, W, V, K;
    const void *logits;
    int64_t ld;
    const float *scores;
    const uint64_t *last;
    uint64_t end;
    float *out_scores;
    int32_t *parents;
    uint64_t *tokens;
    void *ws;
};
size_t beam_workspace(int32_t type, int64_t R, int64_t W, int64_t V, int64_t K);
hipError_t launch_beam(int32_t type, const BeamArgs &a, hipStream_t s);

struct ReorderArgs {
    int64_t n, R, W, K;
    // host arrays, read during the call
    const void *const *in;
    void *const *out;
    const int64_t *bytes;  // of a beam's row
    const int32_t *parents;
};
hipError_t launch_reorder(const ReorderArgs &a, hipStream_t s);

} // namespace tq
