// model_device.h -- what the kernels of selective models share.
#pragma once
#include "model.h"
#include "seq_device.h"

namespace tq {

// exp(v).  The product with log2 e is rounded, an error of up to |v| 2^-24 relative;
// for fp32 inputs what the rounding lost is put back.
template <class T> __device__ __forceinline__ float exp_of(float v)
{
    constexpr float kLog2e = 1.44269504088896341f;
    if constexpr (sizeof(T) == 4) v = v < -1e4f ? -1e4f : v > 1e4f ? 1e4f : v;  // infinities have no remainder; NaN stays
    const float t = v * kLog2e;
    float e = __builtin_amdgcn_exp2f(t);
    if constexpr (sizeof(T) == 4) {
        // log2 e = kLog2e + 1.92596299e-8; ln 2 turns the lost part into a factor
        const float lost = fmaf(v, kLog2e, -t) + v * 1.92596299e-8f;
        e = t < 128.f ? fmaf(e, lost * 0.693147181f, e) : e;
    }
    return e;
}

template <class T> __device__ __forceinline__ float sigmoid(float v)
{
    return __builtin_amdgcn_rcpf(1.f + exp_of<T>(-v));
}

// sigmoid(v) and sigmoid(-v), each to full relative accuracy.
template <class T> __device__ __forceinline__ void sigmoids(float v, float &s, float &c)
{
    const float e = exp_of<T>(-fabsf(v)), r = __builtin_amdgcn_rcpf(1.f + e), er = e * r;
    s = v >= 0.f ? r : er;
    c = v >= 0.f ? er : r;
}

// softplus(v), relative accuracy kept where it is small, and its derivative.
// log(1 + e) = 2 atanh(e / (2 + e)), whose argument is at most 1/3.
template <class T> __device__ __forceinline__ float softplus(float v, float &slope)
{
    const float e = exp_of<T>(-fabsf(v));
    const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
    float p = 1.f / 15.f;
    p = fmaf(p, q, 1.f / 13.f);
    p = fmaf(p, q, 1.f / 11.f);
    p = fmaf(p, q, 1.f / 9.f);
    p = fmaf(p, q, 1.f / 7.f);
    p = fmaf(p, q, 1.f / 5.f);
    p = fmaf(p, q, 1.f / 3.f);
    p = fmaf(p * q, s, s);
    const float r = __builtin_amdgcn_rcpf(1.f + e);
    slope = v >= 0.f ? r : e * r;
    return fmaf(2.f, p, fmaxf(v, 0.f));  // e of NaN is NaN
}

} // namespace tq
