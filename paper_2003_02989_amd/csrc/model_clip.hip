// model_clip.hip -- the norm of many tensors together, and clipping them by it.
//
//   norm = scale (sum over all elements of g^2)^{1/2},
//   out = g scale min(1, max_norm / norm).
//
// Bound by memory: every element is read for the norm, read again and written.
// Squares are summed in 64 bits: the largest fp32 value squared is a number there,
// and a sum's error is none that the norm shows.  The tensors, one after the other,
// make a list of chunks; each wavefront takes a run of the list, so that it looks
// for a tensor once and then goes from one to the next.  Workgroups leave their
// sums, and every workgroup of the second kernel adds them up for itself, in the
// same order: a launch less than a kernel in between would be.  The second kernel
// takes a run from its end: what the first one read last is still in the caches.
// Few elements take one workgroup and one launch.
#include <algorithm>

#include "model.h"
#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

constexpr int kTensors = 100;          // of a launch: their places are kernel arguments
constexpr int kChunk = 4096;           // elements: 8 accesses of 16 bytes a lane, 16 in fp32
constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kBlocks = 1024;          // of a launch at most: 16 wavefronts per compute unit
constexpr int kFew = 1024;             // threads of the only workgroup
constexpr int64_t kFewElements = 1 << 16;

struct Tensors {
    const void *in[kTensors];
    void *out[kTensors];
    int64_t count[kTensors];
    uint32_t first[kTensors + 1];  // chunk
    uint8_t in_type[kTensors], out_type[kTensors];
    int n;
};
static_assert(sizeof(Tensors) < 3700, "kernel arguments are limited to 4096 bytes");

// Calls f with the element type of a code.
template <class F> __device__ __forceinline__ void by_type(int type, F &&f)
{
    if (type == TQ_F32) f(float{});
    else if (type == TQ_BF16) f(__bf16{});
    else f(_Float16{});
}

// The run of chunks of wavefront `wave` of `waves`.
struct Run {
    uint32_t from, to;
    __device__ Run(uint32_t chunks, uint32_t wave, uint32_t waves)
    {
        from = (uint32_t)((uint64_t)chunks * wave / waves);
        to = (uint32_t)((uint64_t)chunks * (wave + 1) / waves);
    }
};

__device__ __forceinline__ int tensor_of(const Tensors &t, uint32_t chunk)
{
    int lo = 0, hi = t.n;  // first[lo] <= chunk < first[hi]
    while (hi - lo > 1) {
        const int m = (lo + hi) / 2;
        if (t.first[m] <= chunk) lo = m;
        else hi = m;
    }
    return lo;
}

// The sum of squares of up to a chunk.  Four sums a lane: what follows another addition
// waits for it.
template <class T> __device__ __forceinline__ double squares(const T *p, int64_t n)
{
    constexpr int V = kVec<T>, N = kChunk / (64 * V);
    const int lane = threadIdx.x & 63;
    double s[4] = {};
    const auto add = [&](const T(&v)[V]) {
#pragma unroll
        for (int j = 0; j < V; j++) {
            const double d = (double)(float)v[j];
            s[j % 4] = fma(d, d, s[j % 4]);
        }
    };
    if (n >= kChunk) {
        T v[N][V];
#pragma unroll
        for (int k = 0; k < N; k++) __builtin_memcpy(v[k], p + (k * 64 + lane) * V, sizeof v[k]);
#pragma unroll
        for (int k = 0; k < N; k++) add(v[k]);
    } else {
        const int whole = (int)n / V;
#pragma unroll 4
        for (int k = lane; k < whole; k += 64) {
            T v[V];
            __builtin_memcpy(v, p + k * V, sizeof v);
            add(v);
        }
        if (lane < (int)n - whole * V) {
            const double d = (double)(float)p[whole * V + lane];
            s[0] = fma(d, d, s[0]);
        }
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

template <class T, class O> __device__ __forceinline__ void scaled(const T *p, O *o, int64_t n, float c)
{
    constexpr int V = kVec<T>, N = kChunk / (64 * V);
    const int lane = threadIdx.x & 63;
    const auto put = [&](int k, const T(&v)[V]) {
        float f[V];
#pragma unroll
        for (int j = 0; j < V; j++) f[j] = (float)v[j] * c;
        store_vec<V>(o + k * V, f);
    };
    if (n >= kChunk) {
        T v[N][V];
#pragma unroll
        for (int k = 0; k < N; k++) __builtin_memcpy(v[k], p + (k * 64 + lane) * V, sizeof v[k]);
#pragma unroll
        for (int k = 0; k < N; k++) put(k * 64 + lane, v[k]);
    } else {
        const int whole = (int)n / V;
#pragma unroll 4
        for (int k = lane; k < whole; k += 64) {
            T v[V];
            __builtin_memcpy(v, p + k * V, sizeof v);
            put(k, v);
        }
        const int at = whole * V + lane;
        if (at < (int)n) o[at] = (O)((float)p[at] * c);
    }
}

// The same with a factor that fp32 holds as a subnormal number or not at all: elements
// near the largest ones still give products that are numbers, formed in 64 bits.  One
// loop for all types: it is seldom taken, and a small kernel waits for its code.
__device__ __forceinline__ void scaled_far(const Tensors &t, int i, int64_t at, double f)
{
    const int64_t to = min(at + kChunk, t.count[i]);
    for (int64_t k = at + (threadIdx.x & 63); k < to; k += 64) {
        float v;
        by_type(t.in_type[i], [&](auto x) { v = (float)((const decltype(x) *)t.in[i])[k]; });
        const float o = (float)((double)v * f);
        by_type(t.out_type[i], [&](auto y) { ((decltype(y) *)t.out[i])[k] = (decltype(y))o; });
    }
}

// A wavefront's sum over its run.
__device__ __forceinline__ double sum_run(const Tensors &t, Run r)
{
    double s = 0;
    if (r.from < r.to) {
        int i = tensor_of(t, r.from);
        for (uint32_t c = r.from; c < r.to; c++) {
            while (c >= t.first[i + 1]) i++;
            const int64_t at = (int64_t)(c - t.first[i]) * kChunk;
            by_type(t.in_type[i], [&](auto x) { s += squares((const decltype(x) *)t.in[i] + at, t.count[i] - at); });
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    return s;
}

// A run from its end.  Where nothing changes, in place, nothing is written.
__device__ __forceinline__ void scale_run(const Tensors &t, Run r, double f)
{
    if (r.from >= r.to) return;
    const float c = (float)f;
    const bool far = f > 0. && f < 0x1p-126;
    int i = tensor_of(t, r.to - 1);
    for (uint32_t k = r.to; k-- > r.from;) {
        while (k < t.first[i]) i--;
        if (c == 1.f && t.in[i] == t.out[i]) continue;
        const int64_t at = (int64_t)(k - t.first[i]) * kChunk;
        if (far) {
            scaled_far(t, i, at, f);
            continue;
        }
        by_type(t.in_type[i], [&](auto x) {
            by_type(t.out_type[i], [&](auto y) {
                scaled((const decltype(x) *)t.in[i] + at, (decltype(y) *)t.out[i] + at, t.count[i] - at, c);
            });
        });
    }
}

// The factor of the elements from the sum of their squares; a norm that is not a
// number gives factors that are none, an infinite one zeros.
__device__ __forceinline__ double factor(const ClipArgs &a, double sum, float *norm)
{
    const double n = sqrt(sum) * (double)a.scale;
    if (norm) *norm = (float)n;
    return (double)a.scale * (n <= (double)a.max_norm ? 1. : (double)a.max_norm / n);
}

__global__ __launch_bounds__(kThreads) void k_clip_sum(Tensors t, double *part)
{
    __shared__ double red[kWaves];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const double s = sum_run(t, Run(t.first[t.n], blockIdx.x * kWaves + wave, gridDim.x * kWaves));
    if ((threadIdx.x & 63) == 0) red[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kThreads) void k_clip_scale(Tensors t, ClipArgs a, const double *part, int parts, float *norm)
{
    __shared__ double red[kWaves];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double s = 0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) red[wave] = s;
    __syncthreads();
    s = (red[0] + red[1]) + (red[2] + red[3]);
    const double f = factor(a, s, blockIdx.x == 0 && threadIdx.x == 0 ? norm : nullptr);
    scale_run(t, Run(t.first[t.n], blockIdx.x * kWaves + wave, gridDim.x * kWaves), f);
}

__global__ __launch_bounds__(kFew) void k_clip_few(Tensors t, ClipArgs a)
{
    __shared__ double red[kFew / 64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Run r(t.first[t.n], wave, kFew / 64);
    double s = sum_run(t, r);
    if ((threadIdx.x & 63) == 0) red[wave] = s;
    __syncthreads();
    s = 0;
#pragma unroll
    for (int w = 0; w < kFew / 64; w++) s += red[w];
    scale_run(t, r, factor(a, s, threadIdx.x == 0 ? a.norm : nullptr));
}

uint32_t chunks_of(int64_t count) { return (uint32_t)((count + kChunk - 1) / kChunk); }

// Calls f with each launch's tensors and the number of workgroups for them.
template <class F> void by_launch(const ClipArgs &a, F &&f)
{
    Tensors t;
    for (int64_t i = 0; i < a.n;) {
        uint32_t chunks = 0;
        // the chunks of one launch are counted in 32 bits: a tensor holds fewer than 2^30
        for (t.n = 0; i < a.n && t.n < kTensors && (t.n == 0 || chunks < 1u << 30); i++) {
            if (a.counts[i] == 0) continue;
            t.in[t.n] = a.in[i], t.out[t.n] = a.out[i], t.count[t.n] = a.counts[i];
            t.in_type[t.n] = (uint8_t)a.types[i], t.out_type[t.n] = (uint8_t)a.out_types[i];
            t.first[t.n++] = chunks;
            chunks += chunks_of(a.counts[i]);
        }
        t.first[t.n] = chunks;
        if (t.n) f(t, (int)std::min<uint32_t>((chunks + kWaves - 1) / kWaves, kBlocks));
    }
}

bool few(const ClipArgs &a)
{
    int64_t n = 0;
    int some = 0;
    for (int64_t i = 0; i < a.n; i++) {
        n += a.counts[i];
        some += a.counts[i] > 0;
        if (n > kFewElements || some > kTensors) return false;
    }
    return true;
}

} // namespace

size_t clip_workspace(int64_t n, const int64_t *counts)
{
    ClipArgs a{};
    a.n = n, a.counts = counts;
    if (few(a)) return 0;
    // launches of kTensors each, or of as many as reach 2^30 chunks
    int64_t chunks = 0;
    for (int64_t i = 0; i < n; i++) chunks += chunks_of(counts[i]);
    return sizeof(double) * kBlocks * (size_t)((n + kTensors - 1) / kTensors + (chunks >> 30) + 1);
}

hipError_t launch_clip(const ClipArgs &a, hipStream_t s)
{
    if (few(a)) {
        Tensors t;
        t.n = 0;
        t.first[0] = 0;
        by_launch(a, [&](const Tensors &all, int) { t = all; });
        k_clip_few<<<1, kFew, 0, s>>>(t, a);
        return hipGetLastError();
    }
    double *part = (double *)a.ws;
    int parts = 0;
    by_launch(a, [&](const Tensors &t, int blocks) {
        k_clip_sum<<<blocks, kThreads, 0, s>>>(t, part + parts);
        parts += blocks;
    });
    float *norm = a.norm;
    by_launch(a, [&](const Tensors &t, int blocks) {
        k_clip_scale<<<blocks, kThreads, 0, s>>>(t, a, part, parts, norm);
        norm = nullptr;
    });
    return hipGetLastError();
}

} // namespace tq
