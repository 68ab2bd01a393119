// model_scan.hip -- the selective state space scan over time and its gradients.
//
//   d_t = softplus(dt_t + bias),  h_t = exp(d_t A) h_{t-1} + d_t x_t B_t,
//   y_t = (C_t . h_t + skip x_t) silu(z_t),
//
// D channels of S states each.  What bounds it is the exponential of every
// channel, state and step, which takes four of the eight issue slots that an
// element of state costs.  So an element's exponential is formed once, and nothing
// else is done per state that can be done per channel: a lane holds a channel with
// four of its states in registers, and a workgroup of W wavefronts holds 64
// channels with up to 4 W states.  Steps go in tiles of 16: the wavefronts share
// out the steps to form d, d x and the gates, leave them and the B and C of all
// states in LDS, step through the tile with their own states, and leave their parts
// of C . h in LDS, which the wavefront that a step belongs to adds up.
//
// Where there are too few channels to fill the chip, time is cut into chunks.  A
// first kernel forms the state at each chunk's end from zero and the sum of its d
// (exp(A sum d) is the chunk's whole decay); the scan proper then starts each
// chunk from the chunks before it, in their order.
//
// The gradient takes the tiles from the last one back.  A tile's states are formed
// again from the state saved before it and stay in registers, with their decays,
// while l goes backwards through the tile.  dB and dC are sums over the channels:
// over a wavefront's 64 by exchanges between lanes, over the slabs of 64 by a
// second kernel that adds their parts in order, as dA's over records and chunks.
#include <algorithm>
#include <type_traits>

#include "model.h"
#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

constexpr int kTile = TQ_STATES_PIECE;  // steps
constexpr int kOwn = 4;                 // states of a lane
constexpr float kLog2e = 1.44269504088896341f;

struct Geom {
    uint32_t blocks;       // of the launch
    uint32_t slabs, rows;  // slabs of 64 channels; gradient: workgroups per slab
    int chunks;
    int64_t chunk;         // steps of a chunk, whole tiles
    float *start;          // [B][S][D]: the state before the first step
    float *ends, *sums;    // [B][chunks][S][D], [B][chunks][D]
    float *part_bc;        // [slabs][B][T][2][S]
    float *part_a, *part_v;  // [rows][S][D], [rows][2][D]
};

// d = softplus(v), relative accuracy kept where it is small, and its derivative.
// log(1 + e) = 2 atanh(e / (2 + e)), whose argument is at most 1/3.
__device__ __forceinline__ float softplus(float v, float &slope)
{
    const float e = expf(-fabsf(v));
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
    return fmaf(2.f, p, v > 0.f ? v : v == v ? 0.f : v);
}

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + expf(-v)); }

template <class T> __device__ __forceinline__ const T *row_of(const Steps &s, int64_t b, int64_t t)
{
    return (const T *)s.p + b * s.batch + t * s.step;
}
template <class T> __device__ __forceinline__ T *row_of(const StepsOut &s, int64_t b, int64_t t)
{
    return (T *)s.p + b * s.batch + t * s.step;
}

// What a workgroup and a lane work on.
struct Place {
    int64_t b, len, t0, t1, n1;  // the chunk's steps [t0, t1), of the record [t0, n1)
    int chunk, wave, lane;
    uint32_t slab;
    int64_t d, dc;  // the lane's channel, and one that there is
    bool in;
    __device__ void lanes(uint32_t slab_, int64_t D)
    {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        slab = slab_;
        d = (int64_t)slab * 64 + lane;
        in = d < D;
        dc = in ? d : D - 1;
    }
    __device__ void steps(const SelectArgs &a, const Geom &g, uint32_t item)
    {
        b = item / (uint32_t)g.chunks;
        chunk = (int)(item - (uint32_t)b * (uint32_t)g.chunks);
        len = a.T;
        if (a.lengths) len = min(max((int64_t)a.lengths[b], (int64_t)0), a.T);
        t0 = chunk * g.chunk;
        t1 = min(t0 + g.chunk, a.T);
        n1 = min(t1, len);
    }
};

// The decays' exponents to base 2 of a lane's states, and the others at zero: a
// padded step has d = 0, and exp2(0) = 1 has to come out of A = -infinity too.
__device__ __forceinline__ float exponent(float A)
{
    const float v = A * kLog2e;
    return fabsf(v) <= 3.4e38f || v != v ? v : copysignf(3.4e38f, v);
}

// A tile's inputs: one read ahead by registers, and what the wavefronts share of
// it.  Steps are dealt out in runs of kTile / W; steps past the record's end read
// its last one and count as zero.
template <class T, int W, int R, bool X, bool Z, bool DY, bool PB, bool PC> struct Tile {
    static constexpr int PER = kTile / W, BC = R * 2;  // B and C elements per thread
    T x[X ? PER : 1], dt[PER], z[Z ? PER : 1], dy[DY ? PER : 1], bc[BC];
    __device__ __forceinline__ void fetch(const SelectArgs &a, const Place &at, int64_t tile)
    {
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int64_t t = min(tile + at.wave * PER + i, at.len - 1);
            if constexpr (X) x[i] = row_of<T>(a.x, at.b, t)[at.dc];
            dt[i] = row_of<T>(a.dt, at.b, t)[at.dc];
            if constexpr (Z)
                if (a.z.p) z[i] = row_of<T>(a.z, at.b, t)[at.dc];
            if constexpr (DY) dy[i] = row_of<T>(a.dy, at.b, t)[at.dc];
        }
#pragma unroll
        for (int i = 0; i < BC; i++) {
            const int v = threadIdx.x + i * 64 * W, n = v % (4 * W * R);
            const bool c = v / (4 * W * R) % 2;
            const int64_t t = min(tile + v / (8 * W * R), at.len - 1);
            bc[i] = (T)0.f;
            if (n < a.S && (c ? PC : PB)) bc[i] = row_of<T>(c ? a.Cm : a.Bm, at.b, t)[n];
        }
    }
    // B and C, [step][group of four states][B, C]
    __device__ __forceinline__ void share_bc(const Place &at, int64_t tile, float (*to)[W * R][2][4]) const
    {
#pragma unroll
        for (int i = 0; i < BC; i++) {
            const int v = threadIdx.x + i * 64 * W, n = v % (4 * W * R), c = v / (4 * W * R) % 2, t = v / (8 * W * R);
            to[t][n / 4][c][n % 4] = tile + t < at.len ? (float)bc[i] : 0.f;
        }
    }
};

template <int N> __device__ __forceinline__ float sum_of(const float (*p)[kTile][64], int t, int lane, int waves)
{
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < N; w++)
        if (w < waves) s += p[w][t][lane];
    return s;
}

// The scan, or with ENDS only the state at the chunk's end (from zero but for the
// first chunk) and the sum of its d.
template <class T, int W, bool ENDS> __global__ __launch_bounds__(64 * W) void k_select(SelectArgs a, Geom g)
{
    constexpr int PER = kTile / W;
    __shared__ float s_d[kTile][64], s_u[kTile][64];
    __shared__ __attribute__((aligned(16))) float s_bc[kTile][W][2][4];
    __shared__ float s_p[ENDS ? 1 : W][kTile][64];
    const uint32_t item = block_of();
    if (item >= g.blocks) return;
    Place at;
    const uint32_t rest = item / g.slabs;
    at.lanes(item - rest * g.slabs, a.D);
    if constexpr (ENDS) {  // the last chunk's is not needed
        const uint32_t b = rest / (uint32_t)(g.chunks - 1);
        at.steps(a, g, rest + b);
    } else at.steps(a, g, rest);
    const int n0 = at.wave * kOwn, waves = (a.S + kOwn - 1) / kOwn;
    const bool some = n0 < a.S;  // the wavefront has states

    float A[kOwn], h[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; j++) {
        const bool there = at.in && n0 + j < a.S;
        A[j] = there && a.A ? exponent(a.A[at.d * a.S + n0 + j]) : 0.f;
        h[j] = 0.f;
        if (!there) continue;
        if (at.chunk == 0) {
            if (!ENDS && g.chunks > 1) h[j] = g.start[(at.b * a.S + n0 + j) * a.D + at.d];
            else if (a.h0) h[j] = a.h0[(at.b * a.D + at.d) * a.S + n0 + j];
            if (ENDS) g.start[(at.b * a.S + n0 + j) * a.D + at.d] = h[j];
        }
    }
    if (!ENDS && at.chunk > 0 && at.t0 < at.len && some && at.in) {  // from the chunks before
        const float *end = g.ends + (at.b * g.chunks * a.S + n0) * a.D + at.d, *sum = g.sums + at.b * g.chunks * a.D + at.d;
        const int own = min(kOwn, a.S - n0);
#pragma unroll 4
        for (int k = 0; k < at.chunk; k++) {
            const float s = sum[(int64_t)k * a.D];
#pragma unroll
            for (int j = 0; j < kOwn; j++)
                if (j < own) {
                    const float e = end[((int64_t)k * a.S + j) * a.D];
                    h[j] = k == 0 ? e : fmaf(__builtin_amdgcn_exp2f(s * A[j]), h[j], e);
                }
        }
    }
    const float bias = a.dt_bias ? a.dt_bias[at.dc] : 0.f;
    const float skip = !ENDS && a.skip ? a.skip[at.dc] : 0.f;
    float total = 0.f;
    Tile<T, W, 1, true, !ENDS, false, true, !ENDS> now, next;
    if (at.t0 < at.n1) next.fetch(a, at, at.t0);
    for (int64_t tile = at.t0; tile < at.n1; tile += kTile) {
        now = next;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int t = at.wave * PER + i;
            float slope, d = softplus((float)now.dt[i] + bias, slope), u = d * (float)now.x[i];
            if (tile + t >= at.len) d = u = 0.f;
            s_d[t][at.lane] = d;
            s_u[t][at.lane] = u;
            if (ENDS) total += d;
        }
        now.share_bc(at, tile, s_bc);
        __syncthreads();
        if (tile + kTile < at.n1) next.fetch(a, at, tile + kTile);
        if (some) {
            if (!ENDS && a.states && at.in) {
                float *to = a.states + ((at.b * ((a.T + kTile - 1) / kTile) + tile / kTile) * a.S + n0) * a.D + at.d;
#pragma unroll
                for (int j = 0; j < kOwn; j++)
                    if (n0 + j < a.S) to[(int64_t)j * a.D] = h[j];
            }
#pragma unroll
            for (int t = 0; t < kTile; t++) {
                if (t % 4 == 0 && tile + t >= at.n1) break;
                const float d = s_d[t][at.lane], u = s_u[t][at.lane];
                float p = 0.f;
#pragma unroll
                for (int j = 0; j < kOwn; j++) {
                    h[j] = fmaf(__builtin_amdgcn_exp2f(d * A[j]), h[j], u * s_bc[t][at.wave][0][j]);
                    if (!ENDS) p = fmaf(s_bc[t][at.wave][1][j], h[j], p);
                }
                if (!ENDS) s_p[at.wave][t][at.lane] = p;
            }
        }
        __syncthreads();
        if constexpr (!ENDS) {
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int t = at.wave * PER + i;
                if (tile + t >= at.n1 || !at.in) continue;
                float y = fmaf(skip, (float)now.x[i], sum_of<W>(s_p, t, at.lane, waves));
                if (a.z.p) y *= (float)now.z[i] * sigmoid((float)now.z[i]);
                row_of<T>(a.y, at.b, tile + t)[at.d] = (T)y;
            }
        }
    }
    if (ENDS) {
        float *end = g.ends + ((at.b * g.chunks + at.chunk) * a.S + n0) * a.D + at.d;
#pragma unroll
        for (int j = 0; j < kOwn; j++)
            if (at.in && n0 + j < a.S) end[(int64_t)j * a.D] = h[j];
        s_d[at.wave][at.lane] = total;
        __syncthreads();
        if (at.wave == 0 && at.in) {
            float s = 0.f;
            for (int w = 0; w < W; w++) s += s_d[w][at.lane];
            g.sums[(at.b * g.chunks + at.chunk) * a.D + at.d] = s;
        }
        return;
    }
    const bool last = at.len == 0 ? at.chunk == 0 : at.t0 < at.len && at.len <= at.t1;
    if (a.h_last && last && at.in)
#pragma unroll
        for (int j = 0; j < kOwn; j++)
            if (n0 + j < a.S) a.h_last[(at.b * a.D + at.d) * a.S + n0 + j] = h[j];
    if (at.in)
        for (int64_t t = max(at.t0, at.len) + at.wave; t < at.t1; t += W) row_of<T>(a.y, at.b, t)[at.d] = (T)0.f;
}

// ---------------------------------------------------------------- backward

// What l of a chunk's first step hands to the chunk before it, from nothing behind
// the chunk (the record's last chunk: from dh_last), and the sum of its d.
template <class T, int W> __global__ __launch_bounds__(64 * W) void k_select_back(SelectArgs a, Geom g)
{
    constexpr int PER = kTile / W;
    __shared__ float s_d[kTile][64], s_q[kTile][64];
    __shared__ __attribute__((aligned(16))) float s_bc[kTile][W][2][4];
    const uint32_t item = block_of();
    if (item >= g.blocks) return;
    Place at;
    const uint32_t rest = item / g.slabs, b = rest / (uint32_t)(g.chunks - 1);
    at.lanes(item - rest * g.slabs, a.D);
    at.steps(a, g, rest + b + 1);  // all but the first chunk
    if (at.t0 >= at.len) return;
    const int n0 = at.wave * kOwn;
    float A[kOwn], m[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; j++) {
        const bool there = at.in && n0 + j < a.S;
        A[j] = there ? exponent(a.A[at.d * a.S + n0 + j]) : 0.f;
        m[j] = there && a.dh_last && at.len <= at.t1 ? a.dh_last[(at.b * a.D + at.d) * a.S + n0 + j] : 0.f;
    }
    const float bias = a.dt_bias ? a.dt_bias[at.dc] : 0.f;
    float total = 0.f;
    Tile<T, W, 1, false, true, true, false, true> now, next;
    const int64_t top = at.t0 + (at.n1 - at.t0 - 1) / kTile * kTile;
    next.fetch(a, at, top);
    for (int64_t tile = top; tile >= at.t0; tile -= kTile) {
        now = next;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int t = at.wave * PER + i;
            float slope, d = softplus((float)now.dt[i] + bias, slope), q = (float)now.dy[i];
            if (a.z.p) q *= (float)now.z[i] * sigmoid((float)now.z[i]);
            if (tile + t >= at.len) d = q = 0.f;
            s_d[t][at.lane] = d;
            s_q[t][at.lane] = q;
            total += d;
        }
        now.share_bc(at, tile, s_bc);
        __syncthreads();
        if (tile > at.t0) next.fetch(a, at, tile - kTile);
#pragma unroll
        for (int t = kTile - 1; t >= 0; t--) {
            const float d = s_d[t][at.lane], q = s_q[t][at.lane];
#pragma unroll
            for (int j = 0; j < kOwn; j++)
                m[j] = __builtin_amdgcn_exp2f(d * A[j]) * fmaf(s_bc[t][at.wave][1][j], q, m[j]);
        }
        __syncthreads();
    }
    float *end = g.ends + ((at.b * g.chunks + at.chunk) * a.S + n0) * a.D + at.d;
#pragma unroll
    for (int j = 0; j < kOwn; j++)
        if (at.in && n0 + j < a.S) end[(int64_t)j * a.D] = m[j];
    s_d[at.wave][at.lane] = total;
    __syncthreads();
    if (at.wave == 0 && at.in) {
        float s = 0.f;
        for (int w = 0; w < W; w++) s += s_d[w][at.lane];
        g.sums[(at.b * g.chunks + at.chunk) * a.D + at.d] = s;
    }
}

template <int ROR> __device__ __forceinline__ float turned(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + ROR, 0xf, 0xf, true));
}

// The sums of four values over a wavefront's lanes: lanes 16 r to 16 r + 15 end with
// that of value 0, 2, 1, 3 for r = 0 .. 3.
__device__ __forceinline__ float sums_of_four(const float (&v)[4])
{
    const auto bits = [](float f) { return __builtin_bit_cast(unsigned, f); };
    const auto val = [](unsigned u) { return __builtin_bit_cast(float, u); };
    const auto p = __builtin_amdgcn_permlane32_swap(bits(v[0]), bits(v[1]), false, false);
    const auto q = __builtin_amdgcn_permlane32_swap(bits(v[2]), bits(v[3]), false, false);
    const float m = val(p[0]) + val(p[1]), n = val(q[0]) + val(q[1]);  // halves: value 0, 1; value 2, 3
    const auto r = __builtin_amdgcn_permlane16_swap(bits(m), bits(n), false, false);
    float s = val(r[0]) + val(r[1]);
    s += turned<8>(s);
    s += turned<4>(s);
    s += turned<2>(s);
    s += turned<1>(s);
    return s;
}

template <class T, int W, int R> __global__ __launch_bounds__(64 * W) void k_select_grad(SelectArgs a, Geom g)
{
    constexpr int PER = kTile / W;
    __shared__ float s_d[kTile][64], s_u[kTile][64], s_q[kTile][64];
    __shared__ __attribute__((aligned(16))) float s_bc[kTile][W * R][2][4];
    __shared__ float s_p[W][kTile][64], s_l[W][kTile][64], s_w[W][kTile][64];
    const uint32_t block = block_of();
    if (block >= g.blocks) return;
    Place at;
    const uint32_t first = block / g.slabs;
    at.lanes(block - first * g.slabs, a.D);
    const int waves = min((a.S + kOwn - 1) / kOwn, W);
    const float bias = a.dt_bias ? a.dt_bias[at.dc] : 0.f, skip = a.skip ? a.skip[at.dc] : 0.f;
    float A[R][kOwn], dA[R][kOwn], m[R][kOwn], dskip = 0.f, dbias = 0.f;
    const auto state = [&](int r, int j) { return (r * W + at.wave) * kOwn + j; };
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int j = 0; j < kOwn; j++) {
            const int n = state(r, j);
            A[r][j] = at.in && n < a.S && a.A ? exponent(a.A[at.d * a.S + n]) : 0.f;
            dA[r][j] = 0.f;
        }
    const int64_t pieces = (a.T + kTile - 1) / kTile;
    for (uint32_t item = first; item < (uint32_t)(a.B * g.chunks); item += g.rows) {
        at.steps(a, g, item);
        const int top_chunk = at.len > 0 ? (int)((at.len - 1) / g.chunk) : 0;
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int j = 0; j < kOwn; j++) {
                const int n = state(r, j);
                m[r][j] = 0.f;
                if (!at.in || n >= a.S || at.chunk > top_chunk) continue;
                if (at.chunk == top_chunk) {
                    if (a.dh_last) m[r][j] = a.dh_last[(at.b * a.D + at.d) * a.S + n];
                } else {  // from the chunks behind
                    for (int k = top_chunk; k > at.chunk; k--) {
                        const float e = g.ends[((at.b * g.chunks + k) * a.S + n) * a.D + at.d];
                        const float s = g.sums[(at.b * g.chunks + k) * a.D + at.d];
                        m[r][j] = k == top_chunk ? e : fmaf(__builtin_amdgcn_exp2f(s * A[r][j]), m[r][j], e);
                    }
                }
            }
        Tile<T, W, R, true, true, true, true, true> now, next;
        const int64_t top = at.t0 + (at.n1 - at.t0 - 1) / kTile * kTile;
        if (at.t0 < at.n1) next.fetch(a, at, top);
        for (int64_t tile = top; tile >= at.t0 && at.t0 < at.n1; tile -= kTile) {
            now = next;
            float delta[PER], slope[PER], q[PER], dz[PER];
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int t = at.wave * PER + i;
                delta[i] = softplus((float)now.dt[i] + bias, slope[i]);
                const float dy = (float)now.dy[i];
                q[i] = dy;
                dz[i] = 0.f;
                if (a.z.p) {
                    const float z = (float)now.z[i], s = sigmoid(z);
                    q[i] = dy * (z * s);
                    dz[i] = dy * (s * fmaf(z, 1.f - s, 1.f));
                }
                const bool there = at.in && tile + t < at.len;
                s_d[t][at.lane] = there ? delta[i] : 0.f;
                s_u[t][at.lane] = there ? delta[i] * (float)now.x[i] : 0.f;
                s_q[t][at.lane] = there ? q[i] : 0.f;
            }
            now.share_bc(at, tile, s_bc);
            __syncthreads();
            if (tile > at.t0) next.fetch(a, at, tile - kTile);
#pragma unroll
            for (int r = 0; r < R; r++) {
                const int n0 = state(r, 0), group = r * W + at.wave;
                if (n0 >= a.S) continue;
                float h[kTile + 1][kOwn], e[kTile][kOwn];
#pragma unroll
                for (int j = 0; j < kOwn; j++)
                    h[0][j] = at.in && n0 + j < a.S
                                  ? a.states_in[((at.b * pieces + tile / kTile) * a.S + n0 + j) * a.D + at.d] : 0.f;
#pragma unroll
                for (int t = 0; t < kTile; t++) {
                    const float d = s_d[t][at.lane], u = s_u[t][at.lane];
                    float p = 0.f;
#pragma unroll
                    for (int j = 0; j < kOwn; j++) {
                        e[t][j] = __builtin_amdgcn_exp2f(d * A[r][j]);
                        h[t + 1][j] = fmaf(e[t][j], h[t][j], u * s_bc[t][group][0][j]);
                        p = fmaf(s_bc[t][group][1][j], h[t + 1][j], p);
                    }
                    s_p[at.wave][t][at.lane] = r ? s_p[at.wave][t][at.lane] + p : p;
                }
                float to_b = 0.f, to_c = 0.f;
#pragma unroll
                for (int t = kTile - 1; t >= 0; t--) {
                    const float d = s_d[t][at.lane], u = s_u[t][at.lane], q = s_q[t][at.lane];
                    float bl = 0.f, aw = 0.f, vb[kOwn], vc[kOwn];
#pragma unroll
                    for (int j = 0; j < kOwn; j++) {
                        const float l = fmaf(s_bc[t][group][1][j], q, m[r][j]);
                        vc[j] = q * h[t + 1][j];
                        vb[j] = u * l;
                        bl = fmaf(s_bc[t][group][0][j], l, bl);
                        m[r][j] = e[t][j] * l;
                        const float w = m[r][j] * h[t][j];
                        aw = fmaf(A[r][j], w, aw);
                        dA[r][j] = fmaf(d, w, dA[r][j]);
                    }
                    s_l[at.wave][t][at.lane] = r ? s_l[at.wave][t][at.lane] + bl : bl;
                    s_w[at.wave][t][at.lane] = r ? s_w[at.wave][t][at.lane] + aw : aw;
                    const float sb = sums_of_four(vb), sc = sums_of_four(vc);
                    const bool mine = (at.lane & 15) == t;
                    to_b = mine ? sb : to_b;
                    to_c = mine ? sc : to_c;
                }
                // lane: step lane % 16, state 0, 2, 1, 3 of the four
                const int quarter = at.lane >> 4, n = n0 + (quarter >> 1 | (quarter & 1) << 1);
                const int64_t t = tile + (at.lane & 15);
                if (t < at.n1 && n < a.S) {
                    float *to = g.part_bc + ((at.slab * a.B + at.b) * a.T + t) * 2 * a.S + n;
                    to[0] = to_b;
                    to[a.S] = to_c;
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int t = at.wave * PER + i;
                if (tile + t >= at.n1 || !at.in) continue;
                const float x = (float)now.x[i], p = fmaf(skip, x, sum_of<W>(s_p, t, at.lane, waves));
                const float bl = sum_of<W>(s_l, t, at.lane, waves), aw = sum_of<W>(s_w, t, at.lane, waves);
                // aw is in units of the exponents to base 2
                const float ddt = fmaf(x, bl, aw * 0.693147181f) * slope[i];
                row_of<T>(a.dx, at.b, tile + t)[at.d] = (T)fmaf(delta[i], bl, skip * q[i]);
                row_of<T>(a.ddt, at.b, tile + t)[at.d] = (T)ddt;
                if (a.z.p) row_of<T>(a.dz, at.b, tile + t)[at.d] = (T)(dz[i] * p);
                dskip = fmaf(q[i], x, dskip);
                dbias += ddt;
            }
        }
        if (at.in)
            for (int64_t t = max(at.t0, at.len) + at.wave; t < at.t1; t += W) {
                row_of<T>(a.dx, at.b, t)[at.d] = (T)0.f;
                row_of<T>(a.ddt, at.b, t)[at.d] = (T)0.f;
                if (a.z.p) row_of<T>(a.dz, at.b, t)[at.d] = (T)0.f;
            }
        if (a.dh0 && at.chunk == 0 && at.in)
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int j = 0; j < kOwn; j++)
                    if (state(r, j) < a.S) a.dh0[(at.b * a.D + at.d) * a.S + state(r, j)] = m[r][j];
    }
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int j = 0; j < kOwn; j++)
            if (at.in && state(r, j) < a.S) g.part_a[((int64_t)first * a.S + state(r, j)) * a.D + at.d] = dA[r][j];
    __syncthreads();
    s_p[at.wave][0][at.lane] = dskip;
    s_p[at.wave][1][at.lane] = dbias;
    __syncthreads();
    if (at.wave < 2 && at.in)
        for (int k = at.wave; k < 2; k += W)
            g.part_v[((int64_t)first * 2 + k) * a.D + at.d] = sum_of<W>(s_p, k, at.lane, W);
}

// dB and dC: the slabs' parts in order.
template <class T> __global__ __launch_bounds__(256) void k_select_join_bc(SelectArgs a, Geom g)
{
    const int64_t i = (int64_t)block_of() * 256 + threadIdx.x, row = a.S * 2, rows = a.B * a.T;
    if (i >= rows * row) return;
    const int64_t bt = i / row, b = bt / a.T, t = bt - b * a.T;
    const int k = (int)(i - bt * row);
    const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), a.T) : a.T;
    float s = 0.f;
    if (t < len)
        for (uint32_t p = 0; p < g.slabs; p++) s += g.part_bc[p * rows * row + i];
    if (k < a.S) row_of<T>(a.dB, b, t)[k] = (T)s;
    else row_of<T>(a.dC, b, t)[k - a.S] = (T)s;
}

// dA, dskip and ddt_bias: the workgroups' parts in order, 64 channels of one state
// per workgroup, its wavefronts taking every fourth part.
__global__ __launch_bounds__(256) void k_select_join(SelectArgs a, Geom g)
{
    __shared__ float red[4][64];
    const uint32_t block = block_of();
    if (block >= g.slabs * (uint32_t)(a.S + 2)) return;
    const int n = (int)(block / g.slabs), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t d = (int64_t)(block % g.slabs) * 64 + lane;
    const float *from = n < a.S ? g.part_a + n * a.D : g.part_v + (n - a.S) * a.D;
    const int64_t step = (n < a.S ? a.S : 2) * a.D;
    float s = 0.f;
    if (d < a.D)
#pragma unroll 4
        for (uint32_t r = wave; r < g.rows; r += 4) s += from[r * step + d];
    red[wave][lane] = s;
    __syncthreads();
    if (wave || d >= a.D) return;
    s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
    if (n < a.S) a.dA[d * a.S + n] = s;
    else if (n == a.S && a.dskip) a.dskip[d] = s;
    else if (n == a.S + 1 && a.ddt_bias) a.ddt_bias[d] = s;
}

// ------------------------------------------------------------------ launches

int64_t slabs_of(int64_t D) { return (D + 63) / 64; }

// Wavefronts of a workgroup: a power of two that holds all states, kOwn each.
int waves_of(int64_t S, int most)
{
    int w = 1;
    while (w < most && w * kOwn < S) w *= 2;
    return w;
}

// Chunks of time.
struct Cut {
    int chunks;
    int64_t chunk;
};
Cut cut_of(int64_t B, int64_t T, int64_t D, int64_t S)
{
    const int64_t rows = std::max<int64_t>(1, B * slabs_of(D)), full = 512 * 4 / waves_of(S, 8);
    int64_t n = 1;
    if (rows * 3 <= full) n = std::min((full + rows - 1) / rows, (T + 127) / 128);
    if (n < 3) n = 1;
    const int64_t chunk = std::max<int64_t>(kTile, ((T + n - 1) / n + kTile - 1) / kTile * kTile);
    return {(int)std::max<int64_t>(1, (T + chunk - 1) / chunk), chunk};
}

// Workgroups per slab of the gradient, each of which leaves its sums for dA.
int64_t grad_rows(int64_t B, const Cut &c, int64_t D)
{
    return std::min(B * c.chunks, std::max<int64_t>(1, 4096 / slabs_of(D)));
}

size_t place(const SelectArgs &a, bool grad, Geom &g)
{
    Carver ws;
    const Cut c = cut_of(a.B, a.T, a.D, a.S);
    const size_t f = sizeof(float), bsd = (size_t)a.B * a.S * a.D;
    g.chunks = c.chunks, g.chunk = c.chunk;
    g.slabs = (uint32_t)slabs_of(a.D);
    char *base = (char *)a.ws;
    const auto take = [&](size_t n) { return (float *)(base + ws.take(n * f)); };
    if (c.chunks > 1) {
        if (!grad) g.start = take(bsd);
        g.ends = take(bsd * c.chunks);
        g.sums = take((size_t)a.B * c.chunks * a.D);
    }
    if (grad) {
        g.rows = (uint32_t)grad_rows(a.B, c, a.D);
        g.part_bc = take((size_t)g.slabs * a.B * a.T * 2 * a.S);
        g.part_a = take((size_t)g.rows * a.S * a.D);
        g.part_v = take((size_t)g.rows * 2 * a.D);
    }
    return ws.used;
}

template <class T, int W> hipError_t select_w(const SelectArgs &a, Geom g, hipStream_t s)
{
    if (g.chunks > 1) {
        const int64_t blocks = a.B * (g.chunks - 1) * g.slabs;
        g.blocks = (uint32_t)blocks;
        k_select<T, W, true><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
    }
    const int64_t blocks = a.B * g.chunks * g.slabs;
    g.blocks = (uint32_t)blocks;
    k_select<T, W, false><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
    return hipGetLastError();
}

template <class T> hipError_t select_t(const SelectArgs &a, hipStream_t s)
{
    Geom g{};
    place(a, false, g);
    switch (waves_of(a.S, 16)) {
    case 1: return select_w<T, 1>(a, g, s);
    case 2: return select_w<T, 2>(a, g, s);
    case 4: return select_w<T, 4>(a, g, s);
    case 8: return select_w<T, 8>(a, g, s);
    default: return select_w<T, 16>(a, g, s);
    }
}

template <class T, int W, int R> hipError_t grad_w(const SelectArgs &a, Geom g, hipStream_t s)
{
    if (g.rows) {
        const int64_t blocks = (int64_t)g.rows * g.slabs;
        g.blocks = (uint32_t)blocks;
        k_select_grad<T, W, R><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
    }
    return hipGetLastError();
}

template <class T, int W> void back_w(const SelectArgs &a, Geom g, hipStream_t s)
{
    const int64_t blocks = a.B * (g.chunks - 1) * g.slabs;
    g.blocks = (uint32_t)blocks;
    k_select_back<T, W><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
}

template <class T> hipError_t grad_t(const SelectArgs &a, hipStream_t s)
{
    Geom g{};
    place(a, true, g);
    if (g.chunks > 1 && g.rows) switch (waves_of(a.S, 16)) {
        case 1: back_w<T, 1>(a, g, s); break;
        case 2: back_w<T, 2>(a, g, s); break;
        case 4: back_w<T, 4>(a, g, s); break;
        case 8: back_w<T, 8>(a, g, s); break;
        default: back_w<T, 16>(a, g, s);
        }
    hipError_t e;
    switch (waves_of(a.S, 8)) {
    case 1: e = grad_w<T, 1, 1>(a, g, s); break;
    case 2: e = grad_w<T, 2, 1>(a, g, s); break;
    case 4: e = grad_w<T, 4, 1>(a, g, s); break;
    default: e = a.S <= 32 ? grad_w<T, 8, 1>(a, g, s) : grad_w<T, 8, 2>(a, g, s);
    }
    if (e != hipSuccess) return e;
    const int64_t n = a.B * a.T * 2 * a.S;
    if (n) k_select_join_bc<T><<<grid_of((n + 255) / 256), 256, 0, s>>>(a, g);
    k_select_join<<<grid_of((int64_t)g.slabs * (a.S + 2)), 256, 0, s>>>(a, g);
    return hipGetLastError();
}

} // namespace

size_t select_workspace(int64_t B, int64_t T, int64_t D, int64_t S)
{
    SelectArgs a{};
    a.B = B, a.T = T, a.D = D, a.S = (int)S;
    Geom g{};
    return place(a, false, g);
}

size_t select_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t S)
{
    SelectArgs a{};
    a.B = B, a.T = T, a.D = D, a.S = (int)S;
    Geom g{};
    return place(a, true, g);
}

hipError_t launch_select(int32_t type, const SelectArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return select_t<float>(a, s);
    if (type == TQ_BF16) return select_t<__bf16>(a, s);
    return select_t<_Float16>(a, s);
}

hipError_t launch_select_grad(int32_t type, const SelectArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return grad_t<float>(a, s);
    if (type == TQ_BF16) return grad_t<__bf16>(a, s);
    return grad_t<_Float16>(a, s);
}

} // namespace tq
