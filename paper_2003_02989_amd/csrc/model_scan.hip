// model_scan.hip -- the selective state space scan over time and its gradients.
//
//   d_t = softplus(dt_t + bias),  h_t = exp(d_t A) h_{t-1} + d_t x_t B_t,
//   y_t = (C_t . h_t + skip x_t) silu(z_t),
//
// D channels of S states each.  What bounds it are the vector units: an element of
// state, that is a channel, state and step, costs some nine issue slots, two of them
// its exponential, which runs at half rate.  So an element's exponential is formed
// once, and nothing else is done per state that can be done per channel: a lane holds
// a channel with four of its states in registers, and a workgroup of W wavefronts
// holds 64 channels with up to 4 W states.  Steps go in tiles of 16: the wavefronts share
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

#include "model_device.h"
#include "seq.h"

namespace tq {
namespace {

constexpr int kTile = TQ_STATES_PIECE;  // steps
constexpr int kFewSteps = 4;            // of a gradient's records, for the form for few
constexpr int kOwn = 4;                 // states of a lane
constexpr float kLog2e = 1.44269504088896341f;

struct Geom {
    uint32_t blocks;       // of the launch
    uint32_t slabs, rows;  // slabs of 64 channels; gradient: workgroups per slab
    int chunks;
    int64_t chunk;         // steps of a chunk, whole tiles
    float *ends, *sums;    // [B][chunks][S][D], [B][chunks][D]
    float *part_bc;        // [slabs][B][T][2][S]
    float *part_a, *part_v;  // [rows][S][D], [rows][2][D]
};

// What a workgroup and a lane work on.
struct Place {
    int64_t b, len, t0, t1, n1;  // the chunk's steps [t0, t1), of the record [t0, n1)
    int chunk, wave, lane;
    uint32_t slab;
    int64_t d;    // the lane's channel
    uint32_t dc;  // one that there is
    bool in;
    __device__ void lanes(uint32_t slab_, int64_t D)
    {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        slab = slab_;
        d = (int64_t)slab * 64 + lane;
        in = d < D;
        dc = (uint32_t)(in ? d : D - 1);
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
// A log2 e is rounded, as the product with d is: a decay is off by up to |d A| 2^-24
// more than exp(d A) would be.  Putting the lost part back, as exp_of does for what is
// formed once per channel, would take one more instruction per element of state.
__device__ __forceinline__ float exponent(float A)
{
    const float v = A * kLog2e;
    return fabsf(v) <= 3.4e38f || v != v ? v : copysignf(3.4e38f, v);
}

// The rows of an array that a wavefront reads or writes: the first of its steps in
// a tile, going on by whole tiles, and the lane's element.
template <class T> struct Rows {
    char *p;
    int64_t step;  // bytes
    template <class S> __device__ __forceinline__ void start(const S &s, int64_t b, int64_t t)
    {
        step = s.step * (int64_t)sizeof(T);
        p = (char *)s.p + b * s.batch * (int64_t)sizeof(T) + t * step;
    }
    __device__ __forceinline__ void move(int steps) { p += steps * step; }
    __device__ __forceinline__ T get(int64_t i, uint32_t c) const { return *(const T *)(p + i * step + c * (uint32_t)sizeof(T)); }
    __device__ __forceinline__ void put(int64_t i, uint32_t c, float v) const
    {
        *(T *)(p + i * step + c * (uint32_t)sizeof(T)) = (T)v;
    }
};

// A tile's inputs: one read ahead by registers, and what the wavefronts share of
// it.  Steps are dealt out in runs of kTile / W; steps past the record's end read
// its last one and count as zero.  R: groups of four states of a wavefront.
template <class T, int W, int R, bool X, bool Z, bool DY, bool PB, bool PC> struct Feed {
    static constexpr int PER = kTile / W, BC = R * 2;  // steps, B and C elements of a thread
    static constexpr int APART = 8 / R;                // steps from one of the latter to the next
    Rows<T> rx, rdt, rz, rdy;
    const T *pbc;
    int64_t step_bc;
    bool on_bc;
    int t_bc, slot_bc;
    T x[X ? PER : 1], dt[PER], z[Z ? PER : 1], dy[DY ? PER : 1], bc[BC];
    __device__ __forceinline__ void start(const SelectArgs &a, const Place &at, int64_t tile)
    {
        const int64_t t = tile + at.wave * PER;
        if constexpr (X) rx.start(a.x, at.b, t);
        rdt.start(a.dt, at.b, t);
        if constexpr (Z) rz.start(a.z, at.b, t);
        if constexpr (DY) rdy.start(a.dy, at.b, t);
        const int v = threadIdx.x, n = v % (4 * W * R);
        const bool c = v / (4 * W * R) % 2;
        t_bc = v / (8 * W * R);
        slot_bc = (n / 4) * 8 + c * 4 + n % 4;
        on_bc = n < a.S && (c ? PC : PB);
        const Steps &from = c ? a.Cm : a.Bm;
        step_bc = from.step;
        pbc = (const T *)from.p + at.b * from.batch + (tile + t_bc) * from.step + min(n, a.S - 1);
    }
    __device__ __forceinline__ void move(int steps)
    {
        if constexpr (X) rx.move(steps);
        rdt.move(steps);
        if constexpr (Z) rz.move(steps);
        if constexpr (DY) rdy.move(steps);
        pbc += steps * step_bc;
    }
    __device__ __forceinline__ void fetch(const SelectArgs &a, const Place &at, int64_t tile)
    {
        if (tile + kTile <= at.len) take([](int i) { return i; }, [](int i) { return i; }, a, at);
        else {
            const int left = (int)(at.len - 1 - tile);  // the last step there is
            take([&](int i) { return min(i, left - at.wave * PER); }, [&](int i) { return min(i, left - t_bc); }, a, at);
        }
    }
    template <class F, class G>
    __device__ __forceinline__ void take(F &&row, G &&row_bc, const SelectArgs &a, const Place &at)
    {
#pragma unroll
        for (int i = 0; i < PER; i++) {
            if constexpr (X) x[i] = rx.get(row(i), at.dc);
            dt[i] = rdt.get(row(i), at.dc);
            if constexpr (DY) dy[i] = rdy.get(row(i), at.dc);
        }
        if constexpr (Z)
            if (a.z.p) {
#pragma unroll
                for (int i = 0; i < PER; i++) z[i] = rz.get(row(i), at.dc);
            }
#pragma unroll
        for (int i = 0; i < BC; i++) bc[i] = pbc[row_bc(i * APART) * step_bc];
    }
    // B and C, [step][group of four states][B, C]
    __device__ __forceinline__ void share_bc(const Place &at, int64_t tile, float *to) const
    {
#pragma unroll
        for (int i = 0; i < BC; i++) {
            const int t = t_bc + i * APART;
            to[t * 8 * W * R + slot_bc] = on_bc && tile + t < at.len ? (float)bc[i] : 0.f;
        }
    }
};

// The wavefronts' parts, in the order in which lanes exchange theirs in k_select_step.
template <int W, int N> __device__ __forceinline__ float sum_of(const float (*p)[N][64], int t, int lane)
{
    float s[W];
#pragma unroll
    for (int w = 0; w < W; w++) s[w] = p[w][t][lane];
#pragma unroll
    for (int n = W / 2; n > 0; n /= 2)
#pragma unroll
        for (int w = 0; w < n; w++) s[w] += s[w + n];
    return s[0];
}

// The steps of a chunk past the record's end.
template <class T> __device__ __forceinline__ void zeros(const StepsOut &to, const Place &at, int waves)
{
    Rows<T> r;
    const int64_t from = max(at.t0, at.len) + at.wave;
    r.start(to, at.b, from);
    if (at.in)
        for (int64_t t = from; t < at.t1; t += waves) {
            r.put(0, at.dc, 0.f);
            r.move(waves);
        }
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
    const int n0 = at.wave * kOwn;
    const bool some = n0 < a.S;  // the wavefront has states

    float A[kOwn], h[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; j++) {
        const bool there = at.in && n0 + j < a.S;
        A[j] = there && a.A ? exponent(a.A[at.d * a.S + n0 + j]) : 0.f;
        h[j] = 0.f;
        if (!there) continue;
        if (!ENDS && g.chunks > 1) h[j] = g.ends[((at.b * g.chunks + at.chunk) * a.S + n0 + j) * a.D + at.d];
        else if (at.chunk == 0 && a.h0) h[j] = a.h0[(at.b * a.D + at.d) * a.S + n0 + j];
    }
    const float bias = a.dt_bias ? a.dt_bias[at.dc] : 0.f;
    const float skip = !ENDS && a.skip ? a.skip[at.dc] : 0.f;
    float total = 0.f;
    if (!ENDS && !some)  // parts that are none
#pragma unroll
        for (int t = 0; t < kTile; t++) s_p[at.wave][t][at.lane] = 0.f;
    Feed<T, W, 1, true, !ENDS, false, true, !ENDS> in;
    Rows<T> ry;
    T x[PER], z[PER];
    if (at.t0 < at.n1) {
        in.start(a, at, at.t0);
        in.fetch(a, at, at.t0);
        if constexpr (!ENDS) ry.start(a.y, at.b, at.t0 + at.wave * PER);
    }
    float *states = !ENDS && a.states
                        ? a.states + ((at.b * ((a.T + kTile - 1) / kTile) + at.t0 / kTile) * a.S + n0) * a.D + at.d : nullptr;
    for (int64_t tile = at.t0; tile < at.n1; tile += kTile) {
        const int n = (int)min((int64_t)kTile, at.n1 - tile);  // steps
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int t = at.wave * PER + i;
            float slope, d = softplus<T>((float)in.dt[i] + bias, slope), u = d * (float)in.x[i];
            if (t >= n) d = u = 0.f;
            s_d[t][at.lane] = d;
            s_u[t][at.lane] = u;
            if constexpr (ENDS) total += d;
            else {
                x[i] = in.x[i];
                z[i] = in.z[i];
            }
        }
        in.share_bc(at, tile, &s_bc[0][0][0][0]);
        __syncthreads();
        if (tile + kTile < at.n1) {
            in.move(kTile);
            in.fetch(a, at, tile + kTile);
        }
        if (some) {
            if (!ENDS && states && at.in) {
#pragma unroll
                for (int j = 0; j < kOwn; j++)
                    if (n0 + j < a.S) states[(int64_t)j * a.D] = h[j];
            }
#pragma unroll
            for (int t = 0; t < kTile; t++) {
                if (t % 4 == 0 && t >= n) break;
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
            if (states) states += (int64_t)a.S * a.D;
            float y[PER];
#pragma unroll
            for (int i = 0; i < PER; i++) y[i] = fmaf(skip, (float)x[i], sum_of<W>(s_p, at.wave * PER + i, at.lane));
            if (a.z.p) {
#pragma unroll
                for (int i = 0; i < PER; i++) y[i] *= (float)z[i] * sigmoid<T>((float)z[i]);
            }
            if (at.in)
#pragma unroll
                for (int i = 0; i < PER; i++)
                    if (at.wave * PER + i < n) ry.put(i, at.dc, y[i]);
            ry.move(kTile);
        }
    }
    if constexpr (ENDS) {
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
    } else {
        const bool last = at.len == 0 ? at.chunk == 0 : at.t0 < at.len && at.len <= at.t1;
        if (a.h_last && last && at.in)
#pragma unroll
            for (int j = 0; j < kOwn; j++)
                if (n0 + j < a.S) a.h_last[(at.b * a.D + at.d) * a.S + n0 + j] = h[j];
        zeros<T>(a.y, at, W);
    }
}

// Turns what the chunks end with into what they start with, chunk by chunk, in
// place: a lane has a channel's state.  Forwards from h0, the first chunk's end being
// the state itself; backwards from the record's last chunk, whose end is it.
template <bool BACK> __global__ __launch_bounds__(64) void k_select_chain(SelectArgs a, Geom g)
{
    const int64_t i = (int64_t)block_of() * 64 + threadIdx.x, sd = a.S * a.D;
    if (i >= a.B * sd) return;
    const int64_t b = i / sd, n = i - b * sd, s = n / a.D, d = n - s * a.D;
    const float A = exponent(a.A[d * a.S + s]);
    const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), a.T) : a.T;
    const int top = BACK ? (int)(max(len - 1, (int64_t)0) / g.chunk) : g.chunks - 1;
    float h = BACK || !a.h0 ? 0.f : a.h0[(b * a.D + d) * a.S + s];
    const int64_t first = b * g.chunks + (BACK ? top : 0), along = BACK ? -1 : 1;
    float *end = g.ends + first * sd + n;
    const float *sum = g.sums + first * a.D + d;
    const auto step = [&](int k, float *at, float e, float w) {
        *at = h;
        h = k == 0 ? e : fmaf(__builtin_amdgcn_exp2f(w * A), h, e);
    };
    constexpr int N = 32;  // read together
    int k = 0;
    for (; k + N <= top; k += N, end += along * N * sd, sum += along * N * a.D) {
        float e[N], w[N];
#pragma unroll
        for (int j = 0; j < N; j++) {
            e[j] = end[along * j * sd];
            w[j] = sum[along * j * a.D];
        }
#pragma unroll
        for (int j = 0; j < N; j++) step(k + j, end + along * j * sd, e[j], w[j]);
    }
#pragma unroll 4
    for (; k < top; k++, end += along * sd, sum += along * a.D) step(k, end, *end, *sum);
    *end = h;  // the last one's own end is not needed
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
    Feed<T, W, 1, false, true, true, false, true> in;
    const int64_t top = at.t0 + (at.n1 - at.t0 - 1) / kTile * kTile;
    in.start(a, at, top);
    in.fetch(a, at, top);
    for (int64_t tile = top; tile >= at.t0; tile -= kTile) {
        const int n = (int)min((int64_t)kTile, at.n1 - tile);
        float gate[PER];
#pragma unroll
        for (int i = 0; i < PER; i++) gate[i] = 1.f;
        if (a.z.p) {
#pragma unroll
            for (int i = 0; i < PER; i++) gate[i] = (float)in.z[i] * sigmoid<T>((float)in.z[i]);
        }
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int t = at.wave * PER + i;
            float slope, d = softplus<T>((float)in.dt[i] + bias, slope), q = (float)in.dy[i] * gate[i];
            if (t >= n) d = q = 0.f;
            s_d[t][at.lane] = d;
            s_q[t][at.lane] = q;
            total += d;
        }
        in.share_bc(at, tile, &s_bc[0][0][0][0]);
        __syncthreads();
        if (tile > at.t0) {
            in.move(-kTile);
            in.fetch(a, at, tile - kTile);
        }
        if (n0 < a.S)
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

// Sums over a wavefront's lanes of eight values of each of 16 steps.  Each exchange
// between lanes adds up two values, either in one half of the lanes: four values over
// the four rows of 16 lanes at once; the sums of two steps over lanes 8 apart, their
// pairs over lanes mirrored in eight, then 2 and 1 apart, until the lanes of a row
// hold a step each.  Three instructions for two values in place of one and an exchange
// a value and distance: the kernel takes 517 us in place of 648 (the mean of 16 x
// 2048 x 1024 and 32 x 1024 x 1024 bf16).
struct LaneSums {
    float held[2][4];
    template <int N> __device__ __forceinline__ static float join(float a, float b)
    {
        // rotation by 8; mirror of eight lanes; permutations of four
        constexpr int kDpp = N == 8 ? 0x128 : N == 4 ? 0x141 : N == 2 ? 0x4e : 0xb1;
        const bool high = threadIdx.x & N;
        const float keep = high ? b : a, give = high ? a : b;
        return keep + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, give), kDpp, 0xf, 0xf, true));
    }
    // of both fours; the rows keep value 0, 2, 1, 3.  (All exchanges of a kind in a row:
    // what was written just before is waited for.)
    __device__ __forceinline__ static void rows(const float (&v)[8], float (&sum)[2])
    {
        const auto bits = [](float f) { return __builtin_bit_cast(unsigned, f); };
        const auto val = [](unsigned u) { return __builtin_bit_cast(float, u); };
        float m[4];
        unsigned a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const auto p = __builtin_amdgcn_permlane32_swap(bits(v[2 * i]), bits(v[2 * i + 1]), false, false);
            a[i] = p[0], b[i] = p[1];
        }
#pragma unroll
        for (int i = 0; i < 4; i++) m[i] = val(a[i]) + val(b[i]);  // halves: value 2 i, 2 i + 1
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const auto p = __builtin_amdgcn_permlane16_swap(bits(m[2 * i]), bits(m[2 * i + 1]), false, false);
            a[i] = p[0], b[i] = p[1];
        }
#pragma unroll
        for (int i = 0; i < 2; i++) sum[i] = val(a[i]) + val(b[i]);
    }
    __device__ __forceinline__ static void enter(int t, float v, float (&held)[4])
    {
        if (t & 1) held[0] = v;
        else if (v = join<8>(v, held[0]); t & 2) held[1] = v;
        else if (v = join<4>(v, held[1]); t & 4) held[2] = v;
        else if (v = join<2>(v, held[2]); t & 8) held[3] = v;
        else held[0] = join<1>(v, held[3]);
    }
    // the steps come from the last (15; what is cleared: zeros) to the first
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int k = 0; k < 4; k++) held[0][k] = held[1][k] = 0.f;
    }
    __device__ __forceinline__ void add(int t, const float (&v)[8])
    {
        float sum[2];
        rows(v, sum);
        enter(t, sum[0], held[0]);
        enter(t, sum[1], held[1]);
    }
    // of four of the values, in the lanes of the step and value below
    __device__ __forceinline__ float sum(int four) const { return held[four][0]; }
    __device__ static int step_of(int lane) { return (int)(__builtin_bitreverse32((uint32_t)lane & 15) >> 28); }
    __device__ static int value_of(int lane) { return lane >> 5 | (lane >> 4 & 1) << 1; }
};

// N: the steps of a tile that are worked on: all of them, or the first four for records of
// no more (1000 x 1 x 2000 fp16: 945 us with all, 692 with four).
// All 256 registers are taken, and a lane spills 44 (W = 8) to 632 bytes (W = 1), for the
// 16 states a channel of most models 132 (W = 4): 16 steps of decays and states are 132
// registers, the nine values that each of a wavefront's 16 / W steps keeps as many as 144.
template <class T, int W, int R, int N> __global__ __launch_bounds__(64 * W, 2) void k_select_grad(SelectArgs a, Geom g)
{
    constexpr int PER = kTile / W;
    __shared__ float s_d[kTile][64], s_u[kTile][64], s_q[kTile][64];
    __shared__ __attribute__((aligned(16))) float s_bc[kTile][W * R][2][4];
    __shared__ float s_p[W][N][64], s_l[W][N][64], s_w[W][N][64];
    const uint32_t block = block_of();
    if (block >= g.blocks) return;
    Place at;
    const uint32_t first = block / g.slabs;
    at.lanes(block - first * g.slabs, a.D);
    const float bias = a.dt_bias ? a.dt_bias[at.dc] : 0.f, skip = a.skip ? a.skip[at.dc] : 0.f;
    float A[R][kOwn], dA[R][kOwn], m[R][kOwn], h0[R][kOwn], dskip = 0.f, dbias = 0.f;
    const auto state = [&](int r, int j) { return (r * W + at.wave) * kOwn + j; };
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int j = 0; j < kOwn; j++) {
            const int n = state(r, j);
            A[r][j] = at.in && n < a.S && a.A ? exponent(a.A[at.d * a.S + n]) : 0.f;
            dA[r][j] = 0.f;
        }
    if (state(0, 0) >= a.S)  // parts that are none
#pragma unroll
        for (int t = 0; t < N; t++) s_p[at.wave][t][at.lane] = s_l[at.wave][t][at.lane] = s_w[at.wave][t][at.lane] = 0.f;
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
                if (at.chunk < top_chunk) m[r][j] = g.ends[((at.b * g.chunks + at.chunk) * a.S + n) * a.D + at.d];
                else if (a.dh_last) m[r][j] = a.dh_last[(at.b * a.D + at.d) * a.S + n];
            }
        Feed<T, W, R, true, true, true, true, true> in;
        Rows<T> rdx, rddt, rdz;
        const int64_t top = at.t0 + (at.n1 - at.t0 - 1) / kTile * kTile;
        const auto saved = [&](int64_t tile) {
            const float *from = a.states_in + (at.b * pieces + tile / kTile) * a.S * a.D + at.dc;
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int j = 0; j < kOwn; j++) {
                    h0[r][j] = 0.f;
                    if (at.in && state(r, j) < a.S) h0[r][j] = from[(int64_t)state(r, j) * a.D];
                }
        };
        if (at.t0 < at.n1) {
            in.start(a, at, top);
            in.fetch(a, at, top);
            saved(top);
            const int64_t t = top + at.wave * PER;
            rdx.start(a.dx, at.b, t);
            rddt.start(a.ddt, at.b, t);
            rdz.start(a.dz, at.b, t);
        }
        float *part = g.part_bc + ((at.slab * a.B + at.b) * a.T + top + LaneSums::step_of(at.lane)) * 2 * a.S;
        for (int64_t tile = top; tile >= at.t0 && at.t0 < at.n1; tile -= kTile) {
            const int n = (int)min((int64_t)kTile, at.n1 - tile);
            float delta[PER], slope[PER], q[PER], dz[PER], x[PER];
#pragma unroll
            for (int i = 0; i < PER; i++) {
                delta[i] = softplus<T>((float)in.dt[i] + bias, slope[i]);
                q[i] = (float)in.dy[i];
                dz[i] = 0.f;
                x[i] = (float)in.x[i];
            }
            if (a.z.p) {
#pragma unroll
                for (int i = 0; i < PER; i++) {
                    const float z = (float)in.z[i], dy = q[i];
                    float s, c;
                    sigmoids<T>(z, s, c);
                    q[i] = dy * (z * s);
                    dz[i] = dy * (s * fmaf(z, c, 1.f));
                }
            }
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int t = at.wave * PER + i;
                const bool there = at.in && t < n;
                s_d[t][at.lane] = there ? delta[i] : 0.f;
                s_u[t][at.lane] = there ? delta[i] * x[i] : 0.f;
                s_q[t][at.lane] = there ? q[i] : 0.f;
            }
            in.share_bc(at, tile, &s_bc[0][0][0][0]);
            __syncthreads();
            float hs[R][kOwn];
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int j = 0; j < kOwn; j++) hs[r][j] = h0[r][j];
            if (tile > at.t0) {
                in.move(-kTile);
                in.fetch(a, at, tile - kTile);
                saved(tile - kTile);
            }
#pragma unroll
            for (int r = 0; r < R; r++) {
                const int n0 = state(r, 0), group = r * W + at.wave;
                if (n0 >= a.S) continue;
                float h[N + 1][kOwn], e[N][kOwn];
#pragma unroll
                for (int j = 0; j < kOwn; j++) h[0][j] = hs[r][j];
#pragma unroll
                for (int t = 0; t < N; t++) {
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
                // what the steps forwards read is read again, not kept: 160 registers
                asm volatile("" ::: "memory");
                LaneSums sums;
                if constexpr (N < kTile) sums.clear();
#pragma unroll
                for (int t = N - 1; t >= 0; t--) {
                    const float d = s_d[t][at.lane], u = s_u[t][at.lane], q = s_q[t][at.lane];
                    float bl = 0.f, aw = 0.f, v[2 * kOwn];
#pragma unroll
                    for (int j = 0; j < kOwn; j++) {
                        const float l = fmaf(s_bc[t][group][1][j], q, m[r][j]);
                        v[kOwn + j] = q * h[t + 1][j];
                        v[j] = u * l;
                        bl = fmaf(s_bc[t][group][0][j], l, bl);
                        m[r][j] = e[t][j] * l;
                        const float w = m[r][j] * h[t][j];
                        aw = fmaf(A[r][j], w, aw);
                        dA[r][j] = fmaf(d, w, dA[r][j]);
                    }
                    s_l[at.wave][t][at.lane] = r ? s_l[at.wave][t][at.lane] + bl : bl;
                    s_w[at.wave][t][at.lane] = r ? s_w[at.wave][t][at.lane] + aw : aw;
                    sums.add(t, v);
                }
                const float sb = sums.sum(0), sc = sums.sum(1);
                const int state_of = n0 + LaneSums::value_of(at.lane);
                if (LaneSums::step_of(at.lane) < n && state_of < a.S) {
                    part[state_of] = sb;
                    part[state_of + a.S] = sc;
                }
            }
            part -= kTile * 2 * a.S;
            __syncthreads();
            float dx[PER], ddt[PER];
#pragma unroll
            for (int i = 0; i < PER; i++) {
                const int t = at.wave * PER + i, in_lds = N < kTile ? min(t, N - 1) : t;
                const float p = fmaf(skip, x[i], sum_of<W>(s_p, in_lds, at.lane));
                const float bl = sum_of<W>(s_l, in_lds, at.lane), aw = sum_of<W>(s_w, in_lds, at.lane);
                // aw is in units of the exponents to base 2
                ddt[i] = fmaf(x[i], bl, aw * 0.693147181f) * slope[i];
                dx[i] = fmaf(delta[i], bl, skip * q[i]);
                dz[i] *= p;
                if (t < n) {
                    dskip = fmaf(q[i], x[i], dskip);
                    dbias += ddt[i];
                }
            }
            if (at.in)
#pragma unroll
                for (int i = 0; i < PER; i++) {
                    if (at.wave * PER + i >= n) continue;
                    rdx.put(i, at.dc, dx[i]);
                    rddt.put(i, at.dc, ddt[i]);
                    if (a.z.p) rdz.put(i, at.dc, dz[i]);
                }
            rdx.move(-kTile);
            rddt.move(-kTile);
            rdz.move(-kTile);
        }
        zeros<T>(a.dx, at, W);
        zeros<T>(a.ddt, at, W);
        if (a.z.p) zeros<T>(a.dz, at, W);
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
        for (int k = at.wave; k < 2; k += W) g.part_v[((int64_t)first * 2 + k) * a.D + at.d] = sum_of<W>(s_p, k, at.lane);
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
    const StepsOut &to = k < a.S ? a.dB : a.dC;
    ((T *)to.p)[b * to.batch + t * to.step + (k < a.S ? k : k - a.S)] = (T)s;
}

// dA, dskip and ddt_bias: the workgroups' parts in order, 64 channels of one state
// per workgroup, its wavefronts taking every 16th part.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void k_select_join(SelectArgs a, Geom g)
{
    __shared__ float red[kJoinWaves][64];
    const uint32_t block = block_of();
    if (block >= g.slabs * (uint32_t)(a.S + 2)) return;
    const int n = (int)(block / g.slabs), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t d = (int64_t)(block % g.slabs) * 64 + lane;
    const float *from = n < a.S ? g.part_a + n * a.D : g.part_v + (n - a.S) * a.D;
    const int64_t step = (n < a.S ? a.S : 2) * a.D;
    float s = 0.f;
    if (d < a.D)
#pragma unroll 8
        for (uint32_t r = wave; r < g.rows; r += kJoinWaves) s += from[r * step + d];
    red[wave][lane] = s;
    __syncthreads();
    if (wave || d >= a.D) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; w++) s += red[w][lane];
    if (n < a.S) a.dA[d * a.S + n] = s;
    else if (n == a.S && a.dskip) a.dskip[d] = s;
    else if (n == a.S + 1 && a.ddt_bias) a.ddt_bias[d] = s;
}

// ------------------------------------------------------------------ one step
// Bound by memory: the state is read and written.  L lanes hold a channel, four
// states each, so that a record's state is read in one piece; a thread takes the same
// channel of N records.  1024 x 512 x 16 bf16: 17.6 us from a cache, 22.5 us, 3.2 TB/s,
// from memory; 4096 records 75 us, 3.8 TB/s.
template <class T, int L, int N> __global__ __launch_bounds__(256) void k_select_step(SelectArgs a, uint32_t blocks)
{
    constexpr int PER = 256 / L;
    const uint32_t block = block_of(), slabs = (uint32_t)((a.D + PER - 1) / PER);
    if (block >= blocks) return;
    const int64_t d = (int64_t)(block % slabs) * PER + threadIdx.x / L, b0 = (int64_t)(block / slabs) * N;
    if (d >= a.D) return;  // all lanes of a channel
    const int n0 = threadIdx.x % L * kOwn, own = max(0, min(kOwn, a.S - n0));
    float h[N][kOwn], Bm[N][kOwn], Cm[N][kOwn], x[N], dt[N], z[N], A[kOwn] = {};
    bool on[N];
    load_part<kOwn>(a.A + d * a.S + n0, own, A);
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int64_t b = min(b0 + i, a.B - 1);
        on[i] = !a.lengths || a.lengths[b] > 0;
        if (a.h0) load_part<kOwn>(a.h0 + (b * a.D + d) * a.S + n0, own, h[i]);
        else
#pragma unroll
            for (int j = 0; j < kOwn; j++) h[i][j] = 0.f;
        x[i] = dt[i] = z[i] = 0.f;
        if (!on[i]) continue;
        x[i] = (float)((const T *)a.x.p)[b * a.x.batch + d];
        dt[i] = (float)((const T *)a.dt.p)[b * a.dt.batch + d];
        if (a.z.p) z[i] = (float)((const T *)a.z.p)[b * a.z.batch + d];
        load_part<kOwn>((const T *)a.Bm.p + b * a.Bm.batch + n0, own, Bm[i]);
        load_part<kOwn>((const T *)a.Cm.p + b * a.Cm.batch + n0, own, Cm[i]);
    }
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.f, skip = a.skip ? a.skip[d] : 0.f;
#pragma unroll
    for (int i = 0; i < N; i++) {
        if (b0 + i >= a.B) break;
        float y = 0.f;
        if (on[i]) {
            float slope, p = 0.f;
            const float delta = softplus<T>(dt[i] + bias, slope), u = delta * x[i];
#pragma unroll
            for (int j = 0; j < kOwn; j++)
                if (j < own) {
                    h[i][j] = fmaf(__builtin_amdgcn_exp2f(delta * exponent(A[j])), h[i][j], u * Bm[i][j]);
                    p = fmaf(Cm[i][j], h[i][j], p);
                }
            y = fmaf(skip, x[i], group_sum<L>(p));
            if (a.z.p) y *= z[i] * sigmoid<T>(z[i]);
        }
        if (a.h_last) store_part<kOwn>(a.h_last + ((b0 + i) * a.D + d) * a.S + n0, own, h[i]);
        if (n0 == 0) ((T *)a.y.p)[(b0 + i) * a.y.batch + d] = (T)y;
    }
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

// Chunks of time.  Forming every exponential once more costs less than leaving part of
// the chip idle; a round is as many workgroups of the gradient as the chip holds.
//  - Up to eight rounds, of chunks of at least 96 steps, and whole ones: forward and
//    gradient of 4 x 4096 x 512 bf16 258 us in two rounds, 280 in 2.7.
//    The forward call alone is cut as its gradient is; it gains nothing from more
//    chunks where there are more channels (400 x 1024 x 64 176 us whole, 204 cut).
//  - Records of different lengths are evened out by more workgroups and gain from
//    chunks where there are more channels: 20 x 1200 x 1200, three quarters of a round,
//    581 us and 709 without chunks (alike: 859 and 788); 64 x 512 x 512 fp32, a whole
//    one, 397 and 303.  Chunks of 64 steps or whole rounds of longer ones are the same
//    there (8 x 4099 x 1024 504 and 502 us, 12 x 3000 x 700 439 and 430).
//  - Where that is less than a round, one round of shorter chunks: 8 x 256 x 128 with 8
//    states 59 us in place of 118, the scan of 1 x 1000 x 200 23 in place of 34; below
//    96 steps there is nothing to gain (2 x 60 x 130: 59 and 51 us without).
struct Cut {
    int chunks;
    int64_t chunk;
};
Cut cut_of(int64_t B, int64_t T, int64_t D, int64_t S, bool ragged)
{
    const int64_t rows = std::max<int64_t>(1, B * slabs_of(D)), round = 2048 / waves_of(S, 8);
    int64_t n = 1;
    if (ragged ? rows * 6 <= round * 5 : rows * 3 <= round * 2) {
        const int64_t least = ragged ? 64 : 96;
        n = std::min((8 * round + rows - 1) / rows, (T + least - 1) / least);
        if (rows * n < round) n = T < 96 ? 1 : std::min(round / rows, T / kTile);
        else if (!ragged) n = rows * n / round * round / rows;
    }
    if (n < 3) n = 1;
    const int64_t chunk = std::max<int64_t>(kTile, ((T + n - 1) / n + kTile - 1) / kTile * kTile);
    return {(int)std::max<int64_t>(1, (T + chunk - 1) / chunk), chunk};
}

// Workgroups per slab of the gradient, each of which leaves its sums for dA.
int64_t grad_rows(int64_t B, const Cut &c, int64_t D)
{
    return std::min(B * c.chunks, std::max<int64_t>(1, 4096 / slabs_of(D)));
}

// (Records of different lengths are cut into no fewer chunks, and need no less space.)
size_t place(const SelectArgs &a, bool grad, bool ragged, Geom &g)
{
    Carver ws;
    const Cut c = cut_of(a.B, a.T, a.D, a.S, ragged);
    const size_t f = sizeof(float), bsd = (size_t)a.B * a.S * a.D;
    g.chunks = c.chunks, g.chunk = c.chunk;
    g.slabs = (uint32_t)slabs_of(a.D);
    char *base = (char *)a.ws;
    const auto take = [&](size_t n) { return (float *)(base + ws.take(n * f)); };
    if (c.chunks > 1) {
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
        k_select_chain<false><<<grid_of((a.B * a.S * a.D + 63) / 64), 64, 0, s>>>(a, g);
    }
    const int64_t blocks = a.B * g.chunks * g.slabs;
    g.blocks = (uint32_t)blocks;
    k_select<T, W, false><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
    return hipGetLastError();
}

// In fp32 a thread takes the same channel of four records where that leaves eight
// workgroups to a compute unit: states that come from memory take 63.7 us in place of
// 80.3 (4096 x 512 x 16), 20.6 in place of 22.6 at 8192 workgroups of one record each,
// at 4096 the same; from a cache 17.7 and 17.9 us, 10.9 and 10.2.  Where a lane holds
// a whole channel it gains nothing (4096 x 512 x 4: 23.3 and 22.6), and 16-bit inputs
// lose (bf16 1024 x 512 x 16: 26.7 and 22.5; 4096 records 80.3 and 75.4).
template <class T, int L> hipError_t step_l(const SelectArgs &a, hipStream_t s)
{
    const int64_t slabs = (a.D + 256 / L - 1) / (256 / L);
    if constexpr (sizeof(T) == 4 && L > 1)
        if (a.B * slabs >= 8192) {
            const int64_t blocks = (a.B + 3) / 4 * slabs;
            k_select_step<T, L, 4><<<grid_of(blocks), 256, 0, s>>>(a, (uint32_t)blocks);
            return hipGetLastError();
        }
    const int64_t blocks = a.B * slabs;
    k_select_step<T, L, 1><<<grid_of(blocks), 256, 0, s>>>(a, (uint32_t)blocks);
    return hipGetLastError();
}

template <class T> hipError_t select_t(const SelectArgs &a, hipStream_t s)
{
    const int lanes = waves_of(a.S, 16);  // of a channel
    // (more workgroups than are counted in 31 bits: the tiles have fewer, and give the same bits)
    if (a.T == 1 && !a.states && a.B * ((a.D + 256 / lanes - 1) / (256 / lanes)) <= INT32_MAX) switch (lanes) {
        case 1: return step_l<T, 1>(a, s);
        case 2: return step_l<T, 2>(a, s);
        case 4: return step_l<T, 4>(a, s);
        case 8: return step_l<T, 8>(a, s);
        default: return step_l<T, 16>(a, s);
        }
    Geom g{};
    if (place(a, false, a.lengths, g) > select_workspace(a.B, a.T, a.D, a.S)) return hipErrorInvalidValue;
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
        if (a.T <= kFewSteps) k_select_grad<T, W, R, kFewSteps><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
        else k_select_grad<T, W, R, kTile><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
    }
    return hipGetLastError();
}

template <class T, int W> void back_w(const SelectArgs &a, Geom g, hipStream_t s)
{
    const int64_t blocks = a.B * (g.chunks - 1) * g.slabs;
    g.blocks = (uint32_t)blocks;
    k_select_back<T, W><<<grid_of(blocks), 64 * W, 0, s>>>(a, g);
    k_select_chain<true><<<grid_of((a.B * a.S * a.D + 63) / 64), 64, 0, s>>>(a, g);
}

template <class T> hipError_t grad_t(const SelectArgs &a, hipStream_t s)
{
    Geom g{};
    if (place(a, true, a.lengths, g) > select_grad_workspace(a.B, a.T, a.D, a.S)) return hipErrorInvalidValue;
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
    k_select_join<<<grid_of((int64_t)g.slabs * (a.S + 2)), 64 * kJoinWaves, 0, s>>>(a, g);
    return hipGetLastError();
}

} // namespace

size_t select_workspace(int64_t B, int64_t T, int64_t D, int64_t S)
{
    SelectArgs a{};
    a.B = B, a.T = T, a.D = D, a.S = (int)S;
    Geom g{};
    return place(a, false, true, g);
}

size_t select_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t S)
{
    SelectArgs a{};
    a.B = B, a.T = T, a.D = D, a.S = (int)S;
    Geom g{};
    return place(a, true, true, g);
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
