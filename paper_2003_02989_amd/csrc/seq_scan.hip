// seq_scan.hip -- the gated linear recurrence over time and its gradients.
//
//   h_t = a_t h_{t-1} + c_t x_t,   a_t = sigmoid(g_t), c_t = 1 - a_t.
//
// Each step is the map h -> a h + b; maps compose to (A, B) pairs, so a stretch
// of time is summed up by one pair per channel.  A workgroup takes a segment of
// time of one record and a slab of channels: its wavefronts read kSteps steps
// each into registers, exchange their pairs through LDS, find the state the
// segment starts from and apply their steps to it: x and g are read once and y
// is written once, which is what bounds it.
//
// The state a segment starts from comes from the pairs of the segments before
// it, which their workgroups publish as soon as they have them, and replace by
// the state at the segment's end once they know that.  A workgroup looks back
// until it meets a state and goes forwards from there, pair by pair: whichever
// state it met, the result is that of one step after the other, to the bit.  A
// slot of all ones is not published yet.  Workgroups take their segments in the
// order in which they start (a ticket), earlier segments of all rows first, and
// wait for segments with lower tickets only; the lowest ticket that is not done
// waits for nobody, so every wait ends.
//
// The backward pass walks time the other way.  Pairs forwards give h_{t-1} from
// the saved state before the piece of TQ_SCAN_PIECE steps, and
//   l_t = dy_t + m_{t+1},  m_t = a_t l_t
// is the same kind of recurrence backwards.
#include <algorithm>
#include <type_traits>

#include "seq.h"
#include "seq_device.h"
#include "seq_slots.h"

namespace tq {
namespace {

// K: element type, channels per lane (16-bit elements of wide rows: two, 32 bits
// of a row), steps per wavefront.
constexpr int kWaves = 8, kThreads = 64 * kWaves;
template <class T_, int CV_, int STEPS> struct Kind {
    using T = T_;
    static constexpr int CV = CV_;
    static constexpr int steps = STEPS, seg = kWaves * steps, slab = 64 * CV;
    static_assert(seg % TQ_SCAN_PIECE == 0 && TQ_SCAN_PIECE % steps == 0,
                  "segments start at pieces, wavefronts at pieces or inside them");
};
constexpr int kPiece = TQ_SCAN_PIECE;
// exp(-v), v >= 0.  The product with log2 e is rounded, an error of up to
// v 2^-24 relative; for fp32 inputs what the rounding lost is put back.
template <class T> __device__ __forceinline__ float exp_neg(float v)
{
    constexpr float kLog2e = 1.44269504088896341f;
    if constexpr (sizeof(T) == 4) v = v > 1e4f ? 1e4f : v;  // infinities have no remainder; NaN stays
    const float t = -v * kLog2e;
    float e = __builtin_amdgcn_exp2f(t);
    if constexpr (sizeof(T) == 4) {
        // log2 e = kLog2e + 1.92596299e-8; ln 2 turns the lost part into a factor
        const float lost = fmaf(-v, kLog2e, -t) - v * 1.92596299e-8f;
        e = fmaf(e, lost * 0.693147181f, e);
    }
    return e;
}

// a = sigmoid(g) and c = 1 - a = sigmoid(-g), each to full relative accuracy.
template <class T> __device__ __forceinline__ void gate(float g, float &a, float &c)
{
    const float e = exp_neg<T>(fabsf(g));
    const float r = __builtin_amdgcn_rcpf(1.f + e), s = e * r;
    a = g >= 0.f ? r : s;
    c = g >= 0.f ? s : r;
}

// ------------------------------------------------------------ published pairs
// One 64-bit access each (seq_slots.h), of which a reader sees all or nothing.
// Agent scope reaches the other XCDs; nothing else is handed over, so no ordering
// is needed.
struct Geom {
    uint32_t rows, slabs;  // rows: records x slabs
    uint32_t first;        // of the launch
    int segs;
    Slot *slots;   // [segs][rows][kSlab]
    unsigned *ticket;
};

__device__ __forceinline__ void publish(Slot *p, Slot v)
{
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Slot look(const Slot *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// What is at p, which was `v` when last looked at, once it is published, or
// (`state`) once it is a state.  The count only keeps a broken launch from
// running for good: it is a matter of seconds, and its outputs are NaN.
__device__ __forceinline__ SlotPair await(const Slot *p, Slot v, bool state)
{
    for (int k = 0; !slot_ready(v, state) && k < 1 << 22; k++) {
        __builtin_amdgcn_s_sleep(1);
        v = look(p);
    }
    return slot_value(v, state);
}

__global__ __launch_bounds__(256) void k_scan_clear(Slot *slots, int64_t n, unsigned *ticket)
{
    const int64_t i = ((int64_t)block_of() * 256 + threadIdx.x) * 2;
    if (i == 0) *ticket = 0;
    if (i < n) *(ulonglong2 *)(slots + i) = make_ulonglong2(kEmpty, kEmpty);  // n is even
}

// What a workgroup works on.
template <class K> struct Place {
    uint32_t row;
    int64_t b;
    int seg, wave, lane, c0, n;  // the lane's first channel and their number
    int64_t len, t0;             // the record's length, the wavefront's first step
    int nv;                      // its steps that the record has
    // Segments of the row, in the order they are taken, that hold steps of the
    // record (one at least): the others write zeros and are not waited for.
    int seg0, seg1;
    __device__ Place(const ScanArgs &a, const Geom &g, uint32_t item, bool back)
    {
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        // in 32 bits: a division of 64 is a hundred instructions
        const uint32_t s = item / g.rows;
        row = item - s * g.rows;
        seg = (int)s;
        const uint32_t record = row / g.slabs;
        b = record;
        c0 = (int)(row - record * g.slabs) * K::slab + lane * K::CV;
        n = (int)max((int64_t)0, min((int64_t)K::CV, a.D - c0));
        if (n == 0) c0 = 0;
        len = a.T;
        if (a.lengths) len = min(max((int64_t)a.lengths[b], (int64_t)0), a.T);
        t0 = (int64_t)(back ? g.segs - 1 - seg : seg) * K::seg + wave * K::steps;
        nv = (int)max((int64_t)0, min((int64_t)K::steps, len - t0));
        const int some = max(1, (int)((len + K::seg - 1) / K::seg));
        seg0 = back ? g.segs - some : 0;
        seg1 = back ? g.segs : some;
    }
    __device__ bool idle() const { return seg < seg0 || seg >= seg1; }
};

__device__ __forceinline__ uint32_t take_item(const Geom &g)
{
    if (g.segs == 1) return g.first + block_of();
    __shared__ uint32_t item;
    if (threadIdx.x == 0) item = atomicAdd(g.ticket, 1u);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(item);
}

// The raw elements of one wavefront's steps.  Steps past the record's end read
// the last step again and lanes past D the first channel: no branches between
// the reads, and nothing is done with them.  With two channels per lane, a
// lane that has only the row's last one reads the one before it, too, and
// shifts (rows have more than 64 channels then).
template <class K> struct Raw {
    using T = typename K::T;
    using Word = std::conditional_t<sizeof(T) * K::CV == 4, uint32_t, uint16_t>;
    Word v[K::steps];
    int shift;
    __device__ __forceinline__ void load(const T *p, int64_t step, const Place<K> &at)
    {
        const bool odd = K::CV == 2 && at.n == 1;
        shift = odd ? 16 : 0;
        const uint32_t c = (uint32_t)(at.c0 - (odd ? 1 : 0)) * (uint32_t)sizeof(T);
        const char *row = (const char *)p;
        const int64_t bytes = step * (int64_t)sizeof(T);
        if (at.nv > 0)
#pragma unroll
            for (int i = 0; i < K::steps; i++) {
                __builtin_memcpy(&v[i], row + c, sizeof(Word));
                if (i + 1 < at.nv) row += bytes;
            }
    }
    __device__ __forceinline__ void at(int i, float (&f)[K::CV]) const
    {
        if constexpr (K::CV == 2) {
            const uint32_t w = v[i] >> shift;
            T lo, hi;
            const uint16_t l = (uint16_t)w, h = (uint16_t)(w >> 16);
            __builtin_memcpy(&lo, &l, 2);
            __builtin_memcpy(&hi, &h, 2);
            f[0] = (float)lo;
            f[1] = (float)hi;
        } else {
            T x;
            __builtin_memcpy(&x, &v[i], sizeof x);
            f[0] = (float)x;
        }
    }
};

// Steps [0, steps) of f, those that the record's array has.
template <class K>
__device__ __forceinline__ void put(typename K::T *p, int64_t step, int64_t T, const Place<K> &at,
                                    const float (&f)[K::steps][K::CV])
{
    using E = typename K::T;
    const int steps = (int)max((int64_t)0, min((int64_t)K::steps, T - at.t0));
    if (at.n == K::CV) {
        const uint32_t c = (uint32_t)at.c0 * (uint32_t)sizeof(E);
        char *row = (char *)p;
        const int64_t bytes = step * (int64_t)sizeof(E);
#pragma unroll
        for (int i = 0; i < K::steps; i++) {
            E e[K::CV];
#pragma unroll
            for (int j = 0; j < K::CV; j++) e[j] = (E)f[i][j];
            if (i < steps) __builtin_memcpy(row + c, e, sizeof e);
            row += bytes;
        }
    } else if (at.n) {
#pragma unroll
        for (int i = 0; i < K::steps; i++)
            if (i < steps) p[i * step + at.c0] = (E)f[i][0];
    }
}

// The state the segment starts from: `first` if it is the first of its row.
// Each wavefront looks at one slot of a window of kWaves, the nearest window
// first; the last of the kWindows windows waits for a state in its oldest slot.
// All wavefronts get the same result.
constexpr int kWindows = 4;
template <class K>
__device__ __forceinline__ void look_back(const Geom &g, const Place<K> &at, SlotPair (*win)[kWaves][K::slab],
                                          const float (&first)[K::CV], float (&h)[K::CV])
{
    constexpr int CV = K::CV;
    const int before = at.seg - at.seg0;  // segments of the row before this one
    int seen = 0;                         // of them, in `win`
    bool found[CV] = {};
    for (int k = 0; k < kWindows && seen < before; k++) {
        const int back = k * kWaves + at.wave;
        SlotPair q[CV];
#pragma unroll
        for (int j = 0; j < CV; j++) q[j] = SlotPair{slot_bits(1.f), 0.f};
        if (back < before) {
            const Slot *p = g.slots + ((int64_t)(at.seg - 1 - back) * g.rows + at.row) * K::slab + at.lane * CV;
            Slot v[CV];
#pragma unroll
            for (int j = 0; j < CV; j++) v[j] = look(p + j);
#pragma unroll
            for (int j = 0; j < CV; j++) q[j] = await(p + j, v[j], back == kWindows * kWaves - 1);
        }
#pragma unroll
        for (int j = 0; j < CV; j++) win[k][at.wave][at.lane * CV + j] = q[j];
        __syncthreads();
        seen = min((k + 1) * kWaves, before);
        bool all = true;
#pragma unroll
        for (int j = 0; j < CV; j++) {
#pragma unroll
            for (int w = 0; w < kWaves; w++) found[j] = found[j] || win[k][w][at.lane * CV + j].a == kState;
            all = all && found[j];
        }
        if (__all(all)) break;  // the same in every wavefront
    }
    // from the oldest slot on: a state starts anew
#pragma unroll
    for (int j = 0; j < CV; j++) h[j] = first[j];
    for (int back = seen - 1; back >= 0; back--)
#pragma unroll
        for (int j = 0; j < CV; j++) h[j] = slot_step(win[back / kWaves][back % kWaves][at.lane * CV + j], h[j]);
}

// ------------------------------------------------------------------ forward
// 24 x 4099 x 1024 bf16, ragged: 106 us, 3.8 TB/s; 1 x 100001 x 331 fp32:
// 113 us, 3.5 TB/s.  What is left to the memory's rate is waiting: for a
// segment's reads, for the other wavefronts' pairs and for the state before it.
template <class K> __global__ __launch_bounds__(kThreads, 4) void k_scan(ScanArgs a, Geom g)
{
    using T = typename K::T;
    constexpr int CV = K::CV, L = K::steps;
    __shared__ float2 agg[kWaves][K::slab];
    __shared__ SlotPair win[kWindows][kWaves][K::slab];
    const Place<K> at(a, g, take_item(g), false);
    T *y = (T *)a.y + at.b * a.yb + at.t0 * a.ys;
    float ga[L][CV], gb[L][CV], A[CV], B[CV];
    if (at.idle()) {
#pragma unroll
        for (int i = 0; i < L; i++)
#pragma unroll
            for (int j = 0; j < CV; j++) ga[i][j] = 0.f;
        put<K>(y, a.ys, a.T, at, ga);
        return;
    }
    Raw<K> rx, rg;
    rg.load((const T *)a.g + at.b * a.gb + at.t0 * a.gs, a.gs, at);
    rx.load((const T *)a.x + at.b * a.xb + at.t0 * a.xs, a.xs, at);
    float first[CV];
#pragma unroll
    for (int j = 0; j < CV; j++) first[j] = a.h0 && j < at.n ? a.h0[at.b * a.D + at.c0 + j] : 0.f;
#pragma unroll
    for (int j = 0; j < CV; j++) A[j] = 1.f, B[j] = 0.f;
    auto gates = [&](auto all) {
#pragma unroll
        for (int i = 0; i < L; i++) {
            const bool on = all.value || i < at.nv;
            float xv[CV], gv[CV];
            rx.at(i, xv);
            rg.at(i, gv);
#pragma unroll
            for (int j = 0; j < CV; j++) {
                float c;
                gate<T>(gv[j], ga[i][j], c);
                gb[i][j] = c * xv[j];
                if (!on) ga[i][j] = 1.f, gb[i][j] = 0.f;
                B[j] = fmaf(ga[i][j], B[j], gb[i][j]);
                A[j] *= ga[i][j];
            }
        }
    };
    if (at.nv == L) gates(std::true_type{});
    else gates(std::false_type{});
#pragma unroll
    for (int j = 0; j < CV; j++) agg[at.wave][at.lane * CV + j] = make_float2(A[j], B[j]);
    __syncthreads();
    const bool shared = at.seg + 1 < at.seg1 && at.wave == 0;  // later segments will ask
    Slot *slot = g.slots + ((int64_t)at.seg * g.rows + at.row) * K::slab + at.lane * CV;
    float wholeA[CV], wholeB[CV];
    if (shared) {
#pragma unroll
        for (int j = 0; j < CV; j++) wholeA[j] = 1.f, wholeB[j] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; w++)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                const float2 q = agg[w][at.lane * CV + j];
                wholeB[j] = fmaf(q.x, wholeB[j], q.y);
                wholeA[j] *= q.x;
            }
#pragma unroll
        for (int j = 0; j < CV; j++) {
            if (at.seg > at.seg0) publish(slot + j, pair_slot(wholeA[j], wholeB[j]));
        }
    }
    float h[CV];
    look_back<K>(g, at, win, first, h);
    if (shared)
#pragma unroll
        for (int j = 0; j < CV; j++) publish(slot + j, state_slot(fmaf(wholeA[j], h[j], wholeB[j])));
    for (int w = 0; w < at.wave; w++)
#pragma unroll
        for (int j = 0; j < CV; j++) {
            const float2 q = agg[w][at.lane * CV + j];
            h[j] = fmaf(q.x, h[j], q.y);
        }
    if (a.states && at.t0 % kPiece == 0 && at.nv > 0) {
        float *st = a.states + (at.b * ((a.T + kPiece - 1) / kPiece) + at.t0 / kPiece) * a.D;
#pragma unroll
        for (int j = 0; j < CV; j++)
            if (j < at.n) st[at.c0 + j] = h[j];
    }
#pragma unroll
    for (int i = 0; i < L; i++)
#pragma unroll
        for (int j = 0; j < CV; j++) {
            h[j] = fmaf(ga[i][j], h[j], gb[i][j]);
            ga[i][j] = i < at.nv ? h[j] : 0.f;
        }
    put<K>(y, a.ys, a.T, at, ga);
    if (a.h_last && at.seg == at.seg1 - 1 && at.wave == kWaves - 1)
#pragma unroll
        for (int j = 0; j < CV; j++)
            if (j < at.n) a.h_last[at.b * a.D + at.c0 + j] = h[j];
}

// ----------------------------------------------------------------- backward
// 24 x 4099 x 1024 bf16, ragged: 194 us, 3.6 TB/s.  Eight steps per wavefront:
// it holds twice what the forward pass holds per step.
template <class K> __global__ __launch_bounds__(kThreads, 4) void k_scan_grad(ScanArgs a, Geom g)
{
    using T = typename K::T;
    constexpr int CV = K::CV, L = K::steps, kBefore = kPiece / L;  // wavefronts of a piece
    __shared__ float2 agg[kWaves][K::slab];
    __shared__ SlotPair win[kWindows][kWaves][K::slab];
    __shared__ float rev[kWaves][K::slab];
    const Place<K> at(a, g, take_item(g), true);
    T *dx = (T *)a.dx + at.b * a.dxb + at.t0 * a.dxs, *dg = (T *)a.dg + at.b * a.dgb + at.t0 * a.dgs;
    float ga[L][CV], gc[L][CV], A[CV], Bf[CV], Br[CV];
    if (at.idle()) {
#pragma unroll
        for (int i = 0; i < L; i++)
#pragma unroll
            for (int j = 0; j < CV; j++) ga[i][j] = 0.f;
        put<K>(dx, a.dxs, a.T, at, ga);
        put<K>(dg, a.dgs, a.T, at, ga);
        return;
    }
    Raw<K> rx, rg, rd;
    rg.load((const T *)a.g + at.b * a.gb + at.t0 * a.gs, a.gs, at);
    rx.load((const T *)a.x + at.b * a.xb + at.t0 * a.xs, a.xs, at);
    rd.load((const T *)a.dy + at.b * a.dyb + at.t0 * a.dys, a.dys, at);
    float last[CV], h[CV];
#pragma unroll
    for (int j = 0; j < CV; j++) {
        last[j] = a.dh_last && j < at.n ? a.dh_last[at.b * a.D + at.c0 + j] : 0.f;
        h[j] = 0.f;
        if (at.nv > 0 && j < at.n)
            h[j] = a.states_in[(at.b * ((a.T + kPiece - 1) / kPiece) + at.t0 / kPiece) * a.D + at.c0 + j];
    }
#pragma unroll
    for (int j = 0; j < CV; j++) A[j] = 1.f, Bf[j] = Br[j] = 0.f;
    auto gates = [&](auto all) {
#pragma unroll
        for (int i = 0; i < L; i++) {
            const bool on = all.value || i < at.nv;
            float xv[CV], gv[CV];
            rx.at(i, xv);
            rg.at(i, gv);
#pragma unroll
            for (int j = 0; j < CV; j++) {
                gate<T>(gv[j], ga[i][j], gc[i][j]);
                float b = gc[i][j] * xv[j];
                if (!on) ga[i][j] = 1.f, gc[i][j] = b = 0.f;
                Bf[j] = fmaf(ga[i][j], Bf[j], b);
                A[j] *= ga[i][j];
            }
        }
#pragma unroll
        for (int i = L - 1; i >= 0; i--) {
            const bool on = all.value || i < at.nv;
            float d[CV];
            rd.at(i, d);
#pragma unroll
            for (int j = 0; j < CV; j++) Br[j] = on ? ga[i][j] * (Br[j] + d[j]) : Br[j];
        }
    };
    if (at.nv == L) gates(std::true_type{});
    else gates(std::false_type{});
#pragma unroll
    for (int j = 0; j < CV; j++) {
        agg[at.wave][at.lane * CV + j] = make_float2(A[j], Bf[j]);
        rev[at.wave][at.lane * CV + j] = Br[j];
    }
    __syncthreads();
    const bool shared = at.seg + 1 < at.seg1 && at.wave == 0;
    Slot *slot = g.slots + ((int64_t)at.seg * g.rows + at.row) * K::slab + at.lane * CV;
    float wholeA[CV], wholeB[CV];
    if (at.wave == 0) {
#pragma unroll
        for (int j = 0; j < CV; j++) wholeA[j] = 1.f, wholeB[j] = 0.f;
#pragma unroll
        for (int w = kWaves - 1; w >= 0; w--)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                const float q = agg[w][at.lane * CV + j].x;
                wholeB[j] = fmaf(q, wholeB[j], rev[w][at.lane * CV + j]);
                wholeA[j] *= q;
            }
#pragma unroll
        for (int j = 0; j < CV; j++) {
            if (shared && at.seg > at.seg0) publish(slot + j, pair_slot(wholeA[j], wholeB[j]));
        }
    }
    float m[CV];
    look_back<K>(g, at, win, last, m);
    if (at.wave == 0)
#pragma unroll
        for (int j = 0; j < CV; j++) {
            const float out = fmaf(wholeA[j], m[j], wholeB[j]);
            if (shared) publish(slot + j, state_slot(out));
            if (a.dh0 && at.seg == g.segs - 1 && j < at.n) a.dh0[at.b * a.D + at.c0 + j] = out;
        }
    for (int w = kWaves - 1; w > at.wave; w--)
#pragma unroll
        for (int j = 0; j < CV; j++) m[j] = fmaf(agg[w][at.lane * CV + j].x, m[j], rev[w][at.lane * CV + j]);
    for (int w = at.wave / kBefore * kBefore; w < at.wave; w++)
#pragma unroll
        for (int j = 0; j < CV; j++) {
            const float2 q = agg[w][at.lane * CV + j];
            h[j] = fmaf(q.x, h[j], q.y);
        }
    float away[L][CV];  // h_{t-1} - x_t, then dg
#pragma unroll
    for (int i = 0; i < L; i++) {
        float xv[CV];
        rx.at(i, xv);
#pragma unroll
        for (int j = 0; j < CV; j++) {
            away[i][j] = h[j] - xv[j];
            h[j] = fmaf(ga[i][j], h[j], gc[i][j] * xv[j]);
        }
    }
#pragma unroll
    for (int i = L - 1; i >= 0; i--) {
        const bool on = i < at.nv;
        float d[CV];
        rd.at(i, d);
#pragma unroll
        for (int j = 0; j < CV; j++) {
            const float l = d[j] + m[j];
            m[j] = on ? ga[i][j] * l : m[j];
            away[i][j] = on ? gc[i][j] * m[j] * away[i][j] : 0.f;
            gc[i][j] = on ? gc[i][j] * l : 0.f;
        }
    }
    put<K>(dx, a.dxs, a.T, at, gc);
    put<K>(dg, a.dgs, a.T, at, away);
}

// ------------------------------------------------------------------- a few steps
// Records that are extended by a step or a few: no exchange between lanes, a
// lane takes VE channels of one record through all steps.  One step of
// 1024 x 512 bf16: 4.5 us.
//
// Up to eight steps always (B = 1: 11 us of a call, as the other kernels take);
// up to 32, backwards 16, if there are many channels, since most wavefronts of a
// segment would be empty: 1024 x 9 x 512 bf16 15 us against 51, backwards 26 against
// 45; 1024 x 32 x 512 38 against 51.  With 64 x 512 channels 32 steps take 31 us
// against 14.
bool few_steps(int64_t B, int64_t T, int64_t D, bool back)
{
    return T <= 8 || (T <= (back ? 16 : 32) && B * D >= 1 << 19);
}
// G steps are read at a time.
template <class T, int G> __global__ __launch_bounds__(256) void k_scan_few(ScanArgs a, int64_t chunks)
{
    constexpr int VE = kVec<T>;
    const int64_t i = (int64_t)block_of() * 256 + threadIdx.x;
    if (i >= a.B * chunks) return;
    const int64_t b = i / chunks, c = i % chunks * VE;
    const int n = (int)min((int64_t)VE, a.D - c);
    int64_t len = a.T;
    if (a.lengths) len = min(max((int64_t)a.lengths[b], (int64_t)0), a.T);
    const T *x = (const T *)a.x + b * a.xb + c, *g = (const T *)a.g + b * a.gb + c;
    T *y = (T *)a.y + b * a.yb + c;
    float h[VE] = {};
    if (a.h0) load_part<VE>(a.h0 + b * a.D + c, n, h);
    if (a.states && len) store_part<VE>(a.states + b * a.D + c, n, h);
    for (int64_t t0 = 0; t0 < a.T; t0 += G) {
        float xv[G][VE] = {}, gv[G][VE] = {};
        if (t0 < len)
#pragma unroll
            for (int i = 0; i < G; i++) {
                const int64_t t = min(t0 + i, len - 1);
                load_part<VE>(x + t * a.xs, n, xv[i]);
                load_part<VE>(g + t * a.gs, n, gv[i]);
            }
#pragma unroll
        for (int i = 0; i < G; i++) {
            const int64_t t = t0 + i;
            if (t >= a.T) break;
            float o[VE] = {};
            if (t < len)
#pragma unroll
                for (int j = 0; j < VE; j++) {
                    float av, cv;
                    gate<T>(gv[i][j], av, cv);
                    o[j] = h[j] = fmaf(av, h[j], cv * xv[i][j]);
                }
            store_part<VE>(y + t * a.ys, n, o);
        }
    }
    if (a.h_last) store_part<VE>(a.h_last + b * a.D + c, n, h);
}

// The gradients of a few steps: the lane keeps the states it passes forwards.
template <class T, int STEPS, int VE>
__global__ __launch_bounds__(256) void k_scan_grad_few(ScanArgs a, int64_t chunks)
{
    const int64_t i = (int64_t)block_of() * 256 + threadIdx.x;
    if (i >= a.B * chunks) return;
    const int64_t b = i / chunks, c = i % chunks * VE;
    const int n = (int)min((int64_t)VE, a.D - c);
    int64_t len = a.T;
    if (a.lengths) len = min(max((int64_t)a.lengths[b], (int64_t)0), a.T);
    const T *x = (const T *)a.x + b * a.xb + c, *g = (const T *)a.g + b * a.gb + c, *dy = (const T *)a.dy + b * a.dyb + c;
    T *dx = (T *)a.dx + b * a.dxb + c, *dg = (T *)a.dg + b * a.dgb + c;
    float m[VE] = {}, h[STEPS][VE], ga[STEPS][VE], gc[STEPS][VE], xv[STEPS][VE];
    if (a.dh_last) load_part<VE>(a.dh_last + b * a.D + c, n, m);
    float s[VE] = {};
    if (len) load_part<VE>(a.states_in + b * a.D + c, n, s);
#pragma unroll
    for (int t = 0; t < STEPS; t++) {
        if (t >= len) break;
        float gv[VE];
        load_part<VE>(x + t * a.xs, n, xv[t]);
        load_part<VE>(g + t * a.gs, n, gv);
#pragma unroll
        for (int j = 0; j < VE; j++) {
            gate<T>(gv[j], ga[t][j], gc[t][j]);
            h[t][j] = s[j];
            s[j] = fmaf(ga[t][j], s[j], gc[t][j] * xv[t][j]);
        }
    }
#pragma unroll
    for (int t = STEPS - 1; t >= 0; t--) {
        if (t >= a.T) continue;
        float ox[VE] = {}, og[VE] = {};
        if (t < len) {
            float d[VE];
            load_part<VE>(dy + t * a.dys, n, d);
#pragma unroll
            for (int j = 0; j < VE; j++) {
                const float l = d[j] + m[j];
                m[j] = ga[t][j] * l;
                ox[j] = gc[t][j] * l;
                og[j] = gc[t][j] * m[j] * (h[t][j] - xv[t][j]);
            }
        }
        store_part<VE>(dx + t * a.dxs, n, ox);
        store_part<VE>(dg + t * a.dgs, n, og);
    }
    if (a.dh0) store_part<VE>(a.dh0 + b * a.D + c, n, m);
}

// ------------------------------------------------------------------ launches
// Rows (records x slabs) and segments of a scan of kind K.
template <class K> struct Layout {
    int64_t rows, items;
    int slabs, segs;
    size_t ticket, slots, bytes;
    Layout(int64_t B, int64_t T, int64_t D)
    {
        slabs = (int)((D + K::slab - 1) / K::slab);
        rows = B * slabs;
        segs = (int)std::max<int64_t>(1, (T + K::seg - 1) / K::seg);
        items = rows * segs;
        Carver c;
        ticket = c.take(segs > 1 ? sizeof(unsigned) : 0);
        slots = c.take(segs > 1 ? sizeof(Slot) * items * K::slab : 0);
        bytes = c.used;
    }
    // workspace and the call's first kernel
    Geom start(void *ws, hipStream_t s) const
    {
        Geom g{};
        g.rows = (uint32_t)rows, g.slabs = (uint32_t)slabs, g.segs = segs;
        if (segs == 1) return g;
        g.slots = (Slot *)((char *)ws + slots);
        g.ticket = (unsigned *)((char *)ws + ticket);
        const int64_t n = items * K::slab;
        k_scan_clear<<<grid_of((n + 511) / 512), 256, 0, s>>>(g.slots, n, g.ticket);
        return g;
    }
};

// Calls f with the kind of a scan.
template <class T, bool BACK, class F> auto by_kind(int64_t D, F &&f)
{
    if constexpr (sizeof(T) == 2)
        if (D > 64) return f(Kind<T, 2, BACK ? 8 : 16>{});
    return f(Kind<T, 1, 16>{});
}

template <class T> hipError_t scan_t(const ScanArgs &a, hipStream_t s)
{
    if (few_steps(a.B, a.T, a.D, false)) {
        const int64_t chunks = (a.D + kVec<T> - 1) / kVec<T>;
        const dim3 blocks = grid_of((a.B * chunks + 255) / 256);
        if (a.T == 1) k_scan_few<T, 1><<<blocks, 256, 0, s>>>(a, chunks);
        else k_scan_few<T, 4><<<blocks, 256, 0, s>>>(a, chunks);
        return hipGetLastError();
    }
    return by_kind<T, false>(a.D, [&](auto kind) {
        using K = decltype(kind);
        const Layout<K> l(a.B, a.T, a.D);
        Geom g = l.start(a.ws, s);
        launch_exactly(l.items, [&](dim3 grid, uint32_t first) {
            g.first = first;
            k_scan<K><<<grid, kThreads, 0, s>>>(a, g);
        });
        return hipGetLastError();
    });
}

template <class T> hipError_t scan_grad_t(const ScanArgs &a, hipStream_t s)
{
    if (few_steps(a.B, a.T, a.D, true)) {
        auto go = [&](auto kernel, int ve) {
            const int64_t chunks = (a.D + ve - 1) / ve;
            kernel<<<grid_of((a.B * chunks + 255) / 256), 256, 0, s>>>(a, chunks);
        };
        if (a.T <= 8) go(k_scan_grad_few<T, 8, 4>, 4);
        else go(k_scan_grad_few<T, 16, 2>, 2);
        return hipGetLastError();
    }
    return by_kind<T, true>(a.D, [&](auto kind) {
        using K = decltype(kind);
        const Layout<K> l(a.B, a.T, a.D);
        Geom g = l.start(a.ws, s);
        launch_exactly(l.items, [&](dim3 grid, uint32_t first) {
            g.first = first;
            k_scan_grad<K><<<grid, kThreads, 0, s>>>(a, g);
        });
        return hipGetLastError();
    });
}

// The largest of what the directions and types take.
template <class F> auto largest(int64_t D, F &&f)
{
    return std::max({by_kind<float, false>(D, f), by_kind<__bf16, false>(D, f), by_kind<float, true>(D, f),
                     by_kind<__bf16, true>(D, f)});
}

} // namespace

int64_t scan_items(int64_t B, int64_t T, int64_t D)
{
    return largest(D, [&](auto kind) { return Layout<decltype(kind)>(B, T, D).items; });
}

size_t scan_workspace(int64_t B, int64_t T, int64_t D)
{
    return largest(D, [&](auto kind) { return Layout<decltype(kind)>(B, T, D).bytes; });
}

hipError_t launch_scan(int32_t type, const ScanArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return scan_t<float>(a, s);
    if (type == TQ_BF16) return scan_t<__bf16>(a, s);
    return scan_t<_Float16>(a, s);
}

hipError_t launch_scan_grad(int32_t type, const ScanArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return scan_grad_t<float>(a, s);
    if (type == TQ_BF16) return scan_grad_t<__bf16>(a, s);
    return scan_grad_t<_Float16>(a, s);
}

} // namespace tq
