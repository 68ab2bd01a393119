// seq_scan.hip -- the gated linear recurrence over time and its gradients.
//
//   h_t = a_t h_{t-1} + c_t x_t,   a_t = sigmoid(g_t), c_t = 1 - a_t.
//
// Each step is the map h -> a h + b; maps compose to (A, B) pairs, so a stretch
// of time is summed up by one pair per channel.  A workgroup takes one record,
// 64 lanes' worth of channels and kPiece steps at a time: its wavefronts read
// kSteps steps each into registers, exchange their pairs through LDS, and then
// apply their steps to the state they start from, so x and g are read once and y
// is written once.  The state of the piece's end is carried to the next piece.
// The backward pass walks the pieces from the last one back: the pairs
// forwards give h_{t-1} (from the saved state before the piece), and
//   l_t = dy_t + m_{t+1},  m_t = a_t l_t
// is the same kind of recurrence backwards.
//
// With few records and channels the time axis is cut into segments of whole
// pieces: a first kernel sums each segment up to its pair, a second joins the
// pairs, and the segments then run side by side.
#include <algorithm>

#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

constexpr int kWaves = 8, kSteps = 8, kPiece = kWaves * kSteps;
constexpr int kThreads = 64 * kWaves;
static_assert(kPiece == TQ_SCAN_PIECE, "states are kept per piece");

// exp(-v), v >= 0.  The product with log2 e is rounded, an error of up to
// v 2^-24 relative; for fp32 inputs what the rounding lost is put back.
template <class T> __device__ __forceinline__ float exp_neg(float v)
{
    constexpr float kLog2e = 1.44269504088896341f;
    if constexpr (sizeof(T) == 4) v = fminf(v, 1e4f);  // infinities have no remainder
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
    if (g != g) a = c = g;
}

// What a workgroup works on.
struct Place {
    int64_t b, len;
    int seg;
    int64_t c0;  // the lane's first channel
    int n;       // its channels
};

template <int CV> __device__ __forceinline__ Place place_of(const ScanArgs &a, int slabs, int segs)
{
    Place p;
    const int64_t blk = blockIdx.x;
    p.seg = (int)(blk / slabs % segs);
    p.b = blk / slabs / segs;
    p.c0 = ((blk % slabs) * 64 + (threadIdx.x & 63)) * CV;
    p.n = (int)max((int64_t)0, min((int64_t)CV, a.D - p.c0));
    if (p.n == 0) p.c0 = 0;
    p.len = a.T;
    if (a.lengths) p.len = min(max((int64_t)a.lengths[p.b], (int64_t)0), a.T);
    return p;
}

// The raw elements of one wavefront's steps; steps past `nv` are not read.
template <class T, int CV> struct Raw {
    T v[kSteps][CV];
    __device__ __forceinline__ void load(const T *p, int64_t step, int nv, int n)
    {
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            if (i >= nv) continue;
            if (n == CV) __builtin_memcpy(v[i], p + i * step, sizeof v[i]);
            else
#pragma unroll
                for (int j = 0; j < CV; j++)
                    if (j < n) v[i][j] = p[i * step + j];
        }
    }
};

// ------------------------------------------------------------------ forward
// start: the states the segments start from ([B, segs, D]), or h0 with one
// segment.  PAIRS: only the segments' pairs are wanted, [B, segs, D] (A, B).
template <class T, int CV, bool PAIRS>
__global__ __launch_bounds__(kThreads) void k_scan(ScanArgs a, int slabs, int segs, int seg_pieces,
                                                  const float *start, float2 *pairs)
{
    __shared__ float2 agg[2][kWaves][64 * CV];
    const Place p = place_of<CV>(a, slabs, segs);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T *x = (const T *)a.x + p.b * a.xb + p.c0, *g = (const T *)a.g + p.b * a.gb + p.c0;
    T *y = (T *)a.y + p.b * a.yb + p.c0;
    const int64_t pieces = (a.T + kPiece - 1) / kPiece;
    const int64_t j0 = (int64_t)p.seg * seg_pieces, j1 = min(j0 + seg_pieces, pieces);
    const int64_t last = min(j1, (p.len + kPiece - 1) / kPiece);  // pieces with steps of the record
    float h[CV], whole[CV];
#pragma unroll
    for (int j = 0; j < CV; j++) {
        h[j] = !PAIRS && start && j < p.n ? start[(p.b * segs + p.seg) * a.D + p.c0 + j] : 0.f;
        whole[j] = 1.f;
    }
    Raw<T, CV> rx, rg;
    auto fetch = [&](int64_t piece) {
        const int64_t t = piece * kPiece + wave * kSteps;
        const int nv = (int)max((int64_t)0, min((int64_t)kSteps, p.len - t));
        rx.load(x + t * a.xs, a.xs, nv, p.n);
        rg.load(g + t * a.gs, a.gs, nv, p.n);
    };
    if (j0 < last) fetch(j0);
    int turn = 0;
    for (int64_t piece = j0; piece < last; piece++, turn ^= 1) {
        const int64_t t = piece * kPiece + wave * kSteps;
        const int nv = (int)max((int64_t)0, min((int64_t)kSteps, p.len - t));
        float ga[kSteps][CV], gb[kSteps][CV], A[CV], Bv[CV];
#pragma unroll
        for (int j = 0; j < CV; j++) A[j] = 1.f, Bv[j] = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; i++)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                float av = 1.f, bv = 0.f;
                if (i < nv && j < p.n) {
                    float c;
                    gate<T>((float)rg.v[i][j], av, c);
                    bv = c * (float)rx.v[i][j];
                }
                ga[i][j] = av;
                gb[i][j] = bv;
                Bv[j] = fmaf(av, Bv[j], bv);
                A[j] *= av;
            }
#pragma unroll
        for (int j = 0; j < CV; j++) agg[turn][wave][lane * CV + j] = make_float2(A[j], Bv[j]);
        if (piece + 1 < last) fetch(piece + 1);
        __syncthreads();
        if (!PAIRS && a.states && wave == 0)
#pragma unroll
            for (int j = 0; j < CV; j++)
                if (j < p.n) a.states[(p.b * pieces + piece) * a.D + p.c0 + j] = h[j];
        float mine[CV];
#pragma unroll
        for (int j = 0; j < CV; j++) mine[j] = h[j];
#pragma unroll
        for (int w = 0; w < kWaves; w++)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                if (!PAIRS && w == wave) mine[j] = h[j];
                const float2 m = agg[turn][w][lane * CV + j];
                h[j] = fmaf(m.x, h[j], m.y);
                whole[j] *= m.x;
            }
        if (PAIRS) continue;
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            float o[CV];
#pragma unroll
            for (int j = 0; j < CV; j++) {
                mine[j] = fmaf(ga[i][j], mine[j], gb[i][j]);
                o[j] = i < nv ? mine[j] : 0.f;
            }
            if (t + i < a.T) store_part<CV>(y + (t + i) * a.ys, p.n, o);
        }
    }
    if (PAIRS) {
        if (wave == 0)
#pragma unroll
            for (int j = 0; j < CV; j++)
                if (j < p.n) pairs[(p.b * segs + p.seg) * a.D + p.c0 + j] = make_float2(whole[j], h[j]);
        return;
    }
    if (a.h_last && wave == 0 && p.seg == segs - 1)
#pragma unroll
        for (int j = 0; j < CV; j++)
            if (j < p.n) a.h_last[p.b * a.D + p.c0 + j] = h[j];
    // pieces past the record's end
    const float zero[CV] = {};
    for (int64_t piece = max(last, j0); piece < j1; piece++) {
        if (a.states && wave == 0)
#pragma unroll
            for (int j = 0; j < CV; j++)
                if (j < p.n) a.states[(p.b * pieces + piece) * a.D + p.c0 + j] = h[j];
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const int64_t t = piece * kPiece + wave * kSteps + i;
            if (t < a.T) store_part<CV>(y + t * a.ys, p.n, zero);
        }
    }
}

// ----------------------------------------------------------------- backward
// end: what the segments' last steps receive from the steps after them
// ([B, segs, D]), or dh_last with one segment.
template <class T, int CV>
__global__ __launch_bounds__(kThreads) void k_scan_grad(ScanArgs a, int slabs, int segs, int seg_pieces,
                                                       const float *end)
{
    __shared__ float2 fwd[2][kWaves][64 * CV];
    __shared__ float rev[2][kWaves][64 * CV];
    const Place p = place_of<CV>(a, slabs, segs);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T *x = (const T *)a.x + p.b * a.xb + p.c0, *g = (const T *)a.g + p.b * a.gb + p.c0;
    const T *dy = (const T *)a.dy + p.b * a.dyb + p.c0;
    T *dx = (T *)a.dx + p.b * a.dxb + p.c0, *dg = (T *)a.dg + p.b * a.dgb + p.c0;
    const int64_t pieces = (a.T + kPiece - 1) / kPiece;
    const int64_t j0 = (int64_t)p.seg * seg_pieces, j1 = min(j0 + seg_pieces, pieces);
    const int64_t last = min(j1, (p.len + kPiece - 1) / kPiece);
    float m[CV];
#pragma unroll
    for (int j = 0; j < CV; j++) m[j] = end && j < p.n ? end[(p.b * segs + p.seg) * a.D + p.c0 + j] : 0.f;
    Raw<T, CV> rx, rg, rd;
    float h_next[CV];  // the state before the piece that is fetched
    auto fetch = [&](int64_t piece) {
        const int64_t t = piece * kPiece + wave * kSteps;
        const int nv = (int)max((int64_t)0, min((int64_t)kSteps, p.len - t));
        rx.load(x + t * a.xs, a.xs, nv, p.n);
        rg.load(g + t * a.gs, a.gs, nv, p.n);
        rd.load(dy + t * a.dys, a.dys, nv, p.n);
#pragma unroll
        for (int j = 0; j < CV; j++)
            h_next[j] = j < p.n ? a.states_in[(p.b * pieces + piece) * a.D + p.c0 + j] : 0.f;
    };
    if (j0 < last) fetch(last - 1);
    int turn = 0;
    for (int64_t piece = last - 1; piece >= j0; piece--, turn ^= 1) {
        const int64_t t = piece * kPiece + wave * kSteps;
        const int nv = (int)max((int64_t)0, min((int64_t)kSteps, p.len - t));
        float ga[kSteps][CV], gc[kSteps][CV], xv[kSteps][CV], dv[kSteps][CV], A[CV], Bf[CV], Br[CV], h[CV];
#pragma unroll
        for (int j = 0; j < CV; j++) A[j] = 1.f, Bf[j] = Br[j] = 0.f, h[j] = h_next[j];
#pragma unroll
        for (int i = 0; i < kSteps; i++)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                float av = 1.f, cv = 0.f, xx = 0.f, d = 0.f;
                if (i < nv && j < p.n) {
                    gate<T>((float)rg.v[i][j], av, cv);
                    xx = (float)rx.v[i][j];
                    d = (float)rd.v[i][j];
                }
                ga[i][j] = av;
                gc[i][j] = cv;
                xv[i][j] = xx;
                dv[i][j] = d;
                Bf[j] = fmaf(av, Bf[j], cv * xx);
                A[j] *= av;
            }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; i--)
#pragma unroll
            for (int j = 0; j < CV; j++) Br[j] = ga[i][j] * (Br[j] + dv[i][j]);
#pragma unroll
        for (int j = 0; j < CV; j++) {
            fwd[turn][wave][lane * CV + j] = make_float2(A[j], Bf[j]);
            rev[turn][wave][lane * CV + j] = Br[j];
        }
        if (piece > j0) fetch(piece - 1);
        __syncthreads();
        float mine[CV];
#pragma unroll
        for (int j = 0; j < CV; j++) mine[j] = m[j];
#pragma unroll
        for (int w = kWaves - 1; w >= 0; w--)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                if (w == wave) mine[j] = m[j];
                m[j] = fmaf(fwd[turn][w][lane * CV + j].x, m[j], rev[turn][w][lane * CV + j]);
            }
        for (int w = 0; w < wave; w++)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                const float2 f = fwd[turn][w][lane * CV + j];
                h[j] = fmaf(f.x, h[j], f.y);
            }
        // forwards: x becomes h_{t-1} - x
#pragma unroll
        for (int i = 0; i < kSteps; i++)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                const float b = gc[i][j] * xv[i][j];
                xv[i][j] = h[j] - xv[i][j];
                h[j] = fmaf(ga[i][j], h[j], b);
            }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; i--) {
            float ox[CV], og[CV];
#pragma unroll
            for (int j = 0; j < CV; j++) {
                const float l = dv[i][j] + mine[j];
                mine[j] = ga[i][j] * l;
                ox[j] = i < nv ? gc[i][j] * l : 0.f;
                og[j] = i < nv ? gc[i][j] * mine[j] * xv[i][j] : 0.f;
            }
            if (t + i < a.T) {
                store_part<CV>(dx + (t + i) * a.dxs, p.n, ox);
                store_part<CV>(dg + (t + i) * a.dgs, p.n, og);
            }
        }
    }
    if (a.dh0 && wave == 0 && p.seg == 0)
#pragma unroll
        for (int j = 0; j < CV; j++)
            if (j < p.n) a.dh0[p.b * a.D + p.c0 + j] = m[j];
    const float zero[CV] = {};
    for (int64_t piece = max(last, j0); piece < j1; piece++)
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const int64_t t = piece * kPiece + wave * kSteps + i;
            if (t < a.T) {
                store_part<CV>(dx + t * a.dxs, p.n, zero);
                store_part<CV>(dg + t * a.dgs, p.n, zero);
            }
        }
}

// The segments' pairs backwards: (A, B) with B what a segment hands to the one
// before it when it receives nothing.
template <class T, int CV>
__global__ __launch_bounds__(kThreads) void k_scan_grad_pairs(ScanArgs a, int slabs, int segs, int seg_pieces,
                                                             float2 *pairs)
{
    __shared__ float2 agg[2][kWaves][64 * CV];
    const Place p = place_of<CV>(a, slabs, segs);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T *g = (const T *)a.g + p.b * a.gb + p.c0, *dy = (const T *)a.dy + p.b * a.dyb + p.c0;
    const int64_t pieces = (a.T + kPiece - 1) / kPiece;
    const int64_t j0 = (int64_t)p.seg * seg_pieces, j1 = min(j0 + seg_pieces, pieces);
    const int64_t last = min(j1, (p.len + kPiece - 1) / kPiece);
    float m[CV], whole[CV];
#pragma unroll
    for (int j = 0; j < CV; j++) m[j] = 0.f, whole[j] = 1.f;
    Raw<T, CV> rg, rd;
    auto fetch = [&](int64_t piece) {
        const int64_t t = piece * kPiece + wave * kSteps;
        const int nv = (int)max((int64_t)0, min((int64_t)kSteps, p.len - t));
        rg.load(g + t * a.gs, a.gs, nv, p.n);
        rd.load(dy + t * a.dys, a.dys, nv, p.n);
    };
    if (j0 < last) fetch(last - 1);
    int turn = 0;
    for (int64_t piece = last - 1; piece >= j0; piece--, turn ^= 1) {
        const int64_t t = piece * kPiece + wave * kSteps;
        const int nv = (int)max((int64_t)0, min((int64_t)kSteps, p.len - t));
        float A[CV], B[CV];
#pragma unroll
        for (int j = 0; j < CV; j++) A[j] = 1.f, B[j] = 0.f;
#pragma unroll
        for (int i = kSteps - 1; i >= 0; i--)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                float av = 1.f, cv, d = 0.f;
                if (i < nv && j < p.n) {
                    gate<T>((float)rg.v[i][j], av, cv);
                    d = (float)rd.v[i][j];
                }
                A[j] *= av;
                B[j] = av * (B[j] + d);
            }
#pragma unroll
        for (int j = 0; j < CV; j++) agg[turn][wave][lane * CV + j] = make_float2(A[j], B[j]);
        if (piece > j0) fetch(piece - 1);
        __syncthreads();
#pragma unroll
        for (int w = kWaves - 1; w >= 0; w--)
#pragma unroll
            for (int j = 0; j < CV; j++) {
                const float2 q = agg[turn][w][lane * CV + j];
                m[j] = fmaf(q.x, m[j], q.y);
                whole[j] *= q.x;
            }
    }
    if (wave == 0)
#pragma unroll
        for (int j = 0; j < CV; j++)
            if (j < p.n) pairs[(p.b * segs + p.seg) * a.D + p.c0 + j] = make_float2(whole[j], m[j]);
}

// What each segment starts from: state[b, s] from the pairs of the segments
// before s (BACK: after s) and first[b] (NULL: zeros).  The workgroup's
// wavefronts take consecutive parts of the segments.
constexpr int kJoinWaves = 16;
template <bool BACK>
__global__ __launch_bounds__(64 * kJoinWaves) void k_scan_join(const float2 *pairs, const float *first, float *state,
                                                              int64_t D, int segs)
{
    __shared__ float2 agg[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t slabs = (D + 63) / 64, b = blockIdx.x / slabs, c = blockIdx.x % slabs * 64 + lane;
    const bool in = c < D;
    const int per = (segs + kJoinWaves - 1) / kJoinWaves;
    const int s0 = min(wave * per, segs), s1 = min(s0 + per, segs);
    auto at = [&](int s) { return (b * segs + (BACK ? segs - 1 - s : s)) * D + c; };
    float2 q = make_float2(1.f, 0.f);
    if (in)
#pragma unroll 8
        for (int s = s0; s < s1; s++) {
            const float2 v = pairs[at(s)];
            q.y = fmaf(v.x, q.y, v.y);
            q.x *= v.x;
        }
    agg[wave][lane] = q;
    __syncthreads();
    if (!in) return;
    float h = first ? first[b * D + c] : 0.f;
    for (int w = 0; w < wave; w++) h = fmaf(agg[w][lane].x, h, agg[w][lane].y);
#pragma unroll 8
    for (int s = s0; s < s1; s++) {
        const float2 v = pairs[at(s)];
        state[at(s)] = h;
        h = fmaf(v.x, h, v.y);
    }
}

// ------------------------------------------------------------------- a few steps
// Records that are extended by a step or a few: no exchange between lanes, a
// lane takes VE channels of one record through all steps.
constexpr int kFew = 8;
template <class T> __global__ __launch_bounds__(256) void k_scan_few(ScanArgs a, int64_t chunks)
{
    constexpr int VE = kVec<T>;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.B * chunks) return;
    const int64_t b = i / chunks, c = i % chunks * VE;
    const int n = (int)min((int64_t)VE, a.D - c);
    int64_t len = a.T;
    if (a.lengths) len = min(max((int64_t)a.lengths[b], (int64_t)0), a.T);
    const T *x = (const T *)a.x + b * a.xb + c, *g = (const T *)a.g + b * a.gb + c;
    T *y = (T *)a.y + b * a.yb + c;
    float h[VE] = {};
    if (a.h0) load_part<VE>(a.h0 + b * a.D + c, n, h);
    if (a.states && a.T) store_part<VE>(a.states + b * a.D + c, n, h);
    for (int64_t t = 0; t < a.T; t++) {
        float o[VE] = {};
        if (t < len) {
            float xv[VE], gv[VE];
            load_part<VE>(x + t * a.xs, n, xv);
            load_part<VE>(g + t * a.gs, n, gv);
#pragma unroll
            for (int j = 0; j < VE; j++) {
                float av, cv;
                gate<T>(gv[j], av, cv);
                o[j] = h[j] = fmaf(av, h[j], cv * xv[j]);
            }
        }
        store_part<VE>(y + t * a.ys, n, o);
    }
    if (a.h_last) store_part<VE>(a.h_last + b * a.D + c, n, h);
}

// How a scan is cut: channels per lane, and segments of the time axis.
struct Cut {
    int cv, segs, seg_pieces;
    int64_t slabs, pieces;
    Cut(int64_t B, int64_t T, int64_t D)
    {
        pieces = (T + kPiece - 1) / kPiece;
        const int64_t want = 1024;  // workgroups that fill the chip
        cv = B * ((D + 127) / 128) >= want / 2 ? 2 : 1;
        slabs = (D + 64 * cv - 1) / (64 * cv);
        const int64_t rows = std::max<int64_t>(1, B * slabs);
        int64_t s = rows >= want / 2 ? 1 : std::min(want / rows, (pieces + 1) / 2);
        s = std::max<int64_t>(s, 1);
        seg_pieces = (int)std::max<int64_t>(1, (pieces + s - 1) / s);
        segs = (int)std::max<int64_t>(1, (pieces + seg_pieces - 1) / seg_pieces);
    }
};

struct ScanSpace {
    size_t pairs, state, bytes;
    ScanSpace(const Cut &c, int64_t B, int64_t D)
    {
        Carver k;
        const size_t n = c.segs > 1 ? (size_t)B * c.segs * D : 0;
        pairs = k.take(sizeof(float2) * n);
        state = k.take(sizeof(float) * n);
        bytes = k.used;
    }
};

template <class T, int CV> hipError_t scan_cv(const ScanArgs &a, const Cut &c, hipStream_t s)
{
    const ScanSpace w(c, a.B, a.D);
    float2 *pairs = (float2 *)((char *)a.ws + w.pairs);
    float *state = (float *)((char *)a.ws + w.state);
    const unsigned grid = (unsigned)(a.B * c.slabs * c.segs);
    const float *start = a.h0;
    if (c.segs > 1) {
        k_scan<T, CV, true><<<grid, kThreads, 0, s>>>(a, (int)c.slabs, c.segs, c.seg_pieces, nullptr, pairs);
        k_scan_join<false><<<(unsigned)(a.B * ((a.D + 63) / 64)), 64 * kJoinWaves, 0, s>>>(pairs, a.h0, state, a.D,
                                                                                        c.segs);
        start = state;
    }
    k_scan<T, CV, false><<<grid, kThreads, 0, s>>>(a, (int)c.slabs, c.segs, c.seg_pieces, start, nullptr);
    return hipGetLastError();
}

template <class T> hipError_t scan_t(const ScanArgs &a, hipStream_t s)
{
    if (a.T <= kFew) {
        const int64_t chunks = (a.D + kVec<T> - 1) / kVec<T>;
        k_scan_few<T><<<(unsigned)((a.B * chunks + 255) / 256), 256, 0, s>>>(a, chunks);
        return hipGetLastError();
    }
    const Cut c(a.B, a.T, a.D);
    return c.cv == 2 ? scan_cv<T, 2>(a, c, s) : scan_cv<T, 1>(a, c, s);
}

template <class T, int CV> hipError_t scan_grad_cv(const ScanArgs &a, const Cut &c, hipStream_t s)
{
    const ScanSpace w(c, a.B, a.D);
    float2 *pairs = (float2 *)((char *)a.ws + w.pairs);
    float *state = (float *)((char *)a.ws + w.state);
    const unsigned grid = (unsigned)(a.B * c.slabs * c.segs);
    const float *end = a.dh_last;
    if (c.segs > 1) {
        k_scan_grad_pairs<T, CV><<<grid, kThreads, 0, s>>>(a, (int)c.slabs, c.segs, c.seg_pieces, pairs);
        k_scan_join<true><<<(unsigned)(a.B * ((a.D + 63) / 64)), 64 * kJoinWaves, 0, s>>>(pairs, a.dh_last, state, a.D,
                                                                                       c.segs);
        end = state;
    }
    k_scan_grad<T, CV><<<grid, kThreads, 0, s>>>(a, (int)c.slabs, c.segs, c.seg_pieces, end);
    return hipGetLastError();
}

template <class T> hipError_t scan_grad_t(const ScanArgs &a, hipStream_t s)
{
    const Cut c(a.B, a.T, a.D);
    return c.cv == 2 ? scan_grad_cv<T, 2>(a, c, s) : scan_grad_cv<T, 1>(a, c, s);
}

} // namespace

size_t scan_workspace(int64_t B, int64_t T, int64_t D) { return ScanSpace(Cut(B, T, D), B, D).bytes; }

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
