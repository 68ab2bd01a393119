// model_beam.hip -- one step of a beam search: the best continuations of all beams
// of a record, and the states that go with them.
//
// A beam's candidates score scores[w] + z_v - lse, lse = log sum_u exp z_u.  Which
// candidates of different beams are the best hangs on the last digits of lse, so the
// exponentials and their sum are formed in 64 bits: what is chosen does not depend
// on the order of a sum.  Reading the logits and these exponentials, some twenty
// instructions each, take about the same time.
//
// A wavefront holds a segment of a beam's logits in registers, 64 lanes of 16
// pieces.  With the segment's maximum it forms the sum; the K-th largest of the
// lanes' maxima is a bound that K elements reach, found bit by bit by ballots, so
// that few elements are looked at again to be entered in the list of the K best,
// which the lanes hold in order, one each.  Lists are of keys that no two elements
// share: a value's bits in the order of values, then the id, lower ids first.
// A second kernel joins a beam's segments and then the beams: a candidate's place is
// the number of candidates before it, counted by binary search in every beam's list.
// Where a beam is one segment, one kernel does both.
//
// Reordering the states is a copy of rows of any number of tensors in one launch.
#include <algorithm>

#include "model.h"
#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

using Key = unsigned long long;
constexpr int kPieces = 16;  // of 16 bytes, a lane's part of a segment
template <class T> constexpr int kSegment = 64 * kPieces * kVec<T>;
constexpr double kNone = -__builtin_inf();

struct Geom {
    uint32_t rows;       // R W
    uint32_t segments;   // of a beam
    int64_t length;      // of a segment
    float *tops;         // [rows][segments]
    double *sums;
    Key *keys;           // [rows][segments][K]
};

// The bits of a float in the order of floats; -0 is 0.
__device__ __forceinline__ uint32_t ordered(float f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(Key k)
{
    const uint32_t u = (uint32_t)(k >> 32);
    return __builtin_bit_cast(float, u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint32_t id_of(Key k) { return ~(uint32_t)k; }

// exp(x) for x <= 0 to about 2^-50: x = n ln 2 + r, the series of e^r to r^12.
// Below -690 the result is that at -690, which no sum of ids shows.
__device__ __forceinline__ double exp_below(double x)
{
    x = x < -690. ? -690. : x;
    const double magic = 0x1.8p52, t = fma(x, 1.4426950408889634, magic), n = t - magic;
    double r = fma(n, -0x1.62e42fefa39efp-1, x);
    r = fma(n, -0x1.abc9e3b39803fp-56, r);
    double p = 1. / 479001600.;
    p = fma(p, r, 1. / 39916800.);
    p = fma(p, r, 1. / 3628800.);
    p = fma(p, r, 1. / 362880.);
    p = fma(p, r, 1. / 40320.);
    p = fma(p, r, 1. / 5040.);
    p = fma(p, r, 1. / 720.);
    p = fma(p, r, 1. / 120.);
    p = fma(p, r, 1. / 24.);
    p = fma(p, r, 1. / 6.);
    p = fma(p, r, .5);
    p = fma(p, r, 1.);
    p = fma(p, r, 1.);
    const uint64_t b = __builtin_bit_cast(uint64_t, p);
    const uint32_t hi = (uint32_t)(b >> 32) + (__builtin_bit_cast(uint64_t, t) << 20);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)b);
}

template <class V> __device__ __forceinline__ V wave_sum(V v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ __forceinline__ Key lane_key(Key k, int lane)
{
    return (Key)__builtin_amdgcn_readlane((uint32_t)(k >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((uint32_t)k, lane);
}

// A wavefront's list of the K best keys, lane i the i-th; zeros where there are fewer.
struct Best {
    Key mine = 0, least = 0;  // the K-th
    int K;
    __device__ explicit Best(int k) : K(k) {}
    __device__ __forceinline__ void enter(Key k)
    {
        const int lane = threadIdx.x & 63, at = __popcll(__ballot(mine > k));
        const Key left = __shfl_up(mine, 1, 64);
        mine = lane < at || lane >= K ? mine : lane == at ? k : left;
        least = lane_key(mine, K - 1);
    }
    // the keys of all lanes that are better than the least so far
    __device__ __forceinline__ void offer(Key k)
    {
        for (unsigned long long left = __ballot(k > least); left; left &= left - 1) {
            const Key one = lane_key(k, __builtin_ctzll(left));
            if (one > least) enter(one);
        }
    }
};

// Part [from, to) of a beam's logits: their maximum, the sum of their exponentials
// relative to it, and the K best.
template <class T> struct Segment {
    static constexpr int V = kVec<T>;
    float top;
    double sum;
    Key best;
    __device__ Segment(const T *row, int64_t from, int64_t to, int K)
    {
        const int lane = threadIdx.x & 63;
        const int n = (int)(to - from);
        T v[kPieces][V];
#pragma unroll
        for (int p = 0; p < kPieces; p++) {
            const int at = (p * 64 + lane) * V;
#pragma unroll
            for (int j = 0; j < V; j++) v[p][j] = (T)(float)kNone;
            if (at + V <= n) __builtin_memcpy(v[p], row + from + at, sizeof v[p]);
            else if (at < n)
#pragma unroll
                for (int j = 0; j < V; j++)
                    if (at + j < n) v[p][j] = row[from + at + j];
        }
        float mine = (float)kNone;
#pragma unroll
        for (int p = 0; p < kPieces; p++) {
#pragma unroll
            for (int j = 0; j < V; j++) mine = fmaxf(mine, (float)v[p][j]);
        }
        top = wave_max(mine);
        // of a segment of -infinity: nothing
        const double base = top == (float)kNone ? 0. : (double)top;
        sum = 0.;
#pragma unroll
        for (int p = 0; p < kPieces; p++) {
            if (p * 64 * V < n) {
                double s = 0.;
#pragma unroll
                for (int j = 0; j < V; j++) s += exp_below((double)(float)v[p][j] - base);
                sum += s;
            }
        }
        if (top == (float)kNone) sum = sum == sum ? 0. : sum;
        sum = wave_sum(sum);
        // a value that K of the lanes reach
        uint32_t bound = 0;
        const uint32_t high = lane * V < n ? ordered(mine) : 0;
#pragma unroll
        for (int bit = 31; bit >= 0; bit--) {
            const uint32_t more = bound | 1u << bit;
            if (__popcll(__ballot(high >= more)) >= K) bound = more;
        }
        Best list(K);
#pragma unroll
        for (int p = 0; p < kPieces; p++) {
            const int at = (p * 64 + lane) * V;
            if (p * 64 * V < n) {
#pragma unroll
                for (int j = 0; j < V; j++) {
                    const uint32_t o = ordered((float)v[p][j]);
                    const bool reaches = o >= bound && at + j < n;
                    if (__ballot(reaches)) {
                        list.offer(reaches ? (Key)o << 32 | (uint32_t)~(uint32_t)(from + at + j) : 0);
                        bound = max(bound, (uint32_t)(list.least >> 32));
                    }
                }
            }
        }
        best = list.mine;
    }
};

// A record's beams and their candidates in LDS, each beam's K in order.
struct Lists {
    double *score;   // [W][K]
    uint32_t *id;    // [W][K]
    int *count;      // [W]
    __device__ Lists(char *lds, int W, int K)
        : score((double *)lds), id((uint32_t *)(score + W * K)), count((int *)(id + W * K))
    {
    }
};

__device__ __forceinline__ bool over(const BeamArgs &a, int64_t row) { return a.last && a.last[row] == a.end; }

// A beam's list from its keys (one per lane), its maximum and its sum.
__device__ __forceinline__ void list_beam(const BeamArgs &a, const Lists &l, int w, int64_t row, Key key, float top,
                                          double sum)
{
    const int lane = threadIdx.x & 63, K = (int)a.K, n = (int)min((int64_t)K, a.V);
    const double score = a.scores[row];
    const bool ended = over(a, row), finite = fabs(score) < __builtin_inf();
    const double lse = ended ? 0. : (double)top + log(sum);
    double s = kNone;
    uint32_t id = (uint32_t)lane;
    if (finite && ended) {  // the end, then the others
        s = lane == 0 ? score : kNone;
        id = lane == 0 ? (uint32_t)a.end : (uint32_t)lane - ((uint32_t)lane <= (uint32_t)a.end);
    } else if (finite && fabs(lse) < __builtin_inf()) {
        s = score + ((double)value_of(key) - lse);
        if (!(s < __builtin_inf())) s = kNone;
        id = id_of(key);
    }
    if (lane < n) {
        l.score[w * K + lane] = s;
        l.id[w * K + lane] = id;
    }
    if (lane == 0) l.count[w] = n;
}

// The places of all candidates among each other.
__device__ __forceinline__ void pick(const BeamArgs &a, const Lists &l, int64_t r, int threads)
{
    const int W = (int)a.W, K = (int)a.K;
    for (int c = threadIdx.x; c < W * K; c += threads) {
        const int w = c / K, k = c - w * K;
        if (k >= l.count[w]) continue;
        const double s = l.score[c];
        int place = k;
        for (int o = 0; o < W && place < K; o++) {
            if (o == w) continue;
            // those of beam o that are before: better, or as good in a lower beam
            int lo = 0, hi = l.count[o];
            while (lo < hi) {
                const int m = (lo + hi) / 2;
                const double t = l.score[o * K + m];
                if (t > s || (t == s && o < w)) lo = m + 1;
                else hi = m;
            }
            place += lo;
        }
        if (place < K) {
            a.out_scores[r * K + place] = (float)s;
            a.parents[r * K + place] = w;
            a.tokens[r * K + place] = l.id[c];
        }
    }
}

constexpr int kRowThreads = 256;
template <class T> __global__ __launch_bounds__(kRowThreads) void k_beam_rows(BeamArgs a, Geom g)
{
    const uint32_t item = block_of() * (kRowThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= g.rows * g.segments) return;
    const int lane = threadIdx.x & 63;
    const uint32_t row = item / g.segments;
    if (over(a, row)) return;
    const int64_t from = (item - row * g.segments) * g.length;
    const Segment<T> s((const T *)a.logits + row * a.ld, from, min(from + g.length, a.V), (int)a.K);
    if (lane == 0) {
        g.tops[item] = s.top;
        g.sums[item] = s.sum;
    }
    if (lane < a.K) g.keys[(int64_t)item * a.K + lane] = s.best;
}

constexpr int kPickThreads = 256;
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(BeamArgs a, Geom g)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int64_t r = block_of();
    if (r >= a.R) return;
    const Lists l(lds, (int)a.W, (int)a.K);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int w = wave; w < a.W; w += kPickThreads / 64) {
        const int64_t row = r * a.W + w;
        float top = (float)kNone;
        double sum = 0.;
        Best list((int)a.K);
        if (!over(a, row)) {
            const int64_t at = row * g.segments;
            for (uint32_t i = lane; i < g.segments; i += 64) top = fmaxf(top, g.tops[at + i]);
            top = wave_max(top);
            for (uint32_t i = lane; i < g.segments; i += 64) {
                const float t = g.tops[at + i];
                const double s = g.sums[at + i];
                // a sum that is not a number stays so; a segment of nothing adds nothing
                sum += s == 0. ? 0. : s * exp_below((double)t - (double)top);
            }
            sum = wave_sum(sum);
            const int n = (int)(g.segments * (uint32_t)a.K);
            for (int i = lane; i - lane < n; i += 64) list.offer(i < n ? g.keys[at * a.K + i] : 0);
        }
        list_beam(a, l, w, row, list.mine, top, sum);
    }
    __syncthreads();
    pick(a, l, r, kPickThreads);
}

// Beams of one segment.
template <class T> __global__ __launch_bounds__(512) void k_beam_small(BeamArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int64_t r = block_of();
    if (r >= a.R) return;
    const Lists l(lds, (int)a.W, (int)a.K);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x / 64;
    for (int w = wave; w < a.W; w += waves) {
        const int64_t row = r * a.W + w;
        if (over(a, row)) {
            list_beam(a, l, w, row, 0, 0.f, 1.);
            continue;
        }
        const Segment<T> s((const T *)a.logits + row * a.ld, 0, a.V, (int)a.K);
        list_beam(a, l, w, row, s.best, s.top, s.sum);
    }
    __syncthreads();
    pick(a, l, r, (int)blockDim.x);
}

size_t lds_of(const BeamArgs &a) { return (size_t)a.W * ((size_t)a.K * 12 + 4); }

int64_t segment_of(int32_t type) { return type == TQ_F32 ? kSegment<float> : kSegment<_Float16>; }

size_t place(int32_t type, const BeamArgs &a, Geom &g)
{
    g.rows = (uint32_t)(a.R * a.W);
    g.segments = (uint32_t)((a.V + segment_of(type) - 1) / segment_of(type));
    if (g.segments == 1) return 0;
    // segments of one length, in whole pieces
    g.length = ((a.V + g.segments - 1) / g.segments + 7) / 8 * 8;
    Carver ws;
    char *base = (char *)a.ws;
    const size_t items = (size_t)g.rows * g.segments;
    g.tops = (float *)(base + ws.take(items * sizeof(float)));
    g.sums = (double *)(base + ws.take(items * sizeof(double)));
    g.keys = (Key *)(base + ws.take(items * (size_t)a.K * sizeof(Key)));
    return ws.used;
}

template <class T> hipError_t beam_t(int32_t type, const BeamArgs &a, hipStream_t s)
{
    Geom g{};
    place(type, a, g);
    if (g.segments == 1) {
        const unsigned threads = 64 * (unsigned)std::min<int64_t>(a.W, 8);
        k_beam_small<T><<<grid_of(a.R), threads, lds_of(a), s>>>(a);
    } else {
        const int64_t waves = (int64_t)g.rows * g.segments, per = kRowThreads / 64;
        k_beam_rows<T><<<grid_of((waves + per - 1) / per), kRowThreads, 0, s>>>(a, g);
        k_beam_pick<<<grid_of(a.R), kPickThreads, lds_of(a), s>>>(a, g);
    }
    return hipGetLastError();
}

// ------------------------------------------------------------------- reorder

constexpr int kTensors = 100;      // of a launch: their places are kernel arguments
constexpr int kCopyBytes = 8192;   // of a wavefront: eight accesses of 16 bytes a lane
constexpr int kCopyThreads = 256;

struct Tensors {
    const char *in[kTensors];
    char *out[kTensors];
    int64_t bytes[kTensors];
    uint64_t first[kTensors + 1];  // piece of a row, over all rows
    int n;
};
static_assert(sizeof(Tensors) < 3700, "kernel arguments are limited to 4096 bytes");

__global__ __launch_bounds__(kCopyThreads) void k_beam_reorder(Tensors t, const int32_t *parents, int64_t W, int64_t K)
{
    const uint64_t piece = (uint64_t)block_of() * (kCopyThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (piece >= t.first[t.n]) return;
    int lo = 0, hi = t.n;  // first[lo] <= piece < first[hi]
    while (hi - lo > 1) {
        const int m = (lo + hi) / 2;
        if (t.first[m] <= piece) lo = m;
        else hi = m;
    }
    const int lane = threadIdx.x & 63;
    const int64_t bytes = t.bytes[lo], pieces = (bytes + kCopyBytes - 1) / kCopyBytes;
    const int64_t at = (int64_t)(piece - t.first[lo]), row = at / pieces, from = (at - row * pieces) * kCopyBytes;
    const int64_t n = min((int64_t)kCopyBytes, bytes - from);
    const int32_t parent = parents[row];
    const bool there = parent >= 0 && parent < W;
    const char *in = t.in[lo] + ((row / K) * W + (there ? parent : 0)) * bytes + from;
    char *out = t.out[lo] + row * bytes + from;
    if (n == kCopyBytes) {
        uint4 v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            v[i] = make_uint4(0, 0, 0, 0);
            if (there) __builtin_memcpy(&v[i], in + (i * 64 + lane) * 16, 16);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) __builtin_memcpy(out + (i * 64 + lane) * 16, &v[i], 16);
        return;
    }
    for (int64_t i = lane * 16; i < n; i += 64 * 16) {
        if (i + 16 <= n) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (there) __builtin_memcpy(&v, in + i, 16);
            __builtin_memcpy(out + i, &v, 16);
        } else
            for (int64_t k = i; k < n; k++) out[k] = there ? in[k] : (char)0;
    }
}

} // namespace

size_t beam_workspace(int32_t type, int64_t R, int64_t W, int64_t V, int64_t K)
{
    BeamArgs a{};
    a.R = R, a.W = W, a.V = V, a.K = K;
    Geom g{};
    return place(type, a, g);
}

hipError_t launch_beam(int32_t type, const BeamArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return beam_t<float>(type, a, s);
    if (type == TQ_BF16) return beam_t<__bf16>(type, a, s);
    return beam_t<_Float16>(type, a, s);
}

hipError_t launch_reorder(const ReorderArgs &a, hipStream_t s)
{
    const int64_t rows = a.R * a.K;
    constexpr int64_t kPer = kCopyThreads / 64, kMost = ((int64_t)1 << 31) * kPer;  // pieces of a launch
    int64_t i = 0;
    while (i < a.n) {
        Tensors t;
        int64_t pieces = 0;
        for (t.n = 0; i < a.n && t.n < kTensors; i++) {
            if (a.bytes[i] == 0) continue;
            const int64_t more = rows * ((a.bytes[i] + kCopyBytes - 1) / kCopyBytes);
            if (t.n && pieces + more > kMost) break;
            t.in[t.n] = (const char *)a.in[i], t.out[t.n] = (char *)a.out[i], t.bytes[t.n] = a.bytes[i];
            t.first[t.n++] = (uint64_t)pieces;
            pieces += more;
        }
        if (t.n == 0) break;
        t.first[t.n] = (uint64_t)pieces;
        k_beam_reorder<<<grid_of((pieces + kPer - 1) / kPer), kCopyThreads, 0, s>>>(t, a.parents, a.W, a.K);
    }
    return hipGetLastError();
}

} // namespace tq
