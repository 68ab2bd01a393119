// model_beam.hip -- one step of a beam search: the best continuations of all beams
// of a record, and the states that go with them.
//
// A beam's candidates score scores[w] + z_v - lse, lse = log sum_u exp z_u.  Which
// candidates of different beams are the best hangs on the last digits of lse, so the
// exponentials and their sum are formed in 64 bits: what is chosen does not depend
// on the order of a sum.  Reading fp32 logits and these exponentials, 25 instructions
// each, take about the same time; 16-bit logits wait for the exponentials (64 x 8 beams
// of 65537 bf16: 47 us, 14 to read them).
//
// A wavefront holds a segment of a beam's logits in registers, 64 lanes of 8 pieces
// of 16 bytes.  With the segment's maximum it forms the sum; the K-th largest of the
// lanes' maxima is a bound that K elements reach, found bit by bit by ballots, so
// that few elements are looked at again.  Up to 64 that reach it are gathered and
// ranked by counting; more are entered one by one in a list of the K best, which the
// lanes hold in order, one each.  Lists are of keys that no two elements share: a
// value's bits in the order of values, then the id, lower ids first.
// A second kernel joins a beam's segments and then the beams, whose lists it takes from
// the front.
// Where a beam is a segment of a few pieces, one kernel does both.
//
// Reordering the states is a copy of rows of any number of tensors in one launch.
#include <algorithm>
#include <type_traits>

#include "model.h"
#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

using Key = unsigned long long;
constexpr int kPieces = 8;  // of 16 bytes, a lane's part of a segment
constexpr int kFewPieces = 2;
template <class T, int P> constexpr int kSegment = 64 * P * kVec<T>;
static_assert(kSegment<float, kPieces> >= 2048, "the limit of a call counts segments of 2048");
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

// exp(x) for -700 <= x <= 0 to about 2^-42: x = n ln 2 + r, the series of e^r to r^10.
// (The rounding of ln 2 costs n 2^-55.)  An instruction takes one constant from scalar
// registers; two are held in vector registers for those that need two.
struct Exp {
    double magic = 0x1.8p52, last = 1. / 3628800.;
    __device__ __forceinline__ Exp() { asm("" : "+v"(magic), "+v"(last)); }
    __device__ __forceinline__ double operator()(double x) const
    {
        const double t = fma(x, 1.4426950408889634, magic), n = t - magic;
        const double r = fma(n, -0x1.62e42fefa39efp-1, x);
        double p = fma(last, r, 1. / 362880.);
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
        const uint32_t hi = (uint32_t)(b >> 32) + ((uint32_t)__builtin_bit_cast(uint64_t, t) << 20);
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)b);
    }
};
constexpr double kFar = -690.;  // what is further below a maximum counts as if it were not

// The larger one, NaN where one is NaN.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <class V> __device__ __forceinline__ V wave_sum(V v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = larger(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ __forceinline__ Key lane_key(Key k, int lane)
{
    return (Key)__builtin_amdgcn_readlane((uint32_t)(k >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((uint32_t)k, lane);
}

// Up to 64 keys that a wavefront finds, put into order by their number of better ones:
// that many instructions as many keys, where entering one after the other takes some
// thirty for each.  64 x 32 beams of 8193 f16, K = 32: 69 us with keys entered one by
// one, 57 us gathered.
struct Gathered {
    Key *room;  // 64 in LDS, the wavefront's own
    int count = 0;
    __device__ explicit Gathered(Key *r) : room(r) {}
    __device__ __forceinline__ void add(bool mine, Key k)
    {
        const unsigned long long all = __ballot(mine);
        const int at = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
        if (mine && at < 64) room[at] = k;
        count += __popcll(all);
    }
    __device__ bool fits() const { return count <= 64; }
    // the K best, one a lane
    __device__ __forceinline__ Key best(int K) const
    {
        const int lane = threadIdx.x & 63;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const Key mine = lane < count ? room[lane] : 0;
        int place = 0;
        for (int i = 0; i < count; i++) place += lane_key(mine, i) > mine;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < count) room[place] = mine;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        return lane < min(count, K) ? room[lane] : 0;
    }
};

// A value, as its bits in the order of values, that K lanes' `high` reach: its first
// bits; 0 where there are not so many lanes.
__device__ __forceinline__ uint32_t reached(uint32_t high, int K)
{
    uint32_t bound = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; bit--) {
        const uint32_t more = bound | 1u << bit;
        if (__popcll(__ballot(high >= more)) >= K) bound = more;
    }
    return bound;
}

// The number of the lane before.
__device__ __forceinline__ uint32_t before(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x138, 0xf, 0xf, true);  // a shift by one over the whole wavefront
}

// A wavefront's list of the K best keys, lane i the i-th; zeros where there are fewer.
struct Best {
    Key mine = 0, least = 0;  // the K-th
    int K;
    __device__ explicit Best(int k) : K(k) {}
    __device__ __forceinline__ void enter(Key k)
    {
        const int lane = threadIdx.x & 63, at = __popcll(__ballot(mine > k));
        const Key left = (Key)before((uint32_t)(mine >> 32)) << 32 | before((uint32_t)mine);
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

// 16 bytes as they are read, so that elements of 16 bits stay two to a register.
template <class T> struct Piece {
    uint32_t w[4];
    __device__ __forceinline__ void load(const T *p, int n)  // n: elements there are
    {
        constexpr int V = kVec<T>;
        if (n >= V) {
            __builtin_memcpy(w, p, sizeof w);
            return;
        }
        T v[V];
#pragma unroll
        for (int j = 0; j < V; j++) {
            v[j] = (T)(float)kNone;
            if (j < n) v[j] = p[j];
        }
        __builtin_memcpy(w, v, sizeof w);
    }
    __device__ __forceinline__ float get(int j) const
    {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[j]);
        else {
            const uint16_t u = (uint16_t)(w[j / 2] >> (j % 2 * 16));
            return (float)__builtin_bit_cast(T, u);
        }
    }
    // what was made of it is not kept in registers
    __device__ __forceinline__ void forget()
    {
        asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
    }
};

// Part [from, to) of a beam's logits, of P pieces a lane: their maximum (NaN where one
// is), the sum of their exponentials relative to it, and the K best.
template <class T, int P> struct Segment {
    static constexpr int V = kVec<T>;
    float top;
    double sum;
    Key best;
    __device__ Segment(const T *row, int64_t from, int64_t to, int K, Key *room)
    {
        const int lane = threadIdx.x & 63;
        const int n = (int)(to - from);
        Piece<T> v[P];
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int at = (p * 64 + lane) * V;
            v[p].load(row + from + at, n - at);
        }
        float mine = (float)kNone, tops[P];
#pragma unroll
        for (int p = 0; p < P; p++) {
            tops[p] = v[p].get(0);
#pragma unroll
            for (int j = 1; j < V; j++) tops[p] = larger(tops[p], v[p].get(j));
            mine = larger(mine, tops[p]);
        }
        top = wave_max(mine);
#pragma unroll
        for (int p = 0; p < P; p++) v[p].forget();
        sum = 0.;
        if (fabsf(top) < (float)-kNone) {
            const Exp exp_below;
            const double base = (double)top;
#pragma unroll
            for (int p = 0; p < P; p++)
                if (p * 64 * V < n) {
                    double s = 0.;
#pragma unroll
                    for (int j = 0; j < V; j++) s += exp_below(fmax((double)v[p].get(j) - base, kFar));
                    sum += s;
                    v[p].forget();
                }
            sum = wave_sum(sum);
        }
        const uint32_t bound = reached(lane * V < n ? ordered(mine) : 0, K);
        float least = bound ? value_of((Key)bound << 32) : (float)kNone;
        if (least != least) least = (float)kNone;  // first bits that no value has
        // calls f with what reaches `least`, a lane's element at a time
        const auto offered = [&](auto &&f) {
#pragma unroll
            for (int p = 0; p < P; p++) {
                const int at = (p * 64 + lane) * V;
                if (p * 64 * V < n && __ballot(tops[p] >= least)) {
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        const float z = v[p].get(j);
                        const bool reaches = z >= least && at + j < n;
                        if (__ballot(reaches)) f(reaches, (Key)ordered(z) << 32 | (uint32_t)~(uint32_t)(from + at + j));
                    }
                }
            }
        };
        Gathered found(room);
        offered([&](bool reaches, Key k) { found.add(reaches, k); });
        if (found.fits()) {
            best = found.best(K);
            return;
        }
        Best list(K);
        offered([&](bool reaches, Key k) {
            list.offer(reaches ? k : 0);
            if (list.least) least = fmaxf(least, value_of(list.least));
        });
        best = list.mine;
    }
};

// The K best candidates of each of a record's beams in LDS, in order.
struct Lists {
    double *score;  // [W][K]
    uint32_t *id;
    Key *room;  // [wavefronts][64]
    __device__ Lists(char *lds, int W, int K)
    {
        room = (Key *)lds;
        score = (double *)(room + blockDim.x);
        id = (uint32_t *)(score + W * K);
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
    // of nothing but -infinity: -infinity; NaN and infinity have no sum
    const double lse = ended ? 0. : (double)top + (fabsf(top) < __builtin_inff() ? log(sum) : 0.);
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
}

// The largest one of a wavefront.
__device__ __forceinline__ uint32_t wave_most(uint32_t v)
{
    const auto moved = [](uint32_t v, auto ctrl, auto rows) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    };
    using std::integral_constant;
    const integral_constant<int, 0xf> all{};
    v = max(v, moved(v, integral_constant<int, 0x111>{}, all));  // lanes 1, 2, 4, 8 before in a row of 16
    v = max(v, moved(v, integral_constant<int, 0x112>{}, all));
    v = max(v, moved(v, integral_constant<int, 0x114>{}, all));
    v = max(v, moved(v, integral_constant<int, 0x118>{}, all));
    v = max(v, moved(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}));  // the row before
    v = max(v, moved(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}));  // both rows before
    return __builtin_amdgcn_readlane(v, 63);
}

// The K best of all beams' candidates: a wavefront takes the best of what the beams
// have left, a lane each, K times; the lower beam where they are as good.
__device__ __forceinline__ void pick(const BeamArgs &a, const Lists &l, int64_t r)
{
    const int W = (int)a.W, K = (int)a.K, n = (int)min((int64_t)K, a.V);  // candidates of a beam
    const int w = threadIdx.x;
    if (w >= 64) return;
    int at = 0;
    double s = 0.;
    uint32_t hi = 0, lo = 0;  // the score's bits in the order of scores; 0: none left
    const auto next = [&] {
        hi = lo = 0;
        if (w >= W || at >= n) return;
        s = l.score[w * K + at];
        const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.);
        const uint64_t o = u ^ ((uint64_t)((int64_t)u >> 63) | (uint64_t)1 << 63);
        hi = (uint32_t)(o >> 32);
        lo = (uint32_t)o;
    };
    next();
    for (int k = 0; k < K; k++) {
        const uint32_t most = wave_most(hi);
        unsigned long long best = __ballot(hi == most);
        if (__popcll(best) > 1) {
            const uint32_t rest = wave_most(hi == most ? lo : 0);  // (of all lanes)
            best = __ballot(hi == most && lo == rest);
        }
        if (w == __builtin_ctzll(best)) {
            a.out_scores[r * K + k] = (float)s;
            a.parents[r * K + k] = w;
            a.tokens[r * K + k] = l.id[w * K + at];
            at++;
            next();
        }
    }
}

constexpr int kRowThreads = 256;
template <class T> __global__ __launch_bounds__(kRowThreads, 4) void k_beam_rows(BeamArgs a, Geom g)
{
    __shared__ Key room[kRowThreads / 64][64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t item = block_of() * (kRowThreads / 64) + wave;
    if (item >= g.rows * g.segments) return;
    const int lane = threadIdx.x & 63;
    const uint32_t row = item / g.segments;
    if (over(a, row)) return;
    const int64_t from = (item - row * g.segments) * g.length;
    const Segment<T, kPieces> s((const T *)a.logits + row * a.ld, from, min(from + g.length, a.V), (int)a.K, room[wave]);
    if (lane == 0) {
        g.tops[item] = s.top;
        g.sums[item] = s.sum;
    }
    if (lane < a.K) g.keys[(int64_t)item * a.K + lane] = s.best;
}

__global__ __launch_bounds__(1024) void k_beam_pick(BeamArgs a, Geom g)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int64_t r = block_of();
    if (r >= a.R) return;
    const Lists l(lds, (int)a.W, (int)a.K);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int w = wave; w < a.W; w += blockDim.x / 64) {
        const int64_t row = r * a.W + w;
        float top = (float)kNone;
        double sum = 0.;
        Key key = 0;
        if (!over(a, row)) {
            const int64_t at = row * g.segments;
            for (uint32_t i = lane; i < g.segments; i += 64) top = larger(top, g.tops[at + i]);
            top = wave_max(top);
            const Exp exp_below;
            if (fabsf(top) < __builtin_inff())
                for (uint32_t i = lane; i < g.segments; i += 64)
                    sum += g.sums[at + i] * exp_below(fmax((double)g.tops[at + i] - (double)top, kFar));
            sum = wave_sum(sum);
            // the best of the segments' lists, as in a segment
            const int K = (int)a.K;
            const int64_t n = (int64_t)g.segments * K;
            const Key *keys = g.keys + at * K;
            uint32_t high = 0;
            for (int64_t i = lane; i < n; i += 64) high = max(high, (uint32_t)(keys[i] >> 32));
            const Key bound = (Key)reached(high, K) << 32;
            Gathered found(l.room + wave * 64);
            for (int64_t i = lane; i - lane < n; i += 64) {
                const Key k = i < n ? keys[i] : 0;
                found.add(k && k >= bound, k);
            }
            if (found.fits()) key = found.best(K);
            else {
                Best list(K);
                for (int64_t i = lane; i - lane < n; i += 64) list.offer(i < n ? keys[i] : 0);
                key = list.mine;
            }
        }
        list_beam(a, l, w, row, key, top, sum);
    }
    __syncthreads();
    pick(a, l, r);
}

// Beams of few pieces.  (Those of one whole segment take two kernels: 580 x 28 beams
// of 1025 fp32 97 us in one, 72 us in two.)
template <class T> __global__ __launch_bounds__(1024) void k_beam_small(BeamArgs a)
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
        const Segment<T, kFewPieces> s((const T *)a.logits + row * a.ld, 0, a.V, (int)a.K, l.room + wave * 64);
        list_beam(a, l, w, row, s.best, s.top, s.sum);
    }
    __syncthreads();
    pick(a, l, r);
}

size_t lds_of(const BeamArgs &a, unsigned threads) { return (size_t)a.W * (size_t)a.K * 12 + threads * sizeof(Key); }

int64_t segment_of(int32_t type) { return type == TQ_F32 ? kSegment<float, kPieces> : kSegment<_Float16, kPieces>; }

bool few(int32_t type, int64_t V)
{
    return V <= (type == TQ_F32 ? kSegment<float, kFewPieces> : kSegment<_Float16, kFewPieces>);
}

size_t place(int32_t type, const BeamArgs &a, Geom &g)
{
    g.rows = (uint32_t)(a.R * a.W);
    g.segments = (uint32_t)((a.V + segment_of(type) - 1) / segment_of(type));
    if (few(type, a.V)) return 0;
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
    if (few(type, a.V)) {
        const unsigned threads = 64 * (unsigned)std::min<int64_t>(a.W, 16);
        k_beam_small<T><<<grid_of(a.R), threads, lds_of(a, threads), s>>>(a);
    } else {
        const int64_t waves = (int64_t)g.rows * g.segments, per = kRowThreads / 64;
        k_beam_rows<T><<<grid_of((waves + per - 1) / per), kRowThreads, 0, s>>>(a, g);
        const unsigned threads = 64 * (unsigned)std::min<int64_t>(a.W, 16);
        k_beam_pick<<<grid_of(a.R), threads, lds_of(a, threads), s>>>(a, g);
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
