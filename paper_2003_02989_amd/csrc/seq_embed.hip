// seq_embed.hip -- embedding lookup with scaling and the gradient of its table.
//
// Lookup: out[i] = scale table[t_i], a gather of rows.  Gradient:
// grad[v] = scale sum_{t_i = v} dout[i].  The tokens are sorted by id with
// their positions (a stable radix sort, so that each id's positions ascend),
// which turns the sums into sums over runs of the sorted list: no atomics on
// floating-point numbers, one fixed order, each row of dout read once and each
// row of grad written once.  The list is cut into equal chunks, whatever the
// runs, so that a few bitstrings that hold most shots of a peaked distribution
// are no different from many that hold one each.
#include <algorithm>
#include <type_traits>

#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

constexpr int kThreads = 256;

// Columns go to lanes W at a time.  The last lane with any takes the row's last
// W, some of them for the second time, so that every access is whole: the same
// numbers are formed and written twice.  W is one 16-byte piece, or 1 for rows
// shorter than that.
template <int W> __device__ __forceinline__ int64_t column(int64_t nominal, int64_t D)
{
    return min(nominal, D - W);
}

// ------------------------------------------------------------------ lookup
// L lanes share a row; a group of them takes kRows rows at a time, so that
// several reads are in flight behind the token reads.  Bound by memory, small
// calls by the launch: 1.9 us for 16 rows of 64 fp32.
constexpr int kRows = 4;

template <class T, int W, int L> __global__ __launch_bounds__(kThreads) void k_embed(EmbedArgs a)
{
    const int lane = threadIdx.x % L;
    const int64_t group = (int64_t)block_of() * (kThreads / L) + threadIdx.x / L;
    const int64_t i0 = group * kRows;
    if (i0 >= a.N) return;
    uint64_t t[kRows];
    const T *from[kRows];
    T *to[kRows];
#pragma unroll
    for (int r = 0; r < kRows; r++) {
        // groups past the end repeat the last row; ids without a row read the first
        const int64_t i = min(i0 + r, a.N - 1);
        t[r] = a.tokens[i];
        from[r] = (const T *)a.table + (int64_t)(t[r] < (uint64_t)a.V ? t[r] : 0) * a.ld_table;
        to[r] = (T *)a.out + i * a.ld_out;
    }
    const bool some = a.V > 0;
    for (int64_t c0 = (int64_t)lane * W; c0 < a.D; c0 += L * W) {
        const int64_t c = column<W>(c0, a.D);
        float f[kRows][W];
#pragma unroll
        for (int r = 0; r < kRows; r++)
            if (some) load_vec<W>(from[r] + c, f[r]);
#pragma unroll
        for (int r = 0; r < kRows; r++) {
            // an id without a row gives zeros whatever the table holds
            const bool on = t[r] < (uint64_t)a.V;
#pragma unroll
            for (int j = 0; j < W; j++) f[r][j] = on ? f[r][j] * a.scale : 0.f;
            store_vec<W>(to[r] + c, f[r]);
        }
    }
}

// Calls f with the elements of a lane and the lanes of a row of D elements.
template <class T, class F> void by_width(int64_t D, F &&f)
{
    using One = std::integral_constant<int, 1>;
    using Whole = std::integral_constant<int, kVec<T>>;
    const int64_t lanes = (D + kVec<T> - 1) / kVec<T>;
    if (D < kVec<T>) f(One{}, std::integral_constant<int, 8>{});
    else if (lanes <= 8) f(Whole{}, std::integral_constant<int, 8>{});
    else if (lanes <= 16) f(Whole{}, std::integral_constant<int, 16>{});
    else if (lanes <= 32) f(Whole{}, std::integral_constant<int, 32>{});
    else f(Whole{}, std::integral_constant<int, 64>{});
}

template <class T> hipError_t embed_t(const EmbedArgs &a, hipStream_t s)
{
    by_width<T>(a.D, [&](auto w, auto l) {
        constexpr int L = decltype(l)::value;
        const int64_t groups = (a.N + kRows - 1) / kRows, per = kThreads / L;
        k_embed<T, decltype(w)::value, L><<<grid_of((groups + per - 1) / per), kThreads, 0, s>>>(a);
    });
    return hipGetLastError();
}

// ------------------------------------------------------------------- sort
// Least-significant-digit radix sort of (id, position).  A workgroup takes
// kSortItems consecutive items; its kSortWaves wavefronts each take a
// contiguous part in steps of 64.  Ranks among equal digits come from ballots
// within a step, from running per-wavefront counters across steps, and from
// prefix sums over wavefronts, workgroups and digits across those: the order
// of equal digits is kept at every level.  At 262144 ids of 17 bits (two passes)
// the three kernels of a pass take 20 us, a few launches' worth each;
// the list (12 bytes an item) is small beside the rows it puts in order.
constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 2048;
constexpr int kSortSteps = kSortItems / kSortThreads;
constexpr int kMaxBits = 11;

// The id of item i: tokens on the first pass (ids without a row sort last, as
// V), sorted ids after it.
__device__ __forceinline__ uint32_t id_of(const uint64_t *tokens, const uint32_t *ids, int64_t i, uint32_t V)
{
    if (ids) return ids[i];
    const uint64_t t = tokens[i];
    return t < V ? (uint32_t)t : V;
}

// Orders the LDS accesses of one wavefront's lanes (they execute in order; this
// keeps the compiler from moving them).
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ uint32_t wave_prefix(uint32_t v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}

// counts[digit][block]
__global__ __launch_bounds__(kSortThreads) void k_sort_count(const uint64_t *tokens, const uint32_t *ids, int64_t N,
                                                            uint32_t V, int shift, int bits, uint32_t *counts)
{
    extern __shared__ uint32_t bins[];
    const int nb = 1 << bits;
    const int64_t i0 = (int64_t)blockIdx.x * kSortItems + threadIdx.x;
    uint32_t id[kSortSteps];
#pragma unroll
    for (int k = 0; k < kSortSteps; k++)
        id[k] = i0 + k * kSortThreads < N ? id_of(tokens, ids, i0 + k * kSortThreads, V) : 0;
    for (int d = threadIdx.x; d < nb; d += kSortThreads) bins[d] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortSteps; k++)
        if (i0 + k * kSortThreads < N) atomicAdd(&bins[(id[k] >> shift) & (nb - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < nb; d += kSortThreads) counts[(int64_t)d * gridDim.x + blockIdx.x] = bins[d];
}

// One wavefront per digit: counts[digit][*] become exclusive prefix sums over
// the blocks, totals[digit] their sum.
__global__ __launch_bounds__(64) void k_sort_scan(uint32_t *counts, int blocks, uint32_t *totals, uint32_t *n_long)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *n_long = 0;  // for k_embed_sums
    uint32_t *row = counts + (int64_t)blockIdx.x * blocks;
    const int lane = threadIdx.x;
    uint32_t carry = 0;
    for (int b0 = 0; b0 < blocks; b0 += 256) {
        uint32_t v[4];
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] = b0 + k * 64 + lane < blocks ? row[b0 + k * 64 + lane] : 0;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const uint32_t s = wave_prefix(v[k]);
            if (b0 + k * 64 + lane < blocks) row[b0 + k * 64 + lane] = carry + s - v[k];
            carry += __shfl(s, 63, 64);
        }
    }
    if (lane == 0) totals[blockIdx.x] = carry;
}

// PER: digits per thread, 2^bits <= PER * kSortThreads.
template <int PER>
__global__ __launch_bounds__(kSortThreads) void k_sort_scatter(const uint64_t *tokens, const uint32_t *ids,
                                                              const uint32_t *pos, int64_t N, uint32_t V, int shift,
                                                              int bits, const uint32_t *counts, const uint32_t *totals,
                                                              uint32_t *ids_out, uint32_t *pos_out)
{
    constexpr int NB = PER * kSortThreads;
    __shared__ uint16_t cnt[kSortWaves][NB];
    __shared__ uint32_t base[NB], wave_sum[kSortWaves];
    const int nb = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d0 = threadIdx.x * PER;
    const int64_t i0 = (int64_t)blockIdx.x * kSortItems + wave * (kSortSteps * 64);
    uint32_t id[kSortSteps], at[kSortSteps], total[PER], before[PER];
#pragma unroll
    for (int k = 0; k < kSortSteps; k++) {
        const int64_t i = i0 + k * 64 + lane;
        id[k] = i < N ? id_of(tokens, ids, i, V) : 0;
        at[k] = i < N ? (pos ? pos[i] : (uint32_t)i) : 0;
    }
#pragma unroll
    for (int j = 0; j < PER; j++) {
        total[j] = d0 + j < nb ? totals[d0 + j] : 0;
        before[j] = d0 + j < nb ? counts[(int64_t)(d0 + j) * gridDim.x + blockIdx.x] : 0;
    }
    for (int d = threadIdx.x; d < kSortWaves * NB / 2; d += kSortThreads) ((uint32_t *)cnt)[d] = 0;
    // exclusive prefix sums of the digits' totals
    uint32_t own = 0;
#pragma unroll
    for (int j = 0; j < PER; j++) own += total[j];
    const uint32_t s = wave_prefix(own);
    if (lane == 63) wave_sum[wave] = s;
    __syncthreads();
    uint32_t run = s - own;
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) run += w < wave ? wave_sum[w] : 0;
#pragma unroll
    for (int j = 0; j < PER; j++) {
        base[d0 + j] = run + before[j];
        run += total[j];
    }
    uint16_t *mine = cnt[wave];
    uint32_t rank[kSortSteps];
#pragma unroll
    for (int k = 0; k < kSortSteps; k++) {
        const bool in = i0 + k * 64 + lane < N;
        const int d = (id[k] >> shift) & (nb - 1);
        uint64_t same = __ballot(in);
        for (int b = 0; b < bits; b++) {
            const bool set = (d >> b) & 1;
            const uint64_t m = __ballot(set);
            same &= set ? m : ~m;
        }
        const int lower = __popcll(same & (((uint64_t)1 << lane) - 1));
        // all lanes read the counters before the first lane of each digit moves
        // its counter on, and those writes come before the next step's reads
        const int seen = in ? mine[d] : 0;
        rank[k] = seen + lower;
        wave_fence();
        if (in && lower == 0) mine[d] = (uint16_t)(seen + __popcll(same));
        wave_fence();
    }
    __syncthreads();
    for (int d = threadIdx.x; d < nb; d += kSortThreads) {
        uint32_t sum = base[d];
#pragma unroll
        for (int w = 0; w < kSortWaves; w++) {
            const uint16_t c = cnt[w][d];
            cnt[w][d] = (uint16_t)(sum - base[d]);
            sum += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortSteps; k++)
        if (i0 + k * 64 + lane < N) {
            const int d = (id[k] >> shift) & (nb - 1);
            const uint32_t o = base[d] + mine[d] + rank[k];
            ids_out[o] = id[k];
            pos_out[o] = at[k];
        }
}

// ------------------------------------------------------------------- sums
// The sorted list is cut into chunks.  A group of L lanes walks a chunk, kAhead
// rows in flight, and adds up its runs of equal ids.  A run that goes at most
// kOver places past the chunk it begins in is finished there, and passed over by
// the group of the next chunk.  Longer runs leave a partial sum per chunk, in
// row 2c + 1 where they begin and 2c where they go on, and k_embed_join adds
// these up; the chunks that long runs begin in are entered into a list (the
// order of the entries is a matter of chance, what is summed is not).
constexpr int kAhead = 8, kOver = 64;

struct SumArgs {
    EmbedGradArgs a;
    const uint32_t *ids, *pos;
    int64_t chunks;
    int chunk, chunk_blocks;
    float *partial;
    uint32_t *n_long, *longs;
};

// Whether the run of `id`, which goes on at place e, the end of a chunk, goes
// on for more than kOver places.
__device__ __forceinline__ bool goes_far(const SumArgs &s, int64_t e, uint32_t id)
{
    return e + kOver < s.a.N && s.ids[e + kOver] == id;
}

template <class T, int W>
__device__ __forceinline__ void sum_chunk(const SumArgs &s, int64_t c, int64_t col, bool first_lane)
{
    const EmbedGradArgs &a = s.a;
    const uint32_t N = (uint32_t)a.N, V = (uint32_t)a.V;
    const uint32_t b = (uint32_t)(c * s.chunk), e = min(b + (uint32_t)s.chunk, N);
    const T *dout = (const T *)a.dout + col;
    uint32_t cur = s.ids[b], i = b, end = e;
    bool began = b == 0 || s.ids[b - 1] != cur;
    if (!began) {
        // passed over, unless it is long: by where it began and how far it goes
        const bool there = b == (uint32_t)s.chunk || s.ids[b - s.chunk - 1] != cur;
        if (there && !goes_far(s, b, cur)) {
            began = true;
            while (i < e && s.ids[i] == cur) i++;
            if (i == e) return;
            cur = s.ids[i];
        }
    }
    if (cur >= V) return;
    const uint32_t last = s.ids[e - 1];
    bool whole = true;  // the chunk's last run ends here
    if (last < V && e < N && s.ids[e] == last) {
        whole = !goes_far(s, e, last) && (s.ids[b] != last || b == 0 || s.ids[b - 1] != last);
        if (whole) end = min(e + (uint32_t)kOver, N);
    }
    float acc[W];
#pragma unroll
    for (int j = 0; j < W; j++) acc[j] = 0.f;
    auto flush = [&](bool ended) {
        if (began && ended) {
#pragma unroll
            for (int j = 0; j < W; j++) acc[j] *= a.scale;
            store_vec<W>((T *)a.grad + (int64_t)cur * a.ld_grad + col, acc);
        } else {
            store_vec<W>(s.partial + (2 * c + (began ? 1 : 0)) * a.D + col, acc);
            if (began && first_lane) s.longs[atomicAdd(s.n_long, 1u)] = (uint32_t)c;
        }
#pragma unroll
        for (int j = 0; j < W; j++) acc[j] = 0.f;
    };
    for (; i < end; i += kAhead) {
        uint32_t id[kAhead], from[kAhead];
        float f[kAhead][W];
#pragma unroll
        for (int r = 0; r < kAhead; r++) {
            const uint32_t k = min(i + r, end - 1);
            id[r] = s.ids[k];
            from[r] = s.pos[k];
        }
#pragma unroll
        for (int r = 0; r < kAhead; r++) load_vec<W>(dout + (int64_t)from[r] * a.ld_dout, f[r]);
#pragma unroll
        for (int r = 0; r < kAhead; r++) {
            if (i + r >= end) break;
            if (id[r] != cur) {
                flush(true);
                began = true;
                cur = id[r];
                if (cur >= V || i + r >= e) return;  // past the chunk only its last run
            }
#pragma unroll
            for (int j = 0; j < W; j++) acc[j] += f[r][j];
        }
    }
    flush(whole);
}

// The first `chunk_blocks` workgroups sum chunks, the others write the zeros of
// ids that no token has: each of their wavefronts looks 64 ids up in the list.
// Bound by memory: 262144 rows of 512 bf16 into 65537 in 74 us, 4.5 TB/s of
// rows read in the order of their ids and rows written.
template <class T, int W, int L> __global__ __launch_bounds__(kThreads) void k_embed_sums(SumArgs s)
{
    constexpr int G = kThreads / L;
    const EmbedGradArgs &a = s.a;
    if ((int)blockIdx.x < s.chunk_blocks) {
        int g = threadIdx.x / L;
        if constexpr (L == 64) g = __builtin_amdgcn_readfirstlane(g);  // addresses and branches are scalar
        const int64_t c = (int64_t)blockIdx.x * G + g;
        if (c >= s.chunks) return;
        for (int64_t c0 = (int64_t)(threadIdx.x % L) * W; c0 < a.D; c0 += L * W)
            sum_chunk<T, W>(s, c, column<W>(c0, a.D), c0 == 0);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int64_t v0 = ((int64_t)(blockIdx.x - s.chunk_blocks) * (kThreads / 64) + (threadIdx.x >> 6)) * 64;
    const uint32_t v = (uint32_t)min(v0 + lane, a.V - 1);
    uint32_t lo = 0, hi = (uint32_t)a.N;
    while (lo < hi) {
        const uint32_t m = (lo + hi) >> 1;
        if (s.ids[m] < v) lo = m + 1;
        else hi = m;
    }
    const bool absent = v0 + lane < a.V && (lo == (uint32_t)a.N || s.ids[lo] != v);
    const float zero[W] = {};
    for (uint64_t m = __ballot(absent); m; m &= m - 1) {
        T *row = (T *)a.grad + (v0 + __ffsll((unsigned long long)m) - 1) * a.ld_grad;
        for (int64_t c0 = (int64_t)lane * W; c0 < a.D; c0 += 64 * W) store_vec<W>(row + column<W>(c0, a.D), zero);
    }
}

// The long runs: the partial sum of the chunk a run begins in and those of the
// chunks after it that begin with the same id.  64 columns per workgroup; its
// wavefronts take equal parts of those chunks.  Two ids that hold nearly all of
// 100003 rows of 200 fp32: 19 us after 20 us for the chunks.
constexpr int kJoinWaves = 16;
template <class T> __global__ __launch_bounds__(kJoinWaves * 64) void k_embed_join(SumArgs s)
{
    __shared__ float part[kJoinWaves][64];
    const EmbedGradArgs &a = s.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n_long = *s.n_long;
    for (uint32_t q = blockIdx.x; q < n_long; q += gridDim.x) {
        const int64_t c = s.longs[q];
        const uint32_t id = s.ids[(c + 1) * s.chunk];
        // n: the chunks after c that begin with it, 64 places tried at a time
        int64_t n = 0, hi = s.chunks - c - 1;
        while (n < hi) {
            const int64_t step = (hi - n + 63) / 64, k = n + lane * step;
            const uint64_t m = __ballot(k < hi && s.ids[(c + 1 + min(k, hi - 1)) * s.chunk] == id);
            const int yes = __popcll(m);  // the first `yes` places begin with it
            if (yes == 0) break;
            hi = min(hi, n + yes * step);
            n += (yes - 1) * step + 1;
        }
        const int64_t col = (int64_t)blockIdx.y * 64 + lane, per = (n + kJoinWaves - 1) / kJoinWaves;
        const int64_t k0 = min(wave * per, n), k1 = min(k0 + per, n);
        float t = 0.f;
        if (col < a.D) {
            if (wave == 0) t = s.partial[(2 * c + 1) * a.D + col];
#pragma unroll 16
            for (int64_t k = k0; k < k1; k++) t += s.partial[2 * (c + 1 + k) * a.D + col];
        }
        part[wave][lane] = t;
        __syncthreads();
        if (wave == 0 && col < a.D) {
            t = 0.f;
#pragma unroll
            for (int w = 0; w < kJoinWaves; w++) t += part[w][lane];
            ((T *)a.grad)[(int64_t)id * a.ld_grad + col] = (T)(t * a.scale);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------- a few tokens
// Up to kFewTokens tokens need no sort: a workgroup marks which of its `rows`
// rows of grad have tokens at all, and a wavefront compares the id of such a row
// with all of them.  One launch in place of five or eight: 8 us against 45 us for
// 62 tokens.  Where all tokens have one id their rows are added by one wavefront,
// which is why wide rows allow fewer tokens: 476 tokens of two ids, 1816 columns
// into 262145 rows, took 350 us in place of 200 us.
constexpr int kFewTokens = 512, kFewRows = 256;
template <class T, int W> __global__ __launch_bounds__(kThreads) void k_embed_few(EmbedGradArgs a, int rows)
{
    __shared__ uint32_t tok[kFewTokens];
    __shared__ uint8_t some[kFewRows];
    const int lane = threadIdx.x & 63, N = (int)a.N;
    const int64_t v0 = (int64_t)blockIdx.x * rows;
    some[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < (N + 63) / 64 * 64; i += kThreads) {
        tok[i] = i < N ? id_of(a.tokens, nullptr, i, (uint32_t)a.V) : (uint32_t)a.V;
        const int64_t r = (int64_t)tok[i] - v0;
        if (r >= 0 && r < rows) some[r] = 1;
    }
    __syncthreads();
    for (int r = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < rows; r += kThreads / 64) {
        const int64_t v = v0 + r;
        if (v >= a.V) return;
        const bool any = __builtin_amdgcn_readfirstlane(some[r]);
        uint64_t has[kFewTokens / 64];  // the tokens with id v
        if (any)
#pragma unroll
            for (int k = 0; k < kFewTokens / 64; k++)
                has[k] = k * 64 < N ? __ballot(tok[k * 64 + lane] == (uint32_t)v) : 0;
        for (int64_t c0 = 0; c0 < a.D; c0 += 64 * W) {
            // lanes past the last column sum it again
            const int64_t col = column<W>(c0 + lane * W, a.D);
            const T *dout = (const T *)a.dout + col;
            float acc[W];
#pragma unroll
            for (int j = 0; j < W; j++) acc[j] = 0.f;
            if (any)
#pragma unroll
                for (int k = 0; k < kFewTokens / 64; k++)
                    for (uint64_t m = has[k]; m;) {
                        float f[kAhead][W];
                        int n = 0, at = 0;
#pragma unroll
                        for (int r = 0; r < kAhead; r++) {
                            if (m) at = k * 64 + __ffsll((unsigned long long)m) - 1, n = r + 1;
                            m &= m - 1;
                            load_vec<W>(dout + (int64_t)at * a.ld_dout, f[r]);
                        }
#pragma unroll
                        for (int r = 0; r < kAhead; r++)
                            if (r < n)
#pragma unroll
                                for (int j = 0; j < W; j++) acc[j] += f[r][j];
                    }
#pragma unroll
            for (int j = 0; j < W; j++) acc[j] = any ? acc[j] * a.scale : 0.f;
            store_vec<W>((T *)a.grad + v * a.ld_grad + col, acc);
        }
    }
}

// What a gradient call needs beside its arrays.
struct GradPlan {
    bool few;
    int bits, passes, chunk;
    int64_t blocks, chunks;
    size_t ids[2], pos[2], counts, totals, partial, n_long, longs, bytes;
    GradPlan(int64_t V, int64_t D, int64_t N)
    {
        bytes = 0;
        few = N * ((D + 255) / 256) <= kFewTokens;
        if (few) return;
        int all = 1;
        while (((int64_t)1 << all) <= V) all++;  // ids 0 .. V
        passes = (all + kMaxBits - 1) / kMaxBits;
        bits = (all + passes - 1) / passes;
        blocks = (N + kSortItems - 1) / kSortItems;
        // About four thousand chunks fill the chip; sums of more, shorter ones
        // would only add to the partial sums.
        chunk = (int)std::max<int64_t>(16, (N / 4096 + kAhead - 1) / kAhead * kAhead);
        chunks = (N + chunk - 1) / chunk;
        Carver c;
        for (int k = 0; k < 2; k++) {
            ids[k] = c.take(4 * N);
            pos[k] = c.take(4 * N);
        }
        counts = c.take(((size_t)4 << bits) * blocks);
        totals = c.take((size_t)4 << bits);
        partial = c.take(sizeof(float) * 2 * chunks * D);
        n_long = c.take(sizeof(uint32_t));
        longs = c.take(sizeof(uint32_t) * chunks);
        bytes = c.used;
    }
};

template <class T> hipError_t embed_grad_t(const EmbedGradArgs &a, hipStream_t s)
{
    const GradPlan p(a.V, a.D, a.N);
    if (p.few) {
        const int rows = (int)std::max<int64_t>(kThreads / 64, std::min<int64_t>((a.V + 8191) / 8192, kFewRows));
        by_width<T>(a.D, [&](auto w, auto) {
            constexpr int W = decltype(w)::value;
            k_embed_few<T, W><<<(unsigned)((a.V + rows - 1) / rows), kThreads, 0, s>>>(a, rows);
        });
        return hipGetLastError();
    }
    char *ws = (char *)a.ws;
    uint32_t *ids[2], *pos[2];
    for (int k = 0; k < 2; k++) {
        ids[k] = (uint32_t *)(ws + p.ids[k]);
        pos[k] = (uint32_t *)(ws + p.pos[k]);
    }
    uint32_t *counts = (uint32_t *)(ws + p.counts), *totals = (uint32_t *)(ws + p.totals);
    const size_t nb = (size_t)1 << p.bits;
    const uint32_t V = (uint32_t)a.V;
    for (int k = 0; k < p.passes; k++) {
        const int shift = k * p.bits;
        const uint32_t *in_ids = k ? ids[(k - 1) & 1] : nullptr, *in_pos = k ? pos[(k - 1) & 1] : nullptr;
        k_sort_count<<<p.blocks, kSortThreads, 4 * nb, s>>>(a.tokens, in_ids, a.N, V, shift, p.bits, counts);
        k_sort_scan<<<nb, 64, 0, s>>>(counts, (int)p.blocks, totals, (uint32_t *)(ws + p.n_long));
        auto scatter = [&](auto kernel) {
            kernel<<<p.blocks, kSortThreads, 0, s>>>(a.tokens, in_ids, in_pos, a.N, V, shift, p.bits, counts, totals,
                                                     ids[k & 1], pos[k & 1]);
        };
        if (nb <= kSortThreads) scatter(k_sort_scatter<1>);
        else if (nb <= 2 * kSortThreads) scatter(k_sort_scatter<2>);
        else scatter(k_sort_scatter<4>);
    }
    SumArgs u{a, ids[(p.passes - 1) & 1], pos[(p.passes - 1) & 1], p.chunks, p.chunk, 0, (float *)(ws + p.partial),
              (uint32_t *)(ws + p.n_long), (uint32_t *)(ws + p.longs)};
    by_width<T>(a.D, [&](auto w, auto l) {
        constexpr int L = decltype(l)::value;
        const int64_t per = kThreads / L, zeros = (a.V + kThreads - 1) / kThreads;
        u.chunk_blocks = (int)((p.chunks + per - 1) / per);
        k_embed_sums<T, decltype(w)::value, L><<<(unsigned)(u.chunk_blocks + zeros), kThreads, 0, s>>>(u);
    });
    // a long run has more than kOver places: with fewer ids there is none to join
    const int64_t most = a.N / (kOver + 1);
    if (most)
        k_embed_join<T><<<dim3((unsigned)std::min<int64_t>(most, 128), (unsigned)((a.D + 63) / 64)), kJoinWaves * 64, 0,
                         s>>>(u);
    return hipGetLastError();
}

} // namespace

hipError_t launch_embed(int32_t type, const EmbedArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return embed_t<float>(a, s);
    if (type == TQ_BF16) return embed_t<__bf16>(a, s);
    return embed_t<_Float16>(a, s);
}

size_t embed_grad_workspace(int64_t V, int64_t D, int64_t N) { return GradPlan(V, D, N).bytes; }

hipError_t launch_embed_grad(int32_t type, const EmbedGradArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return embed_grad_t<float>(a, s);
    if (type == TQ_BF16) return embed_grad_t<__bf16>(a, s);
    return embed_grad_t<_Float16>(a, s);
}

} // namespace tq
