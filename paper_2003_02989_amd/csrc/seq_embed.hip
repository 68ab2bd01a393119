// seq_embed.hip -- embedding lookup with scaling and the gradient of its table.
//
// Lookup: out[i] = scale table[t_i], a gather of rows.  Gradient:
// grad[v] = scale sum_{t_i = v} dout[i].  The tokens are sorted by id with
// their positions (a stable radix sort, so that each id's positions ascend),
// which turns the sums into sums over runs of the sorted list: no atomics on
// floating-point numbers, one fixed order, each row of dout read once and each
// row of grad written once.
#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------ lookup
// L lanes share a row in 16-byte pieces; a group of them takes kRows rows at a
// time, so that several reads are in flight behind the token reads.
constexpr int kRows = 4;

template <class T, int L> __global__ __launch_bounds__(kThreads) void k_embed(EmbedArgs a)
{
    constexpr int VE = kVec<T>;
    const int lane = threadIdx.x % L;
    const int64_t group = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const int64_t i0 = group * kRows;
    if (i0 >= a.N) return;
    const T *table = (const T *)a.table;
    T *out = (T *)a.out;
    uint64_t t[kRows];
#pragma unroll
    for (int r = 0; r < kRows; r++) t[r] = i0 + r < a.N ? a.tokens[i0 + r] : ~(uint64_t)0;
    for (int64_t c = (int64_t)lane * VE; c < a.D; c += L * VE) {
        const int n = (int)min((int64_t)VE, a.D - c);
        float f[kRows][VE];
#pragma unroll
        for (int r = 0; r < kRows; r++) {
            if (t[r] < (uint64_t)a.V) load_part<VE>(table + (int64_t)t[r] * a.ld_table + c, n, f[r]);
            else
#pragma unroll
                for (int j = 0; j < VE; j++) f[r][j] = 0.f;
        }
#pragma unroll
        for (int r = 0; r < kRows; r++) {
            if (i0 + r >= a.N) break;
            // an id without a row gives zeros whatever the scale
            if (t[r] < (uint64_t)a.V)
#pragma unroll
                for (int j = 0; j < VE; j++) f[r][j] *= a.scale;
            store_part<VE>(out + (i0 + r) * a.ld_out + c, n, f[r]);
        }
    }
}

template <class T> hipError_t embed_t(const EmbedArgs &a, hipStream_t s)
{
    const int64_t chunks = (a.D + kVec<T> - 1) / kVec<T>;
    auto go = [&](auto kernel, int L) {
        const int64_t groups = (a.N + kRows - 1) / kRows;
        const int64_t per = kThreads / L;
        kernel<<<(unsigned)((groups + per - 1) / per), kThreads, 0, s>>>(a);
        return hipGetLastError();
    };
    if (chunks <= 8) return go(k_embed<T, 8>, 8);
    if (chunks <= 16) return go(k_embed<T, 16>, 16);
    if (chunks <= 32) return go(k_embed<T, 32>, 32);
    return go(k_embed<T, 64>, 64);
}

// ------------------------------------------------------------------- sort
// Least-significant-digit radix sort of (id, position).  A workgroup takes
// kSortItems consecutive items; its kSortWaves wavefronts each take a
// contiguous part in steps of 64.  Ranks among equal digits come from ballots
// within a step, from running per-wavefront counters across steps, and from
// prefix sums over wavefronts, workgroups and digits across those: the order
// of equal digits is kept at every level.
constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 4096;
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

// counts[digit][block]
__global__ __launch_bounds__(kSortThreads) void k_sort_count(const uint64_t *tokens, const uint32_t *ids, int64_t N,
                                                            uint32_t V, int shift, int bits, uint32_t *counts)
{
    extern __shared__ uint32_t bins[];
    const int nb = 1 << bits;
    for (int d = threadIdx.x; d < nb; d += kSortThreads) bins[d] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * kSortItems;
    for (int k = 0; k < kSortSteps; k++) {
        const int64_t i = i0 + k * kSortThreads + threadIdx.x;
        if (i < N) atomicAdd(&bins[(id_of(tokens, ids, i, V) >> shift) & (nb - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < nb; d += kSortThreads) counts[(int64_t)d * gridDim.x + blockIdx.x] = bins[d];
}

// One wavefront per digit: counts[digit][*] become exclusive prefix sums over
// the blocks, totals[digit] their sum.
__global__ __launch_bounds__(64) void k_sort_scan(uint32_t *counts, int blocks, uint32_t *totals)
{
    uint32_t *row = counts + (int64_t)blockIdx.x * blocks;
    const int lane = threadIdx.x;
    uint32_t carry = 0;
    for (int b0 = 0; b0 < blocks; b0 += 64) {
        const uint32_t v = b0 + lane < blocks ? row[b0 + lane] : 0;
        uint32_t s = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(s, d, 64);
            if (lane >= d) s += o;
        }
        if (b0 + lane < blocks) row[b0 + lane] = carry + s - v;
        carry += __shfl(s, 63, 64);
    }
    if (lane == 0) totals[blockIdx.x] = carry;
}

__global__ __launch_bounds__(kSortThreads) void k_sort_scatter(const uint64_t *tokens, const uint32_t *ids,
                                                              const uint32_t *pos, int64_t N, uint32_t V, int shift,
                                                              int bits, const uint32_t *counts, const uint32_t *totals,
                                                              uint32_t *ids_out, uint32_t *pos_out)
{
    // per wavefront and digit a counter, then one offset per digit
    extern __shared__ uint32_t lds[];
    __shared__ uint32_t wave_sum[kSortWaves];
    const int nb = 1 << bits;
    uint16_t *cnt = (uint16_t *)lds;
    uint32_t *base = lds + (kSortWaves * nb) / 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < kSortWaves * nb / 2; d += kSortThreads) lds[d] = 0;
    // exclusive prefix sums of the digits' totals: a contiguous part per thread
    {
        const int per = (nb + kSortThreads - 1) / kSortThreads;
        const int d0 = threadIdx.x * per;
        uint32_t own = 0;
        for (int j = 0; j < per; j++) own += d0 + j < nb ? totals[d0 + j] : 0;
        uint32_t s = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(s, d, 64);
            if (lane >= d) s += o;
        }
        if (lane == 63) wave_sum[wave] = s;
        __syncthreads();
        uint32_t run = s - own;
        for (int w = 0; w < wave; w++) run += wave_sum[w];
        for (int j = 0; j < per; j++) {
            const int d = d0 + j;
            if (d < nb) {
                base[d] = run + counts[(int64_t)d * gridDim.x + blockIdx.x];
                run += totals[d];
            }
        }
    }
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * kSortItems + wave * (kSortSteps * 64);
    uint16_t *mine = cnt + wave * nb;
    uint32_t id[kSortSteps], at[kSortSteps];
    uint16_t rank[kSortSteps];
#pragma unroll
    for (int k = 0; k < kSortSteps; k++) {
        const int64_t i = i0 + k * 64 + lane;
        const bool in = i < N;
        id[k] = in ? id_of(tokens, ids, i, V) : 0;
        at[k] = in ? (pos ? pos[i] : (uint32_t)i) : 0;
    }
#pragma unroll
    for (int k = 0; k < kSortSteps; k++) {
        const bool in = i0 + k * 64 + lane < N;
        const int d = (id[k] >> shift) & (nb - 1);
        uint64_t same = __ballot(in);
        for (int b = 0; b < bits; b++) {
            const uint64_t m = __ballot((d >> b) & 1);
            same &= ((d >> b) & 1) ? m : ~m;
        }
        const int before = __popcll(same & (((uint64_t)1 << lane) - 1));
        // all lanes read the counters before the first lane of each digit moves
        // its counter on, and those writes come before the next step's reads
        const int seen = in ? mine[d] : 0;
        rank[k] = (uint16_t)(seen + before);
        wave_fence();
        if (in && before == 0) mine[d] = (uint16_t)(seen + __popcll(same));
        wave_fence();
    }
    __syncthreads();
    for (int d = threadIdx.x; d < nb; d += kSortThreads) {
        uint32_t run = 0;
        for (int w = 0; w < kSortWaves; w++) {
            const uint16_t c = cnt[w * nb + d];
            cnt[w * nb + d] = (uint16_t)run;
            run += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortSteps; k++) {
        if (i0 + k * 64 + lane < N) {
            const int d = (id[k] >> shift) & (nb - 1);
            const uint32_t o = base[d] + mine[d] + rank[k];
            ids_out[o] = id[k];
            pos_out[o] = at[k];
        }
    }
}

// ------------------------------------------------------------------- sums
// Runs of equal ids in the sorted list.  A run of at most kShort places is
// summed by one group of lanes.  A longer one (a few bitstrings hold most shots
// of a peaked distribution) is cut into pieces of `piece` places, each summed
// into a row of fp32 partial sums of its own, which k_embed_join adds up.
constexpr int kShort = 64;
constexpr int kAhead = 8;  // rows in flight per group

struct LongRun {
    uint32_t v, start, count, first;  // first: its first row of partial sums
};

// starts[v], v in [0, V]: the first place of an id >= v in the sorted list.
// Long runs are entered into a list; `tally` holds (runs << 32 | pieces), one
// addition per entry, so that the entries' first pieces ascend.  Where an entry
// lands depends on the order of these additions, what is summed does not.
__global__ __launch_bounds__(kThreads) void k_embed_runs(const uint32_t *ids, int64_t N, int64_t V, int piece,
                                                        uint32_t *starts, unsigned long long *tally, LongRun *runs)
{
    const int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (v > V) return;
    auto place = [&](int64_t id) {
        int64_t lo = 0, hi = N;
        while (lo < hi) {
            const int64_t m = (lo + hi) >> 1;
            if (ids[m] < (uint32_t)id) lo = m + 1;
            else hi = m;
        }
        return (uint32_t)lo;
    };
    const uint32_t b = place(v);
    starts[v] = b;
    if (v == V) return;
    // a run longer than kShort has its id kShort places on
    if ((int64_t)b + kShort < N && ids[b + kShort] == (uint32_t)v) {
        const uint32_t count = place(v + 1) - b;
        const uint32_t np = (count + piece - 1) / piece;
        const unsigned long long t = atomicAdd(tally, ((unsigned long long)1 << 32) | np);
        runs[t >> 32] = LongRun{(uint32_t)v, b, count, (uint32_t)t};
    }
}

// Sum of the rows at places [b, e) of the list, in their order.
template <class T>
__device__ __forceinline__ void sum_rows(const T *dout, int64_t ld, const uint32_t *pos, uint32_t b, uint32_t e, int n,
                                         float (&acc)[kVec<T>])
{
    constexpr int VE = kVec<T>;
#pragma unroll
    for (int j = 0; j < VE; j++) acc[j] = 0.f;
    for (uint32_t i = b; i < e; i += kAhead) {
        float f[kAhead][VE];
#pragma unroll
        for (int r = 0; r < kAhead; r++) {
            if (i + r < e) load_part<VE>(dout + (int64_t)pos[i + r] * ld, n, f[r]);
            else
#pragma unroll
                for (int j = 0; j < VE; j++) f[r][j] = 0.f;
        }
#pragma unroll
        for (int r = 0; r < kAhead; r++)
#pragma unroll
            for (int j = 0; j < VE; j++) acc[j] += f[r][j];
    }
}

// Workgroups [0, piece_blocks) sum the pieces of long runs, the others the
// short runs, kThreads / L rows of grad each; absent ids get zeros.
template <class T, int L>
__global__ __launch_bounds__(kThreads) void k_embed_sums(EmbedGradArgs a, const uint32_t *pos, const uint32_t *starts,
                                                        const unsigned long long *tally, const LongRun *runs,
                                                        float *partial, int piece, int piece_blocks)
{
    constexpr int VE = kVec<T>, G = kThreads / L;
    __shared__ float part[G][L * VE];
    const int lane = threadIdx.x % L, g = threadIdx.x / L;
    const T *dout = (const T *)a.dout;
    if ((int)blockIdx.x >= piece_blocks) {
        const int64_t v = (int64_t)(blockIdx.x - piece_blocks) * G + g;
        if (v >= a.V) return;
        const uint32_t b = starts[v], e = starts[v + 1];
        if (e - b > kShort) return;
        for (int64_t c = (int64_t)lane * VE; c < a.D; c += L * VE) {
            const int n = (int)min((int64_t)VE, a.D - c);
            float acc[VE];
            sum_rows<T>(dout + c, a.ld_dout, pos, b, e, n, acc);
            if (b < e)
#pragma unroll
                for (int j = 0; j < VE; j++) acc[j] *= a.scale;
            store_part<VE>((T *)a.grad + v * a.ld_grad + c, n, acc);
        }
        return;
    }
    const unsigned long long t = *tally;
    const uint32_t n_runs = (uint32_t)(t >> 32), n_pieces = (uint32_t)t;
    for (uint32_t p = blockIdx.x; p < n_pieces; p += piece_blocks) {
        uint32_t lo = 0, hi = n_runs;  // the last run with first <= p
        while (hi - lo > 1) {
            const uint32_t m = (lo + hi) >> 1;
            if (runs[m].first <= p) lo = m;
            else hi = m;
        }
        const LongRun r = runs[lo];
        const uint32_t b0 = r.start + (p - r.first) * piece;
        const uint32_t e0 = min(b0 + (uint32_t)piece, r.start + r.count);
        // the groups take equal parts of the piece; their sums are added in order
        const uint32_t per = (e0 - b0 + G - 1) / G;
        const uint32_t b = min(b0 + g * per, e0), e = min(b + per, e0);
        for (int64_t c0 = 0; c0 < a.D; c0 += L * VE) {
            const int64_t c = c0 + lane * VE;
            const int n = (int)max((int64_t)0, min((int64_t)VE, a.D - c));
            float acc[VE];
            sum_rows<T>(dout + (n ? c : 0), a.ld_dout, pos, b, n ? e : b, n, acc);
#pragma unroll
            for (int j = 0; j < VE; j++) part[g][lane * VE + j] = acc[j];
            __syncthreads();
            for (int j = threadIdx.x; j < L * VE; j += kThreads) {
                float s = 0.f;
                for (int k = 0; k < G; k++) s += part[k][j];
                if (c0 + j < a.D) partial[(int64_t)p * a.D + c0 + j] = s;
            }
            __syncthreads();
        }
    }
}

// The partial sums of each long run, added up: the workgroup's wavefronts take
// equal parts of the run's pieces, 64 columns at a time.
constexpr int kJoinWaves = 16;
template <class T>
__global__ __launch_bounds__(kJoinWaves * 64) void k_embed_join(EmbedGradArgs a, const unsigned long long *tally,
                                                               const LongRun *runs, const float *partial, int piece)
{
    __shared__ float part[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n_runs = (uint32_t)(*tally >> 32);
    const int64_t c = (int64_t)blockIdx.y * 64 + lane;
    for (uint32_t k = blockIdx.x; k < n_runs; k += gridDim.x) {
        const LongRun r = runs[k];
        const uint32_t np = (r.count + piece - 1) / piece;
        const uint32_t per = (np + kJoinWaves - 1) / kJoinWaves;
        const uint32_t b = min(wave * per, np), e = min(b + per, np);
        float s = 0.f;
        if (c < a.D)
#pragma unroll 8
            for (uint32_t p = b; p < e; p++) s += partial[(int64_t)(r.first + p) * a.D + c];
        part[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && c < a.D) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < kJoinWaves; w++) t += part[w][lane];
            ((T *)a.grad)[(int64_t)r.v * a.ld_grad + c] = (T)(t * a.scale);
        }
        __syncthreads();
    }
}

__global__ void k_clear_tally(unsigned long long *tally) { *tally = 0; }

// What a gradient call needs beside its arrays.
struct GradPlan {
    int bits, passes, piece;
    int64_t blocks, max_runs, max_pieces;
    size_t ids[2], pos[2], counts, totals, starts, tally, runs, partial, bytes;
    GradPlan(int64_t V, int64_t D, int64_t N)
    {
        int all = 1;
        while (((int64_t)1 << all) <= V) all++;  // ids 0 .. V
        passes = (all + kMaxBits - 1) / kMaxBits;
        bits = (all + passes - 1) / passes;
        blocks = (N + kSortItems - 1) / kSortItems;
        // pieces of a run: at most about a thousand
        piece = 128;
        while (piece < 4096 && (int64_t)piece * 1024 < N) piece *= 2;
        max_runs = N / (kShort + 1);
        max_pieces = max_runs ? N / piece + max_runs : 0;
        Carver c;
        for (int k = 0; k < 2; k++) {
            ids[k] = c.take(4 * N);
            pos[k] = c.take(4 * N);
        }
        counts = c.take(((size_t)4 << bits) * blocks);
        totals = c.take((size_t)4 << bits);
        starts = c.take(4 * (V + 1));
        tally = c.take(8);
        runs = c.take(sizeof(LongRun) * max_runs);
        partial = c.take(sizeof(float) * max_pieces * D);
        bytes = c.used;
    }
};

template <class T> hipError_t embed_grad_t(const EmbedGradArgs &a, hipStream_t s)
{
    const GradPlan p(a.V, a.D, a.N);
    char *ws = (char *)a.ws;
    uint32_t *ids[2], *pos[2];
    for (int k = 0; k < 2; k++) {
        ids[k] = (uint32_t *)(ws + p.ids[k]);
        pos[k] = (uint32_t *)(ws + p.pos[k]);
    }
    uint32_t *counts = (uint32_t *)(ws + p.counts), *totals = (uint32_t *)(ws + p.totals);
    uint32_t *starts = (uint32_t *)(ws + p.starts);
    unsigned long long *tally = (unsigned long long *)(ws + p.tally);
    LongRun *runs = (LongRun *)(ws + p.runs);
    float *partial = (float *)(ws + p.partial);
    const size_t nb = (size_t)1 << p.bits;
    int cur = 0;
    for (int k = 0; k < p.passes; k++) {
        const int shift = k * p.bits;
        const uint32_t *in_ids = k ? ids[cur] : nullptr, *in_pos = k ? pos[cur] : nullptr;
        if (p.blocks) {
            k_sort_count<<<p.blocks, kSortThreads, 4 * nb, s>>>(a.tokens, in_ids, a.N, (uint32_t)a.V, shift, p.bits,
                                                               counts);
            k_sort_scan<<<nb, 64, 0, s>>>(counts, (int)p.blocks, totals);
            k_sort_scatter<<<p.blocks, kSortThreads, 2 * kSortWaves * nb + 4 * nb, s>>>(
                a.tokens, in_ids, in_pos, a.N, (uint32_t)a.V, shift, p.bits, counts, totals, ids[1 - cur],
                pos[1 - cur]);
        }
        cur = 1 - cur;
    }
    k_clear_tally<<<1, 1, 0, s>>>(tally);
    k_embed_runs<<<(a.V + kThreads) / kThreads, kThreads, 0, s>>>(ids[cur], a.N, a.V, p.piece, starts, tally, runs);
    const int64_t chunks = (a.D + kVec<T> - 1) / kVec<T>;
    const int pb = (int)(p.max_pieces < 2048 ? p.max_pieces : 2048);
    auto go = [&](auto kernel, int L) {
        const int64_t per = kThreads / L;
        kernel<<<(unsigned)(pb + (a.V + per - 1) / per), kThreads, 0, s>>>(a, pos[cur], starts, tally, runs, partial,
                                                                          p.piece, pb);
    };
    if (chunks <= 8) go(k_embed_sums<T, 8>, 8);
    else if (chunks <= 16) go(k_embed_sums<T, 16>, 16);
    else if (chunks <= 32) go(k_embed_sums<T, 32>, 32);
    else go(k_embed_sums<T, 64>, 64);
    if (p.max_runs) {
        const dim3 grid((unsigned)(p.max_runs < 256 ? p.max_runs : 256), (unsigned)((a.D + 63) / 64));
        k_embed_join<T><<<grid, kJoinWaves * 64, 0, s>>>(a, tally, runs, partial, p.piece);
    }
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
