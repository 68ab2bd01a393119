// seq_norm.hip -- layer norm of rows and its gradients.
//
// Bound by memory: the forward pass reads x and writes y, the backward pass
// reads x and dy and writes dx.  A row stays in the registers of the lanes that
// share it, so the mean, the variance about it and the output take one read.
// The backward pass walks many rows per wavefront and keeps the sums for
// dweight and dbias in registers over all of them; what is left is one row of
// partial sums per workgroup, added up by a second small kernel.
#include <algorithm>
#include <type_traits>

#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

// A row is shared by L lanes (L <= 64: several rows per wavefront; else a whole
// workgroup of L threads), each holding C chunks of 16 bytes, L chunks apart.
template <int L> constexpr int kThreadsOf = L > 64 ? L : 256;

// Sum over the L lanes of a row.  With L > 64 all threads of the workgroup take
// part, through `red`, which alternates between two halves by `turn`, so that
// one barrier per sum is enough.
template <int L> __device__ __forceinline__ float row_sum(float v, float (*red)[16], int &turn)
{
    if constexpr (L <= 64) return group_sum<L>(v);
    else {
        constexpr int W = L / 64;
        v = group_sum<64>(v);
        if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; w++) s += red[turn][w];
        turn ^= 1;
        return s;
    }
}

// Which columns a lane holds: C pieces of W elements, L pieces apart.  A piece
// that would go past the row's end is the row's last W columns instead, so
// that every access is whole and no branch stands between the reads; the
// columns it shares with the lane before it count there alone, and are formed
// and written twice.  W is one 16-byte piece, or 1 for rows shorter than that.
template <int L, int C, int W> struct Columns {
    int64_t at[C];
    int skip[C];  // elements that do not count here (W: the lane has none)
    __device__ explicit Columns(int64_t D)
    {
        const int lane = threadIdx.x % L;
#pragma unroll
        for (int c = 0; c < C; c++) {
            const int64_t nominal = (int64_t)(c * L + lane) * W;
            at[c] = min(nominal, D - W);
            skip[c] = (int)min(nominal - at[c], (int64_t)W);
        }
    }
    // v where element j of piece c counts, else 0
    __device__ float count(int c, int j, float v) const { return j >= skip[c] ? v : 0.f; }
};

template <class T, int C, int W> struct Pieces {
    T v[C][W];
    template <class Cols> __device__ __forceinline__ void load(const T *row, const Cols &k)
    {
#pragma unroll
        for (int c = 0; c < C; c++) __builtin_memcpy(v[c], row + k.at[c], sizeof v[c]);
    }
};

// Workgroups walk the rows, the weights in registers, the next row's reads on
// their way while a row is worked on.  65536 x 1024 bf16: 49 us, 5.5 TB/s.
template <class T, int L, int C, int W> __global__ __launch_bounds__(kThreadsOf<L>) void k_norm(NormArgs a)
{
    constexpr int R = kThreadsOf<L> / L;
    __shared__ float red[2][16];
    int turn = 0;
    const Columns<L, C, W> k(a.D);
    const int lane = threadIdx.x % L;
    float w[C][W], b[C][W];
#pragma unroll
    for (int c = 0; c < C; c++) {
        load_vec<W>((const T *)a.weight + k.at[c], w[c]);
#pragma unroll
        for (int j = 0; j < W; j++) b[c][j] = 0.f;
        if (a.bias) load_vec<W>((const T *)a.bias + k.at[c], b[c]);
    }
    const float inv = 1.f / (float)a.D;
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L;
    Pieces<T, C, W> x;
    x.load((const T *)a.x + min(row, a.N - 1) * a.ld_x, k);
    // all threads of a workgroup take the same number of turns
    for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < a.N; r0 += step, row += step) {
        float f[C][W], s = 0.f, q = 0.f;
#pragma unroll
        for (int c = 0; c < C; c++)
#pragma unroll
            for (int j = 0; j < W; j++) {
                f[c][j] = (float)x.v[c][j];
                s += k.count(c, j, f[c][j]);
            }
        if (r0 + step < a.N) x.load((const T *)a.x + min(row + step, a.N - 1) * a.ld_x, k);
        const float mean = row_sum<L>(s, red, turn) * inv;
#pragma unroll
        for (int c = 0; c < C; c++)
#pragma unroll
            for (int j = 0; j < W; j++) {
                f[c][j] -= mean;
                q += k.count(c, j, f[c][j] * f[c][j]);
            }
        const float rstd = 1.f / sqrtf(row_sum<L>(q, red, turn) * inv + a.eps);
        if (row >= a.N) continue;
        if (a.mean && lane == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        T *y = (T *)a.y + row * a.ld_y;
#pragma unroll
        for (int c = 0; c < C; c++) {
#pragma unroll
            for (int j = 0; j < W; j++) f[c][j] = fmaf(f[c][j] * rstd, w[c][j], b[c][j]);
            if (k.skip[c] < W) store_vec<W>(y + k.at[c], f[c]);
        }
    }
}

// Rows too wide for registers: a workgroup reads its row three times, the
// second and third time from the caches.  1000 x 100003 bf16: 171 us.
constexpr int kWide = 1024;
template <class T> __global__ __launch_bounds__(kWide) void k_norm_wide(NormArgs a)
{
    constexpr int VE = kVec<T>;
    __shared__ float red[2][16];
    int turn = 0;
    const int64_t row = block_of();
    if (row >= a.N) return;
    const T *x = (const T *)a.x + row * a.ld_x;
    float s = 0.f, q = 0.f;
    for (int64_t at = (int64_t)threadIdx.x * VE; at < a.D; at += kWide * VE) {
        float f[VE];
        load_part<VE>(x + at, (int)min((int64_t)VE, a.D - at), f);
#pragma unroll
        for (int j = 0; j < VE; j++) s += f[j];
    }
    const float mean = row_sum<kWide>(s, red, turn) / (float)a.D;
    for (int64_t at = (int64_t)threadIdx.x * VE; at < a.D; at += kWide * VE) {
        float f[VE];
        const int n = (int)min((int64_t)VE, a.D - at);
        load_part<VE>(x + at, n, f);
#pragma unroll
        for (int j = 0; j < VE; j++)
            if (j < n) q = fmaf(f[j] - mean, f[j] - mean, q);
    }
    const float rstd = 1.f / sqrtf(row_sum<kWide>(q, red, turn) / (float)a.D + a.eps);
    if (a.mean && threadIdx.x == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
    T *y = (T *)a.y + row * a.ld_y;
    for (int64_t at = (int64_t)threadIdx.x * VE; at < a.D; at += kWide * VE) {
        const int n = (int)min((int64_t)VE, a.D - at);
        float f[VE], w[VE], b[VE] = {};
        load_part<VE>(x + at, n, f);
        load_part<VE>((const T *)a.weight + at, n, w);
        if (a.bias) load_part<VE>((const T *)a.bias + at, n, b);
#pragma unroll
        for (int j = 0; j < VE; j++) f[j] = fmaf((f[j] - mean) * rstd, w[j], b[j]);
        store_part<VE>(y + at, n, f);
    }
}

// ---------------------------------------------------------------- backward
// Workgroup b takes R rows at a time, gridDim.x R apart, and leaves its sums of
// dy xh and dy in part[b][2][D].  65536 x 1024 bf16: 81 us, 5.0 TB/s.
template <class T, int L, int C, int W>
__global__ __launch_bounds__(kThreadsOf<L>) void k_norm_grad(NormArgs a, float *part)
{
    constexpr int R = kThreadsOf<L> / L;
    __shared__ float red[2][16];
    __shared__ float join[R > 1 ? R : 1][R > 1 ? L * W : 1];
    int turn = 0;
    const Columns<L, C, W> k(a.D);
    const int lane = threadIdx.x % L, g = threadIdx.x / L;
    float w[C][W], dw[C][W], db[C][W];
#pragma unroll
    for (int c = 0; c < C; c++) {
        load_vec<W>((const T *)a.weight + k.at[c], w[c]);
#pragma unroll
        for (int j = 0; j < W; j++) dw[c][j] = db[c][j] = 0.f;
    }
    const float inv = 1.f / (float)a.D;
    const int64_t step = (int64_t)gridDim.x * R;
    int64_t row = (int64_t)blockIdx.x * R + g;
    Pieces<T, C, W> x, y;
    float mean, rstd;
    auto fetch = [&](int64_t r) {
        r = min(r, a.N - 1);
        x.load((const T *)a.x + r * a.ld_x, k);
        y.load((const T *)a.dy + r * a.ld_dy, k);
        mean = a.mean_in[r];
        rstd = a.rstd_in[r];
    };
    fetch(row);
    for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < a.N; r0 += step, row += step) {
        const bool in = row < a.N;
        float f[C][W], d[C][W], s1 = 0.f, s2 = 0.f;
        const float rs = rstd;
#pragma unroll
        for (int c = 0; c < C; c++)
#pragma unroll
            for (int j = 0; j < W; j++) {
                f[c][j] = ((float)x.v[c][j] - mean) * rstd;  // xh
                d[c][j] = (float)y.v[c][j];
                if (in) {
                    dw[c][j] = fmaf(d[c][j], f[c][j], dw[c][j]);
                    db[c][j] += d[c][j];
                }
                d[c][j] *= w[c][j];  // u
                const float u = k.count(c, j, d[c][j]);
                s1 += u;
                s2 = fmaf(u, f[c][j], s2);
            }
        if (r0 + step < a.N) fetch(row + step);
        const float m1 = row_sum<L>(s1, red, turn) * inv;
        const float m2 = row_sum<L>(s2, red, turn) * inv;
        if (!in) continue;
        T *dx = (T *)a.dx + row * a.ld_dx;
#pragma unroll
        for (int c = 0; c < C; c++) {
#pragma unroll
            for (int j = 0; j < W; j++) f[c][j] = rs * (d[c][j] - m1 - f[c][j] * m2);
            if (k.skip[c] < W) store_vec<W>(dx + k.at[c], f[c]);
        }
    }
    // one row of sums per workgroup
    float *out = part + (int64_t)blockIdx.x * 2 * a.D;
#pragma unroll
    for (int c = 0; c < C; c++)
#pragma unroll
        for (int t = 0; t < 2; t++) {
            float(&v)[W] = t ? db[c] : dw[c];
            if constexpr (R > 1) {
#pragma unroll
                for (int j = 0; j < W; j++) join[g][lane * W + j] = v[j];
                __syncthreads();
                if (g == 0 && k.skip[c] < W) {
#pragma unroll
                    for (int j = 0; j < W; j++) {
                        v[j] = 0.f;
#pragma unroll
                        for (int r = 0; r < R; r++) v[j] += join[r][lane * W + j];
                    }
                    store_vec<W>(out + t * a.D + k.at[c], v);
                }
                __syncthreads();
            } else if (k.skip[c] < W) store_vec<W>(out + t * a.D + k.at[c], v);
        }
}

// Wide rows: the workgroup's sums lie in its row of `part` from the first row on.
// 1000 x 100003 bf16: 586 us.
template <class T> __global__ __launch_bounds__(kWide) void k_norm_grad_wide(NormArgs a, float *part)
{
    constexpr int VE = kVec<T>;
    __shared__ float red[2][16];
    int turn = 0;
    float *out = part + (int64_t)blockIdx.x * 2 * a.D;
    const float inv = 1.f / (float)a.D;
    bool first = true;
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x, first = false) {
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        const T *x = (const T *)a.x + row * a.ld_x, *dy = (const T *)a.dy + row * a.ld_dy;
        float s1 = 0.f, s2 = 0.f;
        for (int64_t at = (int64_t)threadIdx.x * VE; at < a.D; at += kWide * VE) {
            const int n = (int)min((int64_t)VE, a.D - at);
            float f[VE], d[VE], w[VE], pw[VE] = {}, pb[VE] = {};
            load_part<VE>(x + at, n, f);
            load_part<VE>(dy + at, n, d);
            load_part<VE>((const T *)a.weight + at, n, w);
            if (!first) {
                load_part<VE>(out + at, n, pw);
                load_part<VE>(out + a.D + at, n, pb);
            }
#pragma unroll
            for (int j = 0; j < VE; j++) {
                const float xh = j < n ? (f[j] - mean) * rstd : 0.f;
                pw[j] = fmaf(d[j], xh, pw[j]);
                pb[j] += d[j];
                const float u = d[j] * w[j];
                s1 += u;
                s2 = fmaf(u, xh, s2);
            }
            store_part<VE>(out + at, n, pw);
            store_part<VE>(out + a.D + at, n, pb);
        }
        const float m1 = row_sum<kWide>(s1, red, turn) * inv;
        const float m2 = row_sum<kWide>(s2, red, turn) * inv;
        T *dx = (T *)a.dx + row * a.ld_dx;
        for (int64_t at = (int64_t)threadIdx.x * VE; at < a.D; at += kWide * VE) {
            const int n = (int)min((int64_t)VE, a.D - at);
            float f[VE], d[VE], w[VE];
            load_part<VE>(x + at, n, f);
            load_part<VE>(dy + at, n, d);
            load_part<VE>((const T *)a.weight + at, n, w);
#pragma unroll
            for (int j = 0; j < VE; j++) f[j] = rstd * (d[j] * w[j] - m1 - (f[j] - mean) * rstd * m2);
            store_part<VE>(dx + at, n, f);
        }
    }
}

// dweight and dbias: the sums of the `rows` rows of part, 64 columns of the 2 D
// per workgroup, its wavefronts taking every 16th row.  1024 rows of 2 x 1024: 6 us.
constexpr int kJoinWaves = 16;
template <class T>
__global__ __launch_bounds__(kJoinWaves * 64) void k_norm_join(NormArgs a, const float *part, int rows)
{
    __shared__ float red[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)block_of() * 64 + lane;
    float s = 0.f;
    if (c < 2 * a.D)
#pragma unroll 8
        for (int r = wave; r < rows; r += kJoinWaves) s += part[(int64_t)r * 2 * a.D + c];
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < 2 * a.D) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kJoinWaves; w++) t += red[w][lane];
        if (c < a.D) ((T *)a.dweight)[c] = (T)t;
        else if (a.dbias) ((T *)a.dbias)[c - a.D] = (T)t;
    }
}

// Calls f with the lanes, pieces and elements of a piece for rows of D elements,
// or with 0 lanes for rows wider than the registers of a workgroup take (the
// backward pass holds five times as much per element).  Forward, the widest rows
// in registers against reading them three times: 20000 x 8193 bf16 239 us (334),
// 20000 x 8192 fp32 235 us (321), 2000 x 8192 fp32 33 us (36); a row that takes
// little more than half of the workgroup's pieces loses where the reads are served
// by the last-level cache, 2000 x 4097 fp32 27 us (23).
template <class T, bool BACK, class F> hipError_t by_width(int64_t D, F &&f)
{
#define TQ_ROW(L, C, W)                                                                                                \
    do {                                                                                                               \
        if (D <= (int64_t)(L) * (C) * (W))                                                                             \
            return f(std::integral_constant<int, L>{}, std::integral_constant<int, C>{},                               \
                     std::integral_constant<int, W>{});                                                                \
    } while (0)
    constexpr int VE = kVec<T>;
    if (D < VE) TQ_ROW(8, 1, 1);
    TQ_ROW(8, 1, VE);
    TQ_ROW(16, 1, VE);
    TQ_ROW(32, 1, VE);
    TQ_ROW(64, 1, VE);
    TQ_ROW(64, 2, VE);
    TQ_ROW(64, 3, VE);
    TQ_ROW(64, 4, VE);
    TQ_ROW(256, 2, VE);
    TQ_ROW(256, 4, VE);
    if constexpr (BACK) {
        TQ_ROW(512, 4, VE);
    } else {
        TQ_ROW(1024, 2, VE);
    }
#undef TQ_ROW
    return f(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{});
}

// Workgroups of the forward pass: as many as the chip holds, and more for its
// schedulers to even out.
constexpr int64_t kBlocks = 4096;

// Workgroups of the backward pass of narrow rows: enough to fill the chip several
// times, few enough that their rows of sums are small beside x.  Half and a
// quarter of them for wide rows: 2000 x 8192 bf16 36 us with half, 47 with all.
constexpr int64_t kGradBlocks = 1024;

template <class T> hipError_t norm_t(const NormArgs &a, hipStream_t s)
{
    return by_width<T, false>(a.D, [&](auto l, auto c, auto w) {
        constexpr int L = decltype(l)::value, C = decltype(c)::value, W = decltype(w)::value;
        if constexpr (L == 0) k_norm_wide<T><<<grid_of(a.N), kWide, 0, s>>>(a);
        else {
            constexpr int R = kThreadsOf<L> / L;
            k_norm<T, L, C, W><<<(unsigned)std::min((a.N + R - 1) / R, kBlocks), kThreadsOf<L>, 0, s>>>(a);
        }
        return hipGetLastError();
    });
}

template <class T> hipError_t norm_grad_t(const NormArgs &a, hipStream_t s)
{
    return by_width<T, true>(a.D, [&](auto l, auto c, auto w) {
        constexpr int L = decltype(l)::value, C = decltype(c)::value, W = decltype(w)::value;
        float *part = (float *)a.ws;
        int64_t blocks;
        if constexpr (L == 0) {
            blocks = std::min(a.N, kGradBlocks / 4);
            if (blocks) k_norm_grad_wide<T><<<(unsigned)blocks, kWide, 0, s>>>(a, part);
        } else {
            constexpr int R = kThreadsOf<L> / L;
            blocks = std::min((a.N + R - 1) / R, L > 256 ? kGradBlocks / 4 : L > 64 ? kGradBlocks / 2 : kGradBlocks);
            if (blocks) k_norm_grad<T, L, C, W><<<(unsigned)blocks, kThreadsOf<L>, 0, s>>>(a, part);
        }
        k_norm_join<T><<<grid_of((2 * a.D + 63) / 64), kJoinWaves * 64, 0, s>>>(a, part, (int)blocks);
        return hipGetLastError();
    });
}

} // namespace

size_t norm_grad_workspace(int64_t N, int64_t D)
{
    return sizeof(float) * 2 * (size_t)D * (size_t)std::min(N, kGradBlocks);
}

hipError_t launch_norm(int32_t type, const NormArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return norm_t<float>(a, s);
    if (type == TQ_BF16) return norm_t<__bf16>(a, s);
    return norm_t<_Float16>(a, s);
}

hipError_t launch_norm_grad(int32_t type, const NormArgs &a, hipStream_t s)
{
    if (type == TQ_F32) return norm_grad_t<float>(a, s);
    if (type == TQ_BF16) return norm_grad_t<__bf16>(a, s);
    return norm_grad_t<_Float16>(a, s);
}

} // namespace tq
