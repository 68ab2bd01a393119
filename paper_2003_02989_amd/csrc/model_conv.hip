// model_conv.hip -- the short causal convolution over time and its gradients.
//
//   u_t = bias + sum_k w_k x_{t-K+1+k},   y_t = u_t or silu(u_t),
//
// channel by channel, the K - 1 inputs before the first step being the record's
// state.  Bound by memory: x is read and y written once.  A thread holds a piece of
// a row over a run of steps, the last K - 1 inputs in registers, the next batch of
// steps on its way while one is worked on.  A piece is 16 bytes (16 x 2048 x 2112 bf16,
// 4 taps: 63 us, 4.4 TB/s); for the gradient, which holds more per element, 2 elements:
// forward and gradient of 8 x 1024 x 512 fp32 31 us, with 4 elements 36, and 16-bit
// ones with 4 do not fit the registers that four wavefronts per SIMD have.
//
// The gradient walks a run forwards, forms u again and with it g_t = dy_t silu'(u_t);
//   dx_t = sum_k w_k g_{t+K-1-k}
// follows K - 1 steps behind, so that a run ends with g of the K - 1 steps past its
// end, formed a second time.  A state's gradient is dx of the steps before the first.
// dw_k = sum g_t x_{t-K+1+k} and dbias = sum g_t stay in registers over all runs of a
// thread; a second kernel adds the threads' sums in order.
#include <algorithm>
#include <type_traits>

#include "model_device.h"
#include "seq.h"

namespace tq {
namespace {

// steps that are read together
constexpr int kBatch = 8, kGradBatch = 4;
constexpr int kLeast = 8;   // steps of a run at least: K - 1 and more

struct Geom {
    uint32_t items;   // threads with work
    uint32_t pieces;  // of a row
    uint32_t runs;    // of a record
    uint32_t rows;    // gradient: rows of sums, each of runs a stride of `rows` apart
    int64_t run;      // steps of a run, whole batches
    float *part;      // [rows][K + 1][D]
};

// A thread's piece of a row: the last one ends with the row, the elements that it
// shares with the one before belong to that.
template <int V> struct Piece {
    int64_t c;
    int skip;
    __device__ Piece(uint32_t piece, int64_t D)
    {
        const int64_t nominal = (int64_t)piece * V;
        c = min(nominal, D - V);
        skip = (int)(nominal - c);
    }
    template <class T> __device__ __forceinline__ void store(T *row, const float (&f)[V]) const
    {
        if (skip == 0) {
            store_vec<V>(row + c, f);
            return;
        }
#pragma unroll
        for (int j = 0; j < V; j++)
            if (j >= skip) row[c + j] = (T)f[j];
    }
};

template <class T, int V> struct Raw {
    T v[V];
    __device__ __forceinline__ void load(const T *p) { __builtin_memcpy(v, p, sizeof v); }
};

template <class T> __device__ __forceinline__ const T *row_of(const Steps &s, int64_t b, int64_t t)
{
    return (const T *)s.p + b * s.batch + t * s.step;
}
template <class T> __device__ __forceinline__ T *row_of(const StepsOut &s, int64_t b, int64_t t)
{
    return (T *)s.p + b * s.batch + t * s.step;
}

template <class T, int V, int K, int N> __global__ __launch_bounds__(256) void k_conv(ConvArgs a, Geom g)
{
    const uint32_t item = block_of() * 256 + threadIdx.x;
    if (item >= g.items) return;
    const uint32_t row = item / g.pieces, record = row / g.runs, run = row - record * g.runs;
    const Piece<V> at(item - row * g.pieces, a.D);
    const int64_t b = record, t0 = run * g.run, t1 = min(t0 + g.run, a.T);
    const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), a.T) : a.T, n1 = min(t1, len);
    float w[K][V], bias[V], x[N + K - 1][V];
#pragma unroll
    for (int k = 0; k < K; k++) load_vec<V>((const T *)a.weight + k * a.D + at.c, w[k]);
#pragma unroll
    for (int j = 0; j < V; j++) bias[j] = 0.f;
    if (a.bias) load_vec<V>((const T *)a.bias + at.c, bias);
    if (run == 0) {  // runs are longer than the state
        const T *from = (const T *)a.state + b * (K - 1) * a.D + at.c;
#pragma unroll
        for (int k = 0; k + 1 < K; k++) {
#pragma unroll
            for (int j = 0; j < V; j++) x[k][j] = 0.f;
            if (a.state) load_vec<V>(from + k * a.D, x[k]);
        }
        if (a.last) {  // inputs n .. n + K - 2 of the state and the record, all read before the first is written
            Raw<T, V> end[K];
#pragma unroll
            for (int k = 0; k + 1 < K; k++) {
                const int64_t i = len + k;
#pragma unroll
                for (int m = 0; m + 1 < K; m++)
                    if (i == m)
#pragma unroll
                        for (int j = 0; j < V; j++) end[k].v[j] = (T)x[m][j];
                if (i >= K - 1) end[k].load(row_of<T>(a.x, b, i - (K - 1)) + at.c);
            }
#pragma unroll
            for (int k = 0; k + 1 < K; k++) {
                float f[V];
#pragma unroll
                for (int j = 0; j < V; j++) f[j] = (float)end[k].v[j];
                at.store((T *)a.last + (b * (K - 1) + k) * a.D, f);
            }
        }
    } else if (t0 < len) {
#pragma unroll
        for (int k = 0; k + 1 < K; k++) load_vec<V>(row_of<T>(a.x, b, t0 - (K - 1) + k) + at.c, x[k]);
    }
    Raw<T, V> in[N];
    const auto fetch = [&](int64_t t) {
#pragma unroll
        for (int i = 0; i < N; i++) in[i].load(row_of<T>(a.x, b, min(t + i, n1 - 1)) + at.c);
    };
    if (t0 < n1) fetch(t0);
    for (int64_t t = t0; t < n1; t += N) {
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
            for (int j = 0; j < V; j++) x[K - 1 + i][j] = (float)in[i].v[j];
        if (t + N < n1) fetch(t + N);  // on its way meanwhile
#pragma unroll
        for (int i = 0; i < N; i++) {
            if (t + i >= n1) break;
            float y[V];
#pragma unroll
            for (int j = 0; j < V; j++) {
                float u = bias[j];
#pragma unroll
                for (int k = 0; k < K; k++) u = fmaf(w[k][j], x[i + k][j], u);
                y[j] = a.silu ? u * sigmoid<T>(u) : u;
            }
            at.store(row_of<T>(a.y, b, t + i), y);
        }
#pragma unroll
        for (int k = 0; k + 1 < K; k++)
#pragma unroll
            for (int j = 0; j < V; j++) x[k][j] = x[N + k][j];
    }
    const float none[V] = {};
    for (int64_t t = max(t0, len); t < t1; t++) at.store(row_of<T>(a.y, b, t), none);
}

// (four wavefronts per SIMD where the registers of 16-bit rows and few taps allow it)
template <class T, int V, int K>
__global__ __launch_bounds__(256, sizeof(T) == 2 && K <= 4 ? 4 : 2) void k_conv_grad(ConvArgs a, Geom g)
{
    const uint32_t item = block_of() * 256 + threadIdx.x;
    if (item >= g.items) return;
    const uint32_t first = item / g.pieces;
    const Piece<V> at(item - first * g.pieces, a.D);
    float w[K][V], bias[V], dw[K][V], db[V];
#pragma unroll
    for (int j = 0; j < V; j++) bias[j] = db[j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; k++) {
        load_vec<V>((const T *)a.weight + k * a.D + at.c, w[k]);
#pragma unroll
        for (int j = 0; j < V; j++) dw[k][j] = 0.f;
    }
    if (a.bias) load_vec<V>((const T *)a.bias + at.c, bias);
    for (uint32_t row = first; row < (uint32_t)(a.B * g.runs); row += g.rows) {
        const uint32_t record = row / g.runs, run = row - record * g.runs;
        const int64_t b = record, t0 = run * g.run, t1 = min(t0 + g.run, a.T);
        const int64_t len = a.lengths ? min(max((int64_t)a.lengths[b], (int64_t)0), a.T) : a.T, n1 = min(t1, len);
        const float none[V] = {};
        for (int64_t t = max(t0, len); t < t1; t++) store_vec<V>(row_of<T>(a.dx, b, t) + at.c, none);
        if (t0 >= len && run > 0) continue;
        // what comes back from the state after the record: to its last K - 1 inputs
        const auto returned = [&](int64_t t, float (&f)[V]) {
            const int64_t i = t - len + K - 1;
            if (a.dlast && i >= 0) {
                float d[V];
                load_vec<V>((const T *)a.dlast + (b * (K - 1) + i) * a.D + at.c, d);
#pragma unroll
                for (int j = 0; j < V; j++) f[j] += d[j];
            }
        };
        float x[kGradBatch + K - 1][V], q[kGradBatch + K - 1][V];
#pragma unroll
        for (int k = 0; k + 1 < K; k++) {
#pragma unroll
            for (int j = 0; j < V; j++) x[k][j] = q[k][j] = 0.f;
            if (run > 0) load_vec<V>(row_of<T>(a.x, b, t0 - (K - 1) + k) + at.c, x[k]);
            else if (a.state) load_vec<V>((const T *)a.state + (b * (K - 1) + k) * a.D + at.c, x[k]);
        }
        Raw<T, V> in[kGradBatch], up[kGradBatch];
        // the rows of the next read, and of the step that a batch begins with
        const T *px = row_of<T>(a.x, b, t0) + at.c, *pdy = row_of<T>(a.dy, b, t0) + at.c;
        T *pdx = row_of<T>(a.dx, b, t0) + at.c;
        const auto fetch = [&](int64_t t) {
            const int left = (int)min(len - 1 - t, (int64_t)kGradBatch);  // the last step there is
            if (__ballot(left < kGradBatch - 1) == 0) {
#pragma unroll
                for (int i = 0; i < kGradBatch; i++) {
                    in[i].load(px + i * a.x.step);
                    up[i].load(pdy + i * a.dy.step);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kGradBatch; i++) {
                    in[i].load(px + min(i, left) * a.x.step);
                    up[i].load(pdy + min(i, left) * a.dy.step);
                }
            }
            px += kGradBatch * a.x.step;
            pdy += kGradBatch * a.dy.step;
        };
        // A batch of steps from t on; `whole`: all of the run's, and so are those whose
        // dx they complete, none of which the state after the record holds.  (A row's last
        // piece is stored whole: what it shares with the one before is the same in both.)
        const auto batch = [&](int64_t t, auto whole) {
            constexpr bool kWhole = decltype(whole)::value;
#pragma unroll
            for (int i = 0; i < kGradBatch; i++) {
#pragma unroll
                for (int j = 0; j < V; j++) {
                    float &d = q[K - 1 + i][j];
                    if (a.silu) {
                        float u = bias[j];
#pragma unroll
                        for (int k = 0; k < K; k++) u = fmaf(w[k][j], x[i + k][j], u);
                        const float s = sigmoid<T>(u);
                        d *= s * fmaf(u, 1.f - s, 1.f);
                    }
                    if (!kWhole && t + i >= len) d = 0.f;
                    if (kWhole || t + i < n1) {
                        db[j] += d;
#pragma unroll
                        for (int k = 0; k < K; k++) dw[k][j] = fmaf(d, x[i + k][j], dw[k][j]);
                    }
                }
                const int64_t o = t + i - (K - 1);  // the step whose dx is known now
                if (!kWhole && !(o < n1 && (o >= t0 || (run == 0 && o < 0 && a.dstate)))) continue;
                float f[V];
#pragma unroll
                for (int j = 0; j < V; j++) {
                    f[j] = 0.f;
#pragma unroll
                    for (int k = 0; k < K; k++) f[j] = fmaf(w[k][j], q[i + K - 1 - k][j], f[j]);
                }
                if (!kWhole) returned(o, f);
                if (kWhole || o >= 0) store_vec<V>(pdx + (i - (K - 1)) * a.dx.step, f);
                else store_vec<V>((T *)a.dstate + (b * (K - 1) + o + K - 1) * a.D + at.c, f);
            }
            pdx += kGradBatch * a.dx.step;
        };
        if (t0 < len) fetch(t0);
        // dx of the K - 1 steps before a step follow from it: on to K - 1 past the end
        for (int64_t t = t0; t < n1 + K - 1; t += kGradBatch) {
            if (t < len) {
#pragma unroll
                for (int i = 0; i < kGradBatch; i++)
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        x[K - 1 + i][j] = (float)in[i].v[j];
                        q[K - 1 + i][j] = (float)up[i].v[j];
                    }
                if (t + kGradBatch < min(n1 + K - 1, len)) fetch(t + kGradBatch);  // on its way meanwhile
            }
            if (t >= t0 + K - 1 && t + kGradBatch <= n1) batch(t, std::true_type{});
            else batch(t, std::false_type{});
#pragma unroll
            for (int k = 0; k + 1 < K; k++)
#pragma unroll
                for (int j = 0; j < V; j++) {
                    x[k][j] = x[kGradBatch + k][j];
                    q[k][j] = q[kGradBatch + k][j];
                }
        }
    }
    float *out = g.part + (int64_t)first * (K + 1) * a.D;
#pragma unroll
    for (int k = 0; k < K; k++) store_vec<V>(out + k * a.D + at.c, dw[k]);
    store_vec<V>(out + K * a.D + at.c, db);
}

// dweight and dbias: the rows' sums in order, 16 of the (K + 1) D columns per
// workgroup, its 64 groups of 16 lanes taking every 64th row.
constexpr int kJoin = 64, kColumns = 16;
template <class T> __global__ __launch_bounds__(kJoin * kColumns) void k_conv_join(ConvArgs a, Geom g)
{
    __shared__ float red[kJoin][kColumns + 1];
    const int lane = threadIdx.x % kColumns, group = threadIdx.x / kColumns;
    const int64_t c = (int64_t)block_of() * kColumns + lane, columns = (a.K + 1) * a.D;
    float s = 0.f;
    if (c < columns)
#pragma unroll 8
        for (uint32_t r = group; r < g.rows; r += kJoin) s += g.part[r * columns + c];
    red[group][lane] = s;
    __syncthreads();
#pragma unroll
    for (int n = kJoin / 2; n > 0; n /= 2) {
        if (group < n) red[group][lane] += red[group + n][lane];
        __syncthreads();
    }
    if (group || c >= columns) return;
    s = red[0][lane];
    if (c < a.K * a.D) ((T *)a.dweight)[c] = (T)s;
    else if (a.dbias) ((T *)a.dbias)[c - a.K * a.D] = (T)s;
}

template <class T, bool GRAD> constexpr int kPiece = GRAD ? 2 : kVec<T>;

// Steps of a run: as many as leave threads enough to fill the chip; each reads the K - 1
// steps before it once more, and the gradient those behind.
Geom geom_of(const ConvArgs &a, int V, bool grad)
{
    Geom g{};
    g.pieces = (uint32_t)((a.D + V - 1) / V);
    const double threads = grad ? 256 * 512 : 256 * 1024;
    g.run = 64;
    while (g.run > kLeast && (double)a.B * (double)((a.T + g.run - 1) / g.run) * g.pieces < threads) g.run /= 2;
    g.runs = (uint32_t)std::max<int64_t>(1, (a.T + g.run - 1) / g.run);
    g.rows = (uint32_t)(a.B * g.runs);
    // records of different lengths are evened out by more rows of fewer runs
    const int64_t most = a.lengths ? 256 * 2048 : 256 * 1024;
    if (grad) g.rows = (uint32_t)std::min<int64_t>(g.rows, std::max<int64_t>(1, most / g.pieces));
    g.items = g.rows * g.pieces;
    return g;
}

template <class F> hipError_t by_taps(int K, F &&f)
{
    switch (K) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
    }
}

// Elements of a piece; rows without a whole one: one element each.
int piece_of(int32_t type, int64_t D, bool grad)
{
    const int v = grad ? 2 : type == TQ_F32 ? 4 : 8;
    return D < v ? 1 : v;
}

template <class T> hipError_t conv_t(const ConvArgs &a, int V, hipStream_t s)
{
    const Geom g = geom_of(a, V, false);
    const dim3 grid = grid_of(((int64_t)g.items + 255) / 256);
    return by_taps((int)a.K, [&](auto k) {
        constexpr int K = decltype(k)::value;
        if (V == 1) k_conv<T, 1, K, kBatch><<<grid, 256, 0, s>>>(a, g);
        else if (a.T == 1) k_conv<T, kPiece<T, false>, K, 1><<<grid, 256, 0, s>>>(a, g);
        else k_conv<T, kPiece<T, false>, K, kBatch><<<grid, 256, 0, s>>>(a, g);
        return hipGetLastError();
    });
}

template <class T> hipError_t conv_grad_t(const ConvArgs &a, int V, hipStream_t s)
{
    Geom g = geom_of(a, V, true);
    g.part = (float *)a.ws;
    const dim3 grid = grid_of(((int64_t)g.items + 255) / 256);
    const hipError_t e = by_taps((int)a.K, [&](auto k) {
        constexpr int K = decltype(k)::value;
        if (g.items == 0) return hipSuccess;
        if (V == 1) k_conv_grad<T, 1, K><<<grid, 256, 0, s>>>(a, g);
        else k_conv_grad<T, kPiece<T, true>, K><<<grid, 256, 0, s>>>(a, g);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    k_conv_join<T><<<grid_of(((a.K + 1) * a.D + kColumns - 1) / kColumns), kJoin * kColumns, 0, s>>>(a, g);
    return hipGetLastError();
}

} // namespace

int64_t conv_items(int64_t B, int64_t T, int64_t D)
{
    const double n = (double)B * (double)((T + kLeast - 1) / kLeast) *
                     (double)(D < 8 ? D : (D + 3) / 4);
    return n > 1e15 ? (int64_t)1e15 : (int64_t)n;
}

size_t conv_grad_workspace(int64_t B, int64_t T, int64_t D, int64_t K)
{
    static const int32_t some = 0;
    ConvArgs a{};
    a.B = B, a.T = T, a.D = D, a.K = K, a.lengths = &some;  // at most
    return sizeof(float) * geom_of(a, piece_of(TQ_F32, D, true), true).rows * (size_t)(K + 1) * (size_t)D;
}

hipError_t launch_conv(int32_t type, const ConvArgs &a, hipStream_t s)
{
    const int V = piece_of(type, a.D, false);
    if (type == TQ_F32) return conv_t<float>(a, V, s);
    if (type == TQ_BF16) return conv_t<__bf16>(a, V, s);
    return conv_t<_Float16>(a, V, s);
}

hipError_t launch_conv_grad(int32_t type, const ConvArgs &a, hipStream_t s)
{
    const int V = piece_of(type, a.D, true);
    if (type == TQ_F32) return conv_grad_t<float>(a, V, s);
    if (type == TQ_BF16) return conv_grad_t<__bf16>(a, V, s);
    return conv_grad_t<_Float16>(a, V, s);
}

} // namespace tq
