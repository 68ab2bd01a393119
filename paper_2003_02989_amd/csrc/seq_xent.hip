// seq_xent.hip -- softmax cross entropy over a vocabulary, and its gradients.
//
//   z = hidden weight^T [N, V],  lse_i = log sum_v exp z_iv,
//   loss_i = lse_i - z_{i, t_i};   p = softmax(z) - onehot(t),
//   dhidden = diag(up) p weight,   dweight = (diag(up) p)^T hidden.
//
// Bound by the matrix products (2 N V D operations each): they run on the
// matrix cores in 16 bits with fp32 sums, in one kernel for products of two
// operands whose rows run along the summed axis (C = A B^T).  The logits are never
// stored: the forward product's epilogue turns each tile of 256 (or 128) words
// by as many tokens into one maximum and one sum of exponentials per token.  For the
// gradient the vocabulary is taken in pieces; a piece's logits are formed a
// second time, now with lse known, and its p is stored in 16 bits twice, along
// the vocabulary for dhidden and along the tokens for dweight.
//
// 16-bit inputs enter the products as they are.  fp32 inputs enter as two
// 16-bit (f16) numbers each, h + l with l the rounding error of h, after a
// power-of-two scale per row: a b = h_a h_b + h_a l_b + l_a h_b leaves out
// l_a l_b, 2^-22 of the product, and costs three products; fp32 matrix
// instructions would cost sixteen times the 16-bit ones.
#include <algorithm>
#include <type_traits>

#include "seq.h"
#include "seq_device.h"

namespace tq {
namespace {

using f32x16 = __attribute__((__vector_size__(16 * sizeof(float)))) float;
using f32x4 = __attribute__((__vector_size__(4 * sizeof(float)))) float;
template <class T> struct Frag {
    typedef T type __attribute__((ext_vector_type(8)));
};
template <class T> using frag = typename Frag<T>::type;

__device__ __forceinline__ f32x16 mfma32(frag<__bf16> a, frag<__bf16> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(frag<_Float16> a, frag<_Float16> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// p is held as p 2^15 in 16 bits: |p| <= 1 fits f16, whose small numbers would
// otherwise not reach the probabilities of a large vocabulary.
constexpr float kProbScale = 32768.f;

// ------------------------------------------------------------ C = A B^T
// A [M, K] and B [N, K] of 16-bit elements, K a multiple of kBK, rows 16-byte
// aligned.  fp32 operands have two parts each, `a_part` / `b_part` elements
// apart: `terms` products A[pa] B[pb]^T are summed.
constexpr int kBK = 64;

struct Operand {
    const void *p;
    int64_t ld, part;
    int64_t rows;
};

struct ProductArgs {
    Operand a, b;
    int terms;     // 1, or 3 for operands in two parts
    int k_tiles;   // K / kBK
    int splits;    // the K axis is cut into this many parts, one slab of C each
    int m_tiles, n_tiles;
};

// Tile of C, wavefronts WM x WN, each with FM x FN blocks of 32 x 32.
template <int WM_, int WN_, int FM_, int FN_> struct Shape {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    static constexpr int waves = WM * WN, threads = waves * 64;
};
using Big = Shape<2, 4, 4, 2>;    // 256 x 256
using Small = Shape<2, 2, 2, 2>;  // 128 x 128

// Where an element of a wavefront's block lies: C row (within 32) of register i
// of a lane; its column is lane % 32.
__device__ __forceinline__ int block_row(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// One stage of the tile in LDS: rows of kBK elements (eight 16-byte pieces), the
// pieces of row r in the order piece ^ (r % 8), so that 32 lanes reading one piece
// of 32 rows meet all banks.  Read straight from global memory into LDS: a
// wavefront's 64 lanes fill eight rows.
template <class T, int ROWS, int WAVES>
__device__ __forceinline__ void stage(T *lds, const T *src, int64_t ld, int64_t row0, int64_t rows, int wave, int lane)
{
#pragma unroll
    for (int i = 0; i < ROWS / 8 / WAVES; i++) {
        const int r8 = (i * WAVES + wave) * 8;
        const int r = r8 + (lane >> 3);
        // rows past the end repeat the last one: read, never used
        const int64_t row = min(row0 + r, rows - 1);
        const T *g = src + row * ld + ((lane & 7) ^ (lane >> 3)) * 8;
        __builtin_amdgcn_global_load_lds((global_void *)g, (lds_void *)(lds + r8 * kBK), 16, 0, 0);
    }
}

template <class T> __device__ __forceinline__ frag<T> read_frag(const T *lds, int row, int piece)
{
    return *(const frag<T> *)(lds + row * kBK + ((piece ^ (row & 7)) * 8));
}

// The tile's sums over this workgroup's part of K.
template <class T, class S>
__device__ __forceinline__ void product(const ProductArgs &a, int64_t m0, int64_t n0, int split,
                                        f32x16 (&acc)[S::FM][S::FN])
{
    __shared__ alignas(1024) T A0[S::BM * kBK], B0[S::BN * kBK], A1[S::BM * kBK], B1[S::BN * kBK];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
#pragma unroll
    for (int i = 0; i < S::FM; i++)
#pragma unroll
        for (int j = 0; j < S::FN; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;
    const int all = a.terms * a.k_tiles;
    const int k0 = (int)((int64_t)all * split / a.splits), k1 = (int)((int64_t)all * (split + 1) / a.splits);
    auto fetch = [&](int kt, T *la, T *lb) {
        // the small terms first: l_a h_b, h_a l_b, h_a h_b
        const int term = kt / a.k_tiles, k = kt - term * a.k_tiles;
        const bool low_a = a.terms == 3 && term == 0, low_b = a.terms == 3 && term == 1;
        const T *ga = (const T *)a.a.p + (low_a ? a.a.part : 0) + (int64_t)k * kBK;
        const T *gb = (const T *)a.b.p + (low_b ? a.b.part : 0) + (int64_t)k * kBK;
        stage<T, S::BM, S::waves>(la, ga, a.a.ld, m0, a.a.rows, wave, lane);
        stage<T, S::BN, S::waves>(lb, gb, a.b.ld, n0, a.b.rows, wave, lane);
    };
    auto compute = [&](const T *la, const T *lb) {
#pragma unroll
        for (int ks = 0; ks < kBK / 16; ks++) {
            frag<T> fa[S::FM], fb[S::FN];
            const int piece = ks * 2 + (lane >> 5);
#pragma unroll
            for (int i = 0; i < S::FM; i++) fa[i] = read_frag<T>(la, wm + i * 32 + (lane & 31), piece);
#pragma unroll
            for (int j = 0; j < S::FN; j++) fb[j] = read_frag<T>(lb, wn + j * 32 + (lane & 31), piece);
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int j = 0; j < S::FN; j++) acc[i][j] = mfma32(fa[i], fb[j], acc[i][j]);
        }
    };
    if (k0 < k1) fetch(k0, A0, B0);
    __syncthreads();
    for (int kt = k0; kt < k1; kt += 2) {
        if (kt + 1 < k1) fetch(kt + 1, A1, B1);
        compute(A0, B0);
        __syncthreads();
        if (kt + 1 < k1) {
            if (kt + 2 < k1) fetch(kt + 2, A0, B0);
            compute(A1, B1);
            __syncthreads();
        }
    }
}

// Which tile a workgroup takes.  Workgroups go round the eight XCDs in turn, so
// that consecutive tiles of one XCD, which share rows of A and B in its L2, are
// eight workgroups apart; within an XCD's share tiles run down kGroup tile rows
// before the next tile column.
constexpr int kXcds = 8, kGroup = 4;
struct Tile {
    int64_t m, n;
    int split;
};
__device__ __forceinline__ Tile tile_of(const ProductArgs &a)
{
    const int tiles = a.m_tiles * a.n_tiles, all = tiles * a.splits;
    const int blk = blockIdx.x;
    const int per = all / kXcds, more = all % kXcds, xcd = blk % kXcds, at = blk / kXcds;
    int id = xcd * per + min(xcd, more) + at;
    Tile t;
    t.split = id / tiles;
    id -= t.split * tiles;
    const int band = kGroup * a.n_tiles, g = id / band, rows = min(kGroup, a.m_tiles - g * kGroup);
    const int in = id - g * band;
    t.m = g * kGroup + in % rows;
    t.n = in / rows;
    return t;
}

// ------------------------------------------------------------ the logits
// A = weight (rows: words), B = hidden (rows: tokens): a lane's registers hold
// words of one token, so that sums over words stay within a lane until the end.
struct LogitArgs {
    ProductArgs p;
    const float *word_scale, *token_scale;  // of fp32 operands, else NULL
    const uint64_t *targets;
    int64_t V, N;
    int64_t v_base;        // first word of the piece (p.a.p points there)
    float2 *part;          // [N, tiles]: maximum, sum of exponentials
    float *z_target;       // [N]
    const float *lse, *up, *up_max;
    void *prob, *prob_t;   // [N, words] and [words, N] of the piece
    int64_t ld_prob, ld_prob_t, prob_part, prob_t_part;
};

template <class T, class S, bool GRAD, bool TWO> __global__ __launch_bounds__(S::threads) void k_logits(LogitArgs a)
{
    const Tile t = tile_of(a.p);
    f32x16 acc[S::FM][S::FN];
    const int64_t m0 = t.m * S::BM, n0 = t.n * S::BN;
    product<T, S>(a.p, m0, n0, 0, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
    const int64_t words = a.p.a.rows;  // of the piece
    if constexpr (!GRAD) {
        __shared__ float2 join[S::WM][S::BN];
#pragma unroll
        for (int j = 0; j < S::FN; j++) {
            const int64_t n = n0 + wn + j * 32 + (lane & 31);
            const float ts = TWO && n < a.N ? a.token_scale[n] : 1.f;
            const uint64_t target = n < a.N ? a.targets[n] : ~(uint64_t)0;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const int64_t v = m0 + wm + i * 32 + block_row(e, lane);
                    float z = acc[i][j][e];
                    if (TWO) z *= ts * (v < words ? a.word_scale[v] : 0.f);
                    if (v >= words) z = -INFINITY;
                    else if ((uint64_t)v == target) a.z_target[n] = z;
                    acc[i][j][e] = z;
                    top = fmaxf(top, z);
                }
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            // without words there is nothing to add; NaN stays in the sum
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int e = 0; e < 16; e++) sum += __expf(acc[i][j][e] - ref);
            sum += __shfl_xor(sum, 32, 64);
            if (lane < 32) join[wave / S::WN][wn + j * 32 + lane] = make_float2(top, sum);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < S::BN; c += S::threads) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < S::WM; w++) top = fmaxf(top, join[w][c].x);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < S::WM; w++) sum += join[w][c].y * __expf(join[w][c].x - ref);
            if (n0 + c < a.N) a.part[(n0 + c) * a.p.m_tiles + t.m] = make_float2(top, sum);
        }
    } else {
        const float up_inv = 1.f / *a.up_max;
#pragma unroll
        for (int j = 0; j < S::FN; j++) {
            const int64_t n = n0 + wn + j * 32 + (lane & 31);
            const bool in = n < a.N;
            const float ts = TWO && in ? a.token_scale[n] : 1.f;
            const uint64_t target = in ? a.targets[n] : ~(uint64_t)0;
            const bool on = target < (uint64_t)a.V;
            const float lse = on ? a.lse[n] : 0.f;
            const float share = on ? a.up[n] * up_inv : 0.f;
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    // four words in a row
                    const int64_t v = m0 + wm + i * 32 + block_row(4 * q, lane);
                    T hi[4], lo[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        float z = acc[i][j][4 * q + e];
                        if (TWO) z *= ts * (v + e < words ? a.word_scale[v + e] : 0.f);
                        float p = __expf(z - lse);
                        if ((uint64_t)(a.v_base + v + e) == target) p -= 1.f;
                        p = on && v + e < words ? p * kProbScale : 0.f;
                        hi[e] = (T)p;
                        if (TWO) lo[e] = (T)(p - (float)hi[e]);
                        const float pt = p * share;
                        if (n < a.ld_prob_t && v + e < words) {
                            T *o = (T *)a.prob_t + (v + e) * a.ld_prob_t + n;
                            const T ht = (T)pt;
                            o[0] = ht;
                            if (TWO) o[a.prob_t_part] = (T)(pt - (float)ht);
                        }
                    }
                    if (in && v < a.ld_prob) {
                        T *o = (T *)a.prob + n * a.ld_prob + v;
                        __builtin_memcpy(o, hi, sizeof hi);
                        if (TWO) __builtin_memcpy(o + a.prob_part, lo, sizeof lo);
                    }
                }
        }
    }
}

// ------------------------------------------------------------ the products
// out = factor diag(row_factor) C diag(col_scale), or fp32 slabs of C, one per
// split, which later pieces add to and k_finish sums up.
struct StoreArgs {
    ProductArgs p;
    int64_t M, N;
    float *slabs;   // NULL: write `out`
    bool add;       // to what the slabs hold
    void *out;
    int64_t ld_out;
    // of an output row or column; NULL: one
    const float *row_up;        // upstream, where the row has a target
    const uint64_t *targets;
    int64_t V;
    const float *col_max;       // columns of the second operand: scale_of(col_max)
    const float *up_max;
};

// The power of two that brings numbers of magnitude up to m into [2^13, 2^14).
__device__ __forceinline__ float scale_of(float m)
{
    if (!(m > 0.f)) return m == 0.f ? 1.f : m;
    if (m > 3.4e38f) return NAN;
    const int e = max((int)((__float_as_uint(m) >> 23) & 255) - 127, -100);
    return __uint_as_float((uint32_t)(e - 13 + 127) << 23);
}
__device__ __forceinline__ float inverse_of(float scale) { return 1.f / scale; }  // exact: a power of two

__device__ __forceinline__ float row_factor(const StoreArgs &a, int64_t m)
{
    float f = 1.f / kProbScale;
    if (a.row_up) f = a.targets[m] < (uint64_t)a.V ? f * a.row_up[m] : 0.f;
    if (a.up_max) f *= *a.up_max;
    return f;
}
__device__ __forceinline__ float col_factor(const StoreArgs &a, int64_t n)
{
    return a.col_max ? scale_of(a.col_max[n]) : 1.f;
}

template <class T, class S, class Out> __global__ __launch_bounds__(S::threads) void k_product(StoreArgs a)
{
    const Tile t = tile_of(a.p);
    f32x16 acc[S::FM][S::FN];
    const int64_t m0 = t.m * S::BM, n0 = t.n * S::BN;
    product<T, S>(a.p, m0, n0, t.split, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
#pragma unroll
    for (int j = 0; j < S::FN; j++) {
        const int64_t n = n0 + wn + j * 32 + (lane & 31);
        if (n >= a.N) continue;
        const float cf = a.slabs ? 1.f : col_factor(a, n);
#pragma unroll
        for (int i = 0; i < S::FM; i++)
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const int64_t m = m0 + wm + i * 32 + block_row(e, lane);
                if (m >= a.M) continue;
                if (a.slabs) {
                    float *o = a.slabs + ((int64_t)t.split * a.M + m) * a.N + n;
                    *o = a.add ? *o + acc[i][j][e] : acc[i][j][e];
                } else {
                    const float f = row_factor(a, m);
                    // a row without a target is zero whatever the weights hold
                    const float c = a.row_up && f == 0.f ? 0.f : acc[i][j][e] * (f * cf);
                    ((Out *)a.out)[m * a.ld_out + n] = (Out)c;
                }
            }
    }
}

template <class Out> __global__ __launch_bounds__(256) void k_finish(StoreArgs a)
{
    const int64_t n = (int64_t)blockIdx.y * 256 + threadIdx.x, m = blockIdx.x;
    if (n >= a.N) return;
    float s = 0.f;
    for (int k = 0; k < a.p.splits; k++) s += a.slabs[((int64_t)k * a.M + m) * a.N + n];
    const float f = row_factor(a, m);
    ((Out *)a.out)[m * a.ld_out + n] = (Out)(a.row_up && f == 0.f ? 0.f : s * (f * col_factor(a, n)));
}

// ------------------------------------------------------------ laying out
// dst [parts][rows, kp] from src [rows, D]: zeros past D; in two parts with a
// scale per row. One wavefront per row.
template <class In, class T, bool TWO>
__global__ __launch_bounds__(256) void k_pack(const In *src, int64_t ld, int64_t rows, int64_t D, T *dst, int64_t kp,
                                             int64_t part, float *scale)
{
    constexpr int VE = kVec<T>;
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= rows) return;
    src += r * ld;
    float inv = 1.f;
    if constexpr (TWO) {
        float top = 0.f;
        for (int64_t c = lane * VE; c < D; c += 64 * VE) {
            float f[VE];
            load_part<VE>(src + c, (int)min((int64_t)VE, D - c), f);
#pragma unroll
            for (int j = 0; j < VE; j++) top = fmaxf(top, fabsf(f[j]));
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
        const float s = scale_of(top);
        inv = inverse_of(s);
        if (lane == 0) scale[r] = s;
    }
    for (int64_t c = lane * VE; c < kp; c += 64 * VE) {
        float f[VE], lo[VE];
        load_part<VE>(src + (c < D ? c : 0), (int)max((int64_t)0, min((int64_t)VE, D - c)), f);
        if constexpr (TWO) {
#pragma unroll
            for (int j = 0; j < VE; j++) {
                f[j] *= inv;
                lo[j] = f[j] - (float)(T)f[j];
            }
            store_vec<VE>(dst + part + r * kp + c, lo);
        }
        store_vec<VE>(dst + r * kp + c, f);
    }
}

// col_max[d] = max over rows (with a target, if targets are given) of |src[r, d]|.
constexpr int kTile = 64;
__global__ __launch_bounds__(256) void k_col_max(const float *src, int64_t ld, int64_t rows, int64_t D,
                                                const uint64_t *targets, int64_t V, uint32_t *col_max)
{
    const int64_t d = (int64_t)blockIdx.y * 64 + (threadIdx.x & 63);
    const int64_t r0 = (int64_t)blockIdx.x * 256 + (threadIdx.x >> 6) * 64, r1 = min(r0 + 64, rows);
    if (d >= D) return;
    uint32_t top = 0;
    for (int64_t r = r0; r < r1; r++)
        if (!targets || targets[r] < (uint64_t)V) top = max(top, __float_as_uint(src[r * ld + d]) & 0x7fffffffu);
    // bits of magnitudes order like the magnitudes, NaN above all
    if (top) atomicMax(&col_max[d], top);
}

__global__ __launch_bounds__(256) void k_zero(uint32_t *p, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0;
}

// dst [parts][D, rp] = src^T, zeros for rows without a target (if targets are
// given) and for places past `rows`.
template <class In, class T, bool TWO>
__global__ __launch_bounds__(256) void k_pack_t(const In *src, int64_t ld, int64_t rows, int64_t D,
                                               const uint64_t *targets, int64_t V, T *dst, int64_t rp, int64_t part,
                                               const float *col_max)
{
    __shared__ float tile[kTile][kTile + 1];
    const int64_t r0 = (int64_t)blockIdx.x * kTile, d0 = (int64_t)blockIdx.y * kTile;
    for (int k = threadIdx.x; k < kTile * kTile; k += 256) {
        const int64_t r = r0 + k / kTile, d = d0 + k % kTile;
        const bool in = r < rows && d < D && (!targets || targets[r] < (uint64_t)V);
        tile[k / kTile][k % kTile] = in ? (float)src[r * ld + d] : 0.f;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < kTile * kTile; k += 256) {
        const int64_t r = r0 + k % kTile, d = d0 + k / kTile;
        if (d >= D) continue;
        float f = tile[k % kTile][k / kTile];
        if constexpr (TWO) {
            f *= inverse_of(scale_of(col_max[d]));
            dst[part + d * rp + r] = (T)(f - (float)(T)f);
        }
        dst[d * rp + r] = (T)f;
    }
}

// The largest |upstream| of a row with a target (at least 1e-30, to divide by).
__global__ __launch_bounds__(1024) void k_up_max(const float *up, const uint64_t *targets, int64_t N, int64_t V,
                                                float *out)
{
    __shared__ float red[16];
    float top = 0.f;
    for (int64_t i = threadIdx.x; i < N; i += 1024)
        if (targets[i] < (uint64_t)V) top = fmaxf(top, fabsf(up[i]));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 0; w < 16; w++) top = fmaxf(top, red[w]);
        *out = fmaxf(top, 1e-30f);
    }
}

// lse and loss of a token from its tiles' maxima and sums. One wavefront each.
__global__ __launch_bounds__(64) void k_lse(const float2 *part, int tiles, const uint64_t *targets, int64_t V,
                                           const float *z_target, float *loss, float *lse)
{
    const int64_t n = blockIdx.x;
    const int lane = threadIdx.x;
    part += n * tiles;
    float top = -INFINITY;
    for (int k = lane; k < tiles; k += 64) top = fmaxf(top, part[k].x);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    float sum = 0.f;
    for (int k = lane; k < tiles; k += 64) sum += part[k].y * __expf(part[k].x - top);
    sum = group_sum<64>(sum);
    if (lane) return;
    const float l = top + logf(sum);
    lse[n] = l;
    loss[n] = targets[n] < (uint64_t)V ? l - z_target[n] : 0.f;
}

// ------------------------------------------------------- a few tokens
// With up to kFewTokens tokens the weights are what there is to read: wavefronts
// stream kFewRows x 16 words each from memory into 16 x 16 matrix instructions,
// no LDS, no packing; the few hidden rows come from the caches.
constexpr int kFewTokens = 64, kFewRows = 2, kFewWaves = 4;
constexpr int kFewWords = 16 * kFewRows * kFewWaves;  // of a workgroup

template <class T> __device__ __forceinline__ void load_raw(const T *p, int n, T (&r)[kVec<T>])
{
    if (n >= kVec<T>) __builtin_memcpy(r, p, sizeof r);
    else
#pragma unroll
        for (int j = 0; j < kVec<T>; j++) r[j] = j < n ? p[j] : (T)0.f;
}

// One step of the sum: 16 bytes of each lane's row, in four groups of lanes.
__device__ __forceinline__ f32x4 mfma16(const __bf16 (&a)[8], const __bf16 (&b)[8], f32x4 c)
{
    frag<__bf16> x, y;
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = a[j], y[j] = b[j];
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(const _Float16 (&a)[8], const _Float16 (&b)[8], f32x4 c)
{
    frag<_Float16> x, y;
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = a[j], y[j] = b[j];
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(const float (&a)[4], const float (&b)[4], f32x4 c)
{
#pragma unroll
    for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

struct FewArgs {
    const void *hidden, *weight;
    int64_t ld_hidden, ld_weight, N, V, D;
    const uint64_t *targets;
    float2 *part;
    float *z_target;
};

template <class T, int NT> __global__ __launch_bounds__(64 * kFewWaves) void k_few(FewArgs a)
{
    constexpr int VE = kVec<T>, STEP = 4 * VE;
    __shared__ float2 join[kFewWaves][NT * 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t v0 = ((int64_t)blockIdx.x * kFewWaves + wave) * 16 * kFewRows;
    const T *w[kFewRows], *h[NT];
    const int64_t k_lane = (lane >> 4) * VE;
#pragma unroll
    for (int r = 0; r < kFewRows; r++)
        w[r] = (const T *)a.weight + min(v0 + r * 16 + (lane & 15), a.V - 1) * a.ld_weight;
#pragma unroll
    for (int t = 0; t < NT; t++)
        h[t] = (const T *)a.hidden + min((int64_t)t * 16 + (lane & 15), a.N - 1) * a.ld_hidden;
    f32x4 acc[kFewRows][NT];
#pragma unroll
    for (int r = 0; r < kFewRows; r++)
#pragma unroll
        for (int t = 0; t < NT; t++) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t whole = a.D / STEP * STEP;
#pragma unroll 4
    for (int64_t k = k_lane; k < whole; k += STEP) {
        T x[kFewRows][VE], y[NT][VE];
#pragma unroll
        for (int r = 0; r < kFewRows; r++) __builtin_memcpy(x[r], w[r] + k, sizeof x[r]);
#pragma unroll
        for (int t = 0; t < NT; t++) __builtin_memcpy(y[t], h[t] + k, sizeof y[t]);
#pragma unroll
        for (int r = 0; r < kFewRows; r++)
#pragma unroll
            for (int t = 0; t < NT; t++) acc[r][t] = mfma16(x[r], y[t], acc[r][t]);
    }
    if (whole < a.D) {
        const int64_t k = whole + k_lane;
        const int n = (int)max((int64_t)0, min((int64_t)VE, a.D - k));
        const int64_t kk = n ? k : 0;
        T x[kFewRows][VE], y[NT][VE];
#pragma unroll
        for (int r = 0; r < kFewRows; r++) load_raw<T>(w[r] + kk, n, x[r]);
#pragma unroll
        for (int t = 0; t < NT; t++) load_raw<T>(h[t] + kk, n, y[t]);
#pragma unroll
        for (int r = 0; r < kFewRows; r++)
#pragma unroll
            for (int t = 0; t < NT; t++) acc[r][t] = mfma16(x[r], y[t], acc[r][t]);
    }
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int64_t n = t * 16 + (lane & 15);
        const uint64_t target = n < a.N ? a.targets[n] : ~(uint64_t)0;
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < kFewRows; r++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int64_t v = v0 + r * 16 + (lane >> 4) * 4 + e;
                if (v >= a.V) acc[r][t][e] = -INFINITY;
                else if ((uint64_t)v == target) a.z_target[n] = acc[r][t][e];
                top = fmaxf(top, acc[r][t][e]);
            }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < kFewRows; r++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum += __expf(acc[r][t][e] - ref);
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (lane < 16) join[wave][n] = make_float2(top, sum);
    }
    __syncthreads();
    const int n = threadIdx.x;
    if (n < NT * 16 && n < a.N) {
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWaves; k++) top = fmaxf(top, join[k][n].x);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int k = 0; k < kFewWaves; k++) sum += join[k][n].y * __expf(join[k][n].x - ref);
        a.part[(int64_t)n * gridDim.x + blockIdx.x] = make_float2(top, sum);
    }
}

// ------------------------------------------------------------ plan
int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
int64_t ceil_div(int64_t n, int64_t m) { return (n + m - 1) / m; }

// Tiles of 256 x 256 run nearer to the matrix cores' rate, tiles of 128 x 128
// leave fewer compute units idle when there are few of them.
bool big_tiles(int64_t M, int64_t N)
{
    const int64_t big = ceil_div(M, Big::BM) * ceil_div(N, Big::BN);
    const int64_t small = ceil_div(M, Small::BM) * ceil_div(N, Small::BN);
    return ceil_div(big, 256) * 8 <= ceil_div(small, 512) * 5;
}

struct XentPlan {
    bool two, grad, few;
    int elem;
    int64_t N, V, D, kp, np, vp;
    int64_t piece;  // words of a piece
    int max_splits_h, max_splits_w;
    size_t hp, wp, h_scale, w_scale, wt, ht, w_max, h_max, part, z_target, up_max, prob, prob_t, slab_h, slab_w, bytes;

    static int splits_of(int64_t M, int64_t N, int64_t k_tiles)
    {
        if (M == 0 || N == 0) return 1;
        const bool big = big_tiles(M, N);
        const int64_t tiles = big ? ceil_div(M, Big::BM) * ceil_div(N, Big::BN)
                                  : ceil_div(M, Small::BM) * ceil_div(N, Small::BN);
        const int64_t slots = big ? 256 : 512;
        return (int)std::max<int64_t>(1, std::min({slots / tiles, k_tiles / 8, (int64_t)16}));
    }

    XentPlan(int32_t type, int64_t N_, int64_t V_, int64_t D_, bool grad_)
        : two(type == TQ_F32), grad(grad_), N(N_), V(V_), D(D_)
    {
        elem = 2 * (two ? 2 : 1);
        few = !grad && N <= kFewTokens;
        kp = std::max<int64_t>(up_to(D, kBK), kBK);
        np = up_to(N, kBK);
        vp = up_to(V, kBK);
        // pieces long enough that the products over them fill the chip, short
        // enough that p takes at most 2^28 elements
        piece = up_to(V, 256);
        if (grad && N * piece > ((int64_t)1 << 28))
            piece = std::max<int64_t>(256, (((int64_t)1 << 28) / std::max<int64_t>(N, 1)) / 256 * 256);
        Carver c;
        const int64_t tiles = few ? ceil_div(V, kFewWords) : ceil_div(V, Small::BM);
        part = c.take(sizeof(float2) * N * tiles);
        z_target = c.take(sizeof(float) * N);
        if (few) {
            bytes = c.used;
            return;
        }
        hp = c.take((size_t)elem * N * kp);
        wp = c.take((size_t)elem * V * kp);
        h_scale = c.take(two ? sizeof(float) * N : 0);
        w_scale = c.take(two ? sizeof(float) * V : 0);
        if (grad) {
            const int64_t words = std::min(piece, vp);
            wt = c.take((size_t)elem * D * vp);
            ht = c.take((size_t)elem * D * np);
            w_max = c.take(two ? sizeof(float) * D : 0);
            h_max = c.take(two ? sizeof(float) * D : 0);
            up_max = c.take(sizeof(float));
            prob = c.take((size_t)elem * N * words);
            prob_t = c.take((size_t)elem * words * np);
            const int terms = two ? 3 : 1;
            max_splits_h = splits_of(N, D, terms * (words / kBK));
            max_splits_w = splits_of(words, D, terms * (np / kBK));
            slab_h = c.take(sizeof(float) * max_splits_h * N * D);
            slab_w = c.take(max_splits_w > 1 ? sizeof(float) * max_splits_w * words * D : 0);
        }
        bytes = c.used;
    }
};

// Whether the products can read rows of D 16-bit elements where they are.
bool in_place(const void *p, int64_t ld, int64_t D)
{
    return D % kBK == 0 && D > 0 && ld % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

template <class T, class S, bool GRAD, bool TWO> void run_logits(LogitArgs a, hipStream_t s)
{
    a.p.m_tiles = (int)ceil_div(a.p.a.rows, S::BM);
    a.p.n_tiles = (int)ceil_div(GRAD ? a.ld_prob_t : a.N, S::BN);
    a.p.splits = 1;
    k_logits<T, S, GRAD, TWO><<<(unsigned)(a.p.m_tiles * a.p.n_tiles), S::threads, 0, s>>>(a);
}

template <class T, class Out> void run_product(StoreArgs a, bool big, hipStream_t s)
{
    auto go = [&](auto shape) {
        using S = decltype(shape);
        a.p.m_tiles = (int)ceil_div(a.M, S::BM);
        a.p.n_tiles = (int)ceil_div(a.N, S::BN);
        k_product<T, S, Out><<<(unsigned)(a.p.m_tiles * a.p.n_tiles * a.p.splits), S::threads, 0, s>>>(a);
    };
    if (big) go(Big{});
    else go(Small{});
}

// In: type of the arrays; T: of the products' operands; TWO: in two parts.
template <class In, class T, bool TWO> hipError_t xent_t(int32_t type, const XentArgs &a, bool grad, hipStream_t s)
{
    const XentPlan p(type, a.N, a.V, a.D, grad);
    char *ws = (char *)a.ws;
    float2 *part = (float2 *)(ws + p.part);
    float *z_target = (float *)(ws + p.z_target);
    int tiles;
    if (p.few) {
        const FewArgs f{a.hidden, a.weight, a.ld_hidden, a.ld_weight, a.N, a.V, a.D, a.targets, part, z_target};
        tiles = (int)ceil_div(a.V, kFewWords);
        if (a.N <= 16) k_few<In, 1><<<tiles, 64 * kFewWaves, 0, s>>>(f);
        else if (a.N <= 32) k_few<In, 2><<<tiles, 64 * kFewWaves, 0, s>>>(f);
        else k_few<In, 4><<<tiles, 64 * kFewWaves, 0, s>>>(f);
        k_lse<<<(unsigned)a.N, 64, 0, s>>>(part, tiles, a.targets, a.V, z_target, a.loss, a.lse);
        return hipGetLastError();
    }
    if (a.N) {
        const bool h_direct = !TWO && in_place(a.hidden, a.ld_hidden, a.D);
        const bool w_direct = !TWO && in_place(a.weight, a.ld_weight, a.D);
        float *h_scale = (float *)(ws + p.h_scale), *w_scale = (float *)(ws + p.w_scale);
        Operand h{ws + p.hp, p.kp, a.N * p.kp, a.N}, w{ws + p.wp, p.kp, a.V * p.kp, a.V};
        if (h_direct) h.p = a.hidden, h.ld = a.ld_hidden;
        else
            k_pack<In, T, TWO><<<(unsigned)ceil_div(a.N, 4), 256, 0, s>>>((const In *)a.hidden, a.ld_hidden, a.N, a.D,
                                                                        (T *)h.p, p.kp, h.part, h_scale);
        if (w_direct) w.p = a.weight, w.ld = a.ld_weight;
        else
            k_pack<In, T, TWO><<<(unsigned)ceil_div(a.V, 4), 256, 0, s>>>((const In *)a.weight, a.ld_weight, a.V, a.D,
                                                                        (T *)w.p, p.kp, w.part, w_scale);
        const int terms = TWO ? 3 : 1;
        LogitArgs l{};
        l.p.a = w;
        l.p.b = h;
        l.p.terms = terms;
        l.p.k_tiles = (int)(p.kp / kBK);
        l.word_scale = w_scale;
        l.token_scale = h_scale;
        l.targets = a.targets;
        l.V = a.V;
        l.N = a.N;
        l.part = part;
        l.z_target = z_target;
        if (big_tiles(a.V, a.N)) {
            run_logits<T, Big, false, TWO>(l, s);
            tiles = (int)ceil_div(a.V, Big::BM);
        } else {
            run_logits<T, Small, false, TWO>(l, s);
            tiles = (int)ceil_div(a.V, Small::BM);
        }
        k_lse<<<(unsigned)a.N, 64, 0, s>>>(part, tiles, a.targets, a.V, z_target, a.loss, a.lse);
        if (!grad) return hipGetLastError();
        float *up_max = (float *)(ws + p.up_max);
        k_up_max<<<1, 1024, 0, s>>>(a.upstream, a.targets, a.N, a.V, up_max);
        if (a.D == 0) return hipGetLastError();
        // the operands that run along words and along tokens
        T *wt = (T *)(ws + p.wt), *ht = (T *)(ws + p.ht);
        float *w_max = (float *)(ws + p.w_max), *h_max = (float *)(ws + p.h_max);
        if constexpr (TWO) {
            k_zero<<<(unsigned)ceil_div(a.D, 256), 256, 0, s>>>((uint32_t *)w_max, a.D);
            k_zero<<<(unsigned)ceil_div(a.D, 256), 256, 0, s>>>((uint32_t *)h_max, a.D);
            k_col_max<<<dim3((unsigned)ceil_div(a.V, 256), (unsigned)ceil_div(a.D, 64)), 256, 0, s>>>(
                (const float *)a.weight, a.ld_weight, a.V, a.D, nullptr, a.V, (uint32_t *)w_max);
            k_col_max<<<dim3((unsigned)ceil_div(a.N, 256), (unsigned)ceil_div(a.D, 64)), 256, 0, s>>>(
                (const float *)a.hidden, a.ld_hidden, a.N, a.D, a.targets, a.V, (uint32_t *)h_max);
        }
        k_pack_t<In, T, TWO><<<dim3((unsigned)(p.vp / kTile), (unsigned)ceil_div(a.D, kTile)), 256, 0, s>>>(
            (const In *)a.weight, a.ld_weight, a.V, a.D, nullptr, a.V, wt, p.vp, a.D * p.vp, w_max);
        k_pack_t<In, T, TWO><<<dim3((unsigned)(p.np / kTile), (unsigned)ceil_div(a.D, kTile)), 256, 0, s>>>(
            (const In *)a.hidden, a.ld_hidden, a.N, a.D, a.targets, a.V, ht, p.np, a.D * p.np, h_max);
        T *prob = (T *)(ws + p.prob), *prob_t = (T *)(ws + p.prob_t);
        float *slab_h = (float *)(ws + p.slab_h), *slab_w = (float *)(ws + p.slab_w);
        const bool big_h = big_tiles(a.N, a.D);
        int splits_h = 1;
        for (int64_t v0 = 0; v0 < a.V; v0 += p.piece) {
            const int64_t words = std::min(p.piece, a.V - v0), kv = up_to(words, kBK);
            l.p.a.p = (const T *)w.p + v0 * w.ld;
            l.p.a.rows = words;
            l.word_scale = w_scale + v0;
            l.v_base = v0;
            l.lse = a.lse;
            l.up = a.upstream;
            l.up_max = up_max;
            l.prob = prob;
            l.ld_prob = kv;
            l.prob_part = a.N * kv;
            l.prob_t = prob_t;
            l.ld_prob_t = p.np;
            l.prob_t_part = words * p.np;
            if (big_tiles(words, a.N)) run_logits<T, Big, true, TWO>(l, s);
            else run_logits<T, Small, true, TWO>(l, s);
            StoreArgs d{};
            d.p.a = Operand{prob, kv, l.prob_part, a.N};
            d.p.b = Operand{wt + v0, p.vp, a.D * p.vp, a.D};
            d.p.terms = terms;
            d.p.k_tiles = (int)(kv / kBK);
            if (v0 == 0) splits_h = std::min(p.max_splits_h, XentPlan::splits_of(a.N, a.D, terms * (kv / kBK)));
            d.p.splits = splits_h;
            d.M = a.N;
            d.N = a.D;
            d.slabs = slab_h;
            d.add = v0 > 0;
            run_product<T, In>(d, big_h, s);
            StoreArgs e{};
            e.p.a = Operand{prob_t, p.np, l.prob_t_part, words};
            e.p.b = Operand{ht, p.np, a.D * p.np, a.D};
            e.p.terms = terms;
            e.p.k_tiles = (int)(p.np / kBK);
            e.p.splits = std::min(p.max_splits_w, XentPlan::splits_of(words, a.D, terms * (p.np / kBK)));
            e.M = words;
            e.N = a.D;
            e.out = (In *)a.dweight + v0 * a.ld_dweight;
            e.ld_out = a.ld_dweight;
            e.col_max = TWO ? h_max : nullptr;
            e.up_max = up_max;
            if (e.p.splits > 1) e.slabs = slab_w;
            run_product<T, In>(e, big_tiles(words, a.D), s);
            if (e.slabs)
                k_finish<In><<<dim3((unsigned)words, (unsigned)ceil_div(a.D, 256)), 256, 0, s>>>(e);
        }
        StoreArgs f{};
        f.p.splits = splits_h;
        f.M = a.N;
        f.N = a.D;
        f.slabs = slab_h;
        f.out = a.dhidden;
        f.ld_out = a.ld_dhidden;
        f.row_up = a.upstream;
        f.targets = a.targets;
        f.V = a.V;
        f.col_max = TWO ? w_max : nullptr;
        k_finish<In><<<dim3((unsigned)a.N, (unsigned)ceil_div(a.D, 256)), 256, 0, s>>>(f);
        return hipGetLastError();
    }
    // no tokens: no gradient
    if (a.D)
        for (int64_t v = 0; v < a.V; v += 1 << 20) {
            StoreArgs e{};
            e.M = std::min<int64_t>(a.V - v, 1 << 20);
            e.N = a.D;
            e.out = (In *)a.dweight + v * a.ld_dweight;
            e.ld_out = a.ld_dweight;
            k_finish<In><<<dim3((unsigned)e.M, (unsigned)ceil_div(a.D, 256)), 256, 0, s>>>(e);
        }
    return hipGetLastError();
}

} // namespace

size_t xent_workspace(int32_t type, int64_t N, int64_t V, int64_t D, bool grad)
{
    return XentPlan(type, N, V, D, grad).bytes;
}

hipError_t launch_xent(int32_t type, const XentArgs &a, bool grad, hipStream_t s)
{
    if (type == TQ_F32) return xent_t<float, _Float16, true>(type, a, grad, s);
    if (type == TQ_BF16) return xent_t<__bf16, __bf16, false>(type, a, grad, s);
    return xent_t<_Float16, _Float16, false>(type, a, grad, s);
}

} // namespace tq
