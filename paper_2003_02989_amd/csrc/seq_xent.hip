// seq_xent.hip -- softmax cross entropy over a vocabulary, and its gradients.
//
//   z = hidden weight^T [N, V],  lse_i = log sum_v exp z_iv,
//   loss_i = lse_i - z_{i, t_i};   p = softmax(z) - onehot(t),
//   dhidden = diag(up) p weight,   dweight = (diag(up) p)^T hidden.
//
// Bound by the matrix products (2 N V D operations each): they run on the
// matrix cores in 16 bits with fp32 sums, in one kernel for products C = A B^T
// whose operands may each lie along the summed axis or across it.  The logits are never
// stored: the forward product's epilogue turns each tile of 256 (or 128) words
// by as many tokens into one maximum and one sum of exponentials per token.  For the
// gradient the vocabulary is taken in pieces; a piece's logits are formed a
// second time, now with lse known, and its p is stored in 16 bits, to be read
// along the vocabulary for dhidden and along the tokens for dweight.
//
// 16-bit inputs enter the products as they are.  fp32 inputs enter as two
// 16-bit (f16) numbers each, h + l with l the rounding error of h, after a
// power-of-two scale: a b = h_a h_b + h_a l_b + l_a h_b leaves out l_a l_b,
// 2^-22 of the product, and costs three products; fp32 matrix instructions
// would cost sixteen times the 16-bit ones.
//
// The stored p is p itself, up to a power of two: its largest entries are near -1,
// and a factor common to all tokens would put the same rounding error into each.
// upstream multiplies dhidden's rows at the end, in fp32, and enters dweight
// through the hidden rows, relative to the largest.  16-bit rows times that have
// twice the digits, and where any are lost (ups that differ by more than a power of
// two; the mean's equal weights lose none) they enter as two numbers, too, in two
// products: rounded to one, dweight is off by 1.4 to 1.5 times what its own rounding
// costs.  fp32 rows are scaled to magnitudes of 2^13 .. 2^14 on their own where the
// product leaves the row's axis standing; the operands that a product sums over the
// rows of have one scale for all, and their digits count from the largest row's.
#include <algorithm>
#include <cfloat>
#include <climits>
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

// p is held times 2^15 in 16 bits: at most 2^15 fits f16, whose small numbers
// would otherwise not reach the probabilities of a large vocabulary.
constexpr int kProbBits = 15;

// ------------------------------------------------------------ C = A B^T
// Operands of 16-bit elements, rows 16-byte aligned.  Along the summed axis:
// `extent` rows (of C, or columns of C) of K elements, K a multiple of kBK.  Across
// it: `k_rows` rows, one per summed index, of `extent` elements, a multiple of 8.
// What is read past `extent` is never used; past `k_rows` the last row is
// read again, and the other operand is zero there.  fp32 operands have two
// parts, `part` elements apart.
constexpr int kBK = 64;

struct Operand {
    const void *p;
    int64_t ld, part, extent, k_rows;
};

struct ProductArgs {
    Operand a, b;
    int terms;    // 1, 2 if the second operand is in two parts, 3 if both are
    int k_tiles;  // K / kBK
    int m_tiles, n_tiles;
    int full;     // tiles that one workgroup computes alone; the others are
    int splits;   // cut into this many, along K or (logits) along N
};

// Tile of C, wavefronts WM x WN, each with FM x FN blocks of 32 x 32.
template <int WM_, int WN_, int FM_, int FN_> struct Shape {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    static constexpr int waves = WM * WN, threads = waves * 64;
};
using Big = Shape<2, 4, 4, 2>;    // 256 x 256
using Small = Shape<2, 2, 2, 2>;  // 128 x 128
// A half and a quarter of a large tile, for logits of a last, incomplete round.
using Half = Shape<4, 2, 2, 2>;     // 256 x 128
using Quarter = Shape<4, 2, 2, 1>;  // 256 x 64

// Where an element of a wavefront's block lies: C row (within 32) of register i
// of a lane; its column is lane % 32.
__device__ __forceinline__ int block_row(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// One stage of an operand in LDS, W rows (or columns) of C by kBK, read straight
// from global memory, 16 bytes per lane.
//
// Along K: W rows of eight 16-byte pieces, the pieces of row r in the order
// piece ^ (r / 2 % 8): two rows fill the 64 banks once, so that the 16 lanes that
// read one piece of 16 rows at a time meet all banks.  (With piece ^ (r % 8) rows
// r and r + 8 met, and half of the LDS cycles were conflicts.)
template <class T, int W, int WAVES>
__device__ __forceinline__ void stage(T *lds, const T *src, const Operand &o, int64_t k0, int64_t at, int wave, int lane)
{
#pragma unroll
    for (int i = 0; i < W / 8 / WAVES; i++) {
        const int r8 = (i * WAVES + wave) * 8;
        const int64_t row = min(at + r8 + (lane >> 3), o.extent - 1);
        const T *g = src + row * o.ld + k0 + ((lane & 7) ^ (((r8 >> 1) + (lane >> 4)) & 7)) * 8;
        __builtin_amdgcn_global_load_lds((global_void *)g, (lds_void *)(lds + r8 * kBK), 16, 0, 0);
    }
}
template <class T> __device__ __forceinline__ frag<T> read_frag(const T *lds, int at, int ks, int lane)
{
    const int row = at + (lane & 31), piece = ks * 2 + (lane >> 5);
    return *(const frag<T> *)(lds + row * kBK + ((piece ^ ((row >> 1) & 7)) * 8));
}

// Across K: kBK rows of W elements.  The transposing LDS read gives 16 lanes
// four rows each of 16 columns, from 8 bytes at four rows by four pieces of four
// elements; row k has its 16-byte pieces in the order piece ^ 4 (k % 4), so
// that four rows of 32 columns, which 32 lanes read at a time, meet all banks.
template <class T, int W, int WAVES>
__device__ __forceinline__ void stage_t(T *lds, const T *src, const Operand &o, int64_t k0, int64_t at, int wave,
                                        int lane)
{
    constexpr int PIECES = W / 8, ROWS = 64 / PIECES;  // of one instruction
    static_assert(kBK % (ROWS * WAVES) == 0, "whole rows per wavefront");
#pragma unroll
    for (int i = 0; i < kBK / ROWS / WAVES; i++) {
        const int r0 = (i * WAVES + wave) * ROWS, r = r0 + lane / PIECES;
        const int64_t k = min(k0 + r, o.k_rows - 1);
        int64_t col = at + ((lane % PIECES) ^ (4 * (r & 3))) * 8;
        if (col >= o.extent) col = 0;
        __builtin_amdgcn_global_load_lds((global_void *)(src + k * o.ld + col), (lds_void *)(lds + r0 * W), 16, 0, 0);
    }
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
template <class T, int W> __device__ __forceinline__ frag<T> read_frag_t(const T *lds, int at, int ks, int lane)
{
    const int i = lane & 15, g = lane >> 4;
    const int k = ks * 16 + 8 * (g >> 1) + (i >> 2), col = at + 16 * (g & 1) + 4 * (i & 3);
    const T *p = lds + k * W + (((col >> 3) ^ (4 * ((i >> 2) & 3))) * 8) + (col & 7);
    union {
        s16x4 half[2];
        frag<T> all;
    } u;
    u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
    u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * W));
    return u.all;
}

template <class T> struct Stages {
    T *a0, *b0, *a1, *b1;
};
// The four arrays are separate objects: the compiler then knows that reads of
// one stage do not wait for loads into the other.
#define TQ_STAGES(T, S, name)                                                                                          \
    __shared__ alignas(1024) T name##_a0[S::BM * kBK], name##_b0[S::BN * kBK], name##_a1[S::BM * kBK],                 \
        name##_b1[S::BN * kBK];                                                                                        \
    const Stages<T> name{name##_a0, name##_b0, name##_a1, name##_b1}

// The sums of the tile at (m0, n0) over the K tiles [k0, k1) (of all terms).
template <class T, class S, bool TA, bool TB>
__device__ __forceinline__ void product(const ProductArgs &a, const Stages<T> &l, int64_t m0, int64_t n0, int k0,
                                        int k1, f32x16 (&acc)[S::FM][S::FN])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
#pragma unroll
    for (int i = 0; i < S::FM; i++)
#pragma unroll
        for (int j = 0; j < S::FN; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;
    auto fetch = [&](int kt, T *la, T *lb) {
        // the small terms first: l_a h_b, h_a l_b, h_a h_b, or the last ones of these
        const int term = kt / a.k_tiles;
        const int64_t k = (int64_t)(kt - term * a.k_tiles) * kBK;
        const T *ga = (const T *)a.a.p + (term == a.terms - 3 ? a.a.part : 0);
        const T *gb = (const T *)a.b.p + (term == a.terms - 2 ? a.b.part : 0);
        if constexpr (TA) stage_t<T, S::BM, S::waves>(la, ga, a.a, k, m0, wave, lane);
        else stage<T, S::BM, S::waves>(la, ga, a.a, k, m0, wave, lane);
        if constexpr (TB) stage_t<T, S::BN, S::waves>(lb, gb, a.b, k, n0, wave, lane);
        else stage<T, S::BN, S::waves>(lb, gb, a.b, k, n0, wave, lane);
    };
    auto compute = [&](const T *la, const T *lb) {
#pragma unroll
        for (int ks = 0; ks < kBK / 16; ks++) {
            frag<T> fa[S::FM], fb[S::FN];
#pragma unroll
            for (int i = 0; i < S::FM; i++) {
                if constexpr (TA) fa[i] = read_frag_t<T, S::BM>(la, wm + i * 32, ks, lane);
                else fa[i] = read_frag<T>(la, wm + i * 32, ks, lane);
            }
#pragma unroll
            for (int j = 0; j < S::FN; j++) {
                if constexpr (TB) fb[j] = read_frag_t<T, S::BN>(lb, wn + j * 32, ks, lane);
                else fb[j] = read_frag<T>(lb, wn + j * 32, ks, lane);
            }
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int j = 0; j < S::FN; j++) acc[i][j] = mfma32(fa[i], fb[j], acc[i][j]);
        }
    };
    if (k0 < k1) fetch(k0, l.a0, l.b0);
    __syncthreads();
    for (int kt = k0; kt < k1; kt += 2) {
        if (kt + 1 < k1) fetch(kt + 1, l.a1, l.b1);
        compute(l.a0, l.b0);
        __syncthreads();
        if (kt + 1 < k1) {
            if (kt + 2 < k1) fetch(kt + 2, l.a0, l.b0);
            compute(l.a1, l.b1);
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
    int id, split;  // split: -1 when the workgroup has the tile to itself
};
__device__ __forceinline__ Tile tile_of(const ProductArgs &a, int blk)
{
    Tile t;
    if (blk < a.full) {
        const int per = a.full / kXcds, more = a.full % kXcds, xcd = blk % kXcds;
        t.id = xcd * per + min(xcd, more) + blk / kXcds;
        t.split = -1;
    } else {
        const int left = a.m_tiles * a.n_tiles - a.full;
        t.id = a.full + (blk - a.full) % left;
        t.split = (blk - a.full) / left;
    }
    const int band = kGroup * a.n_tiles, g = t.id / band, rows = min(kGroup, a.m_tiles - g * kGroup);
    const int in = t.id - g * band;
    t.m = g * kGroup + in % rows;
    t.n = in / rows;
    return t;
}

// Orders the LDS accesses of one wavefront's lanes (they execute in order; this
// keeps the compiler from moving them).
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Exponent of |v|, finite and not zero (subnormal numbers count as the smallest
// normal ones).
__device__ __forceinline__ int exponent(float v) { return max((int)((__float_as_uint(v) >> 23) & 255), 1) - 127; }

// exp(z - r) from z and r log2 e, with one rounding of the exponent; that of
// r log2 e, up to |r| 2^-23, is common to a row and of the order of lse's own.
constexpr float kLog2e = 1.44269504088896341f;
__device__ __forceinline__ float exp_less(float z, float r2) { return __builtin_amdgcn_exp2f(fmaf(z, kLog2e, -r2)); }

// ------------------------------------------------------------ the logits
// A = weight (rows: words), B = hidden (rows: tokens): a lane's registers hold
// words of one token, so that sums over words stay within a lane until the end.
// 8192 x 65537 x 1024 bf16: 1130 us, 970 TFLOP/s; with p stored, in two
// pieces, 610 us each.
struct LogitArgs {
    ProductArgs p;
    const float *word_scale, *token_scale;  // of fp32 operands
    const uint64_t *targets;
    int64_t V, N;
    int64_t v_base;    // first word of the piece (p.a.p and word_scale point there)
    float2 *part;      // [N, tiles]: maximum, sum of exponentials
    float *z_target;   // [N]
    const float *lse;
    void *prob;        // [tokens, words] of the piece, both up to a multiple of kBK
    int64_t ld_prob, prob_rows, prob_part;
    uint32_t first;    // of the launch
};

//
// join: S::WM rows of S::BN, in LDS (GRAD: unused).
template <class T, class S, bool GRAD, bool TWO>
__device__ __forceinline__ void logits_tile(const LogitArgs &a, const Stages<T> &lds, float2 *join, int64_t m0, int64_t n0)
{
    f32x16 acc[S::FM][S::FN];
    product<T, S, false, false>(a.p, lds, m0, n0, 0, a.p.terms * a.p.k_tiles, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
    const int v0 = (int)m0 + wm;               // the wavefront's first word, in the piece
    const int words = (int)a.p.a.extent - v0;  // words from there on
    if constexpr (TWO) {
        // back from the scaled numbers
        float ts[S::FN];
#pragma unroll
        for (int j = 0; j < S::FN; j++) ts[j] = a.token_scale[min(n0 + wn + j * 32 + (lane & 31), a.N - 1)];
#pragma unroll
        for (int i = 0; i < S::FM; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                // four words in a row; the array goes on past the last word
                const f32x4 ws = *(const f32x4 *)(a.word_scale + v0 + i * 32 + block_row(4 * q, lane));
#pragma unroll
                for (int j = 0; j < S::FN; j++)
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[i][j][4 * q + e] *= ws[e] * ts[j];
                __builtin_amdgcn_sched_barrier(0);  // few loads ahead: registers
            }
    }
    if constexpr (!GRAD) {
#pragma unroll
        for (int j = 0; j < S::FN; j++) {
            const int64_t n = n0 + wn + j * 32 + (lane & 31);
            const uint64_t target = n < a.N ? a.targets[n] : ~(uint64_t)0;
            const int hit = target < (uint64_t)a.V ? (int)target - v0 : -1;
            // few tiles hold a target of theirs, or the end of the vocabulary
            if (__any(hit >= 0 && hit < S::FM * 32)) {
                float zt = 0.f;
#pragma unroll
                for (int i = 0; i < S::FM; i++)
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        if (i * 32 + block_row(e, lane) == hit) zt = acc[i][j][e];
                // the target's word is in one of the two lanes of a token
                if (hit >= 0 && hit < S::FM * 32 && ((hit >> 2) & 1) == lane >> 5) a.z_target[n] = zt;
            }
            if (words < S::FM * 32)
#pragma unroll
                for (int i = 0; i < S::FM; i++)
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        if (i * 32 + block_row(e, lane) >= words) acc[i][j][e] = -INFINITY;
            // four at a time: no long chain of dependent operations
            float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int e = 0; e < 16; e++) top4[e & 3] = fmaxf(top4[e & 3], acc[i][j][e]);
            float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            // without words there is nothing to add; NaN stays in the sum
            const float ref = top == -INFINITY ? 0.f : top;
            const float ref2 = ref * kLog2e;
            float sum4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int e = 0; e < 16; e++) sum4[e & 3] += exp_less(acc[i][j][e], ref2);
            float sum = (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
            sum += __shfl_xor(sum, 32, 64);
            if (lane < 32) join[wave / S::WN * S::BN + wn + j * 32 + lane] = make_float2(top, sum);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < S::BN; c += S::threads) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < S::WM; w++) top = fmaxf(top, join[w * S::BN + c].x);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < S::WM; w++) sum += join[w * S::BN + c].y * __expf(join[w * S::BN + c].x - ref);
            if (n0 + c < a.N) a.part[(n0 + c) * a.p.m_tiles + m0 / S::BM] = make_float2(top, sum);
        }
    } else {
#pragma unroll
        for (int j = 0; j < S::FN; j++) {
            const int64_t n = n0 + wn + j * 32 + (lane & 31);
            const uint64_t target = n < a.N ? a.targets[n] : ~(uint64_t)0;
            const bool on = target < (uint64_t)a.V;
            const float lse = on ? a.lse[n] : 0.f;
            const int64_t away = on ? (int64_t)target - a.v_base - v0 : -1;
            const int hit = away >= 0 && away < S::FM * 32 ? (int)away : -1;
            const float lse2 = lse * kLog2e;
            const bool some = __any(hit >= 0);
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int e = 0; e < 16; e++) acc[i][j][e] = exp_less(acc[i][j][e], lse2);
            if (some)
#pragma unroll
                for (int i = 0; i < S::FM; i++)
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        if (i * 32 + block_row(e, lane) == hit) acc[i][j][e] -= 1.f;
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int e = 0; e < 16; e++) acc[i][j][e] *= (float)(1 << kProbBits);
            // what is not a word of a token with a target is zero, whatever it holds
            const int last = on ? words : 0;
            if (__any(last < S::FM * 32))
#pragma unroll
                for (int i = 0; i < S::FM; i++)
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        if (i * 32 + block_row(e, lane) >= last) acc[i][j][e] = 0.f;
        }
        // Each wavefront turns its words x tokens through LDS (the stages are done
        // with), tokens as rows, 16-byte pieces in the order piece ^ token, and
        // writes whole rows.
        constexpr int WORDS = S::FM * 32, TOKENS = S::FN * 32, PIECES = WORDS / 8, PER = S::waves / 4;
        static_assert(PER * WORDS * TOKENS <= S::BM * kBK && PER * WORDS * TOKENS <= S::BN * kBK, "fits the stages");
        T *const buf = (wave / PER == 0   ? lds.a0
                        : wave / PER == 1 ? lds.b0
                        : wave / PER == 2 ? lds.a1
                                          : lds.b1) +
                       wave % PER * WORDS * TOKENS;
#pragma unroll 1  // unrolled, the addresses of both parts stay in registers and spill
        for (int part = 0; part < (TWO ? 2 : 1); part++) {
#pragma unroll
            for (int j = 0; j < S::FN; j++) {
                const int row = j * 32 + (lane & 31);
#pragma unroll
                for (int i = 0; i < S::FM; i++)
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        T four[4];
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const float p = acc[i][j][4 * q + e];
                            four[e] = (T)p;
                            if constexpr (TWO) acc[i][j][4 * q + e] = p - (float)four[e];
                        }
                        const int piece = i * 4 + q;
                        __builtin_memcpy(__builtin_assume_aligned(buf + row * WORDS + ((piece ^ (row & (PIECES - 1))) * 8) +
                                                                      4 * (lane >> 5),
                                                                  8),
                                         four, 8);
                    }
            }
            wave_fence();
            T *out = (T *)a.prob + part * a.prob_part;
#pragma unroll
            for (int k = 0; k < TOKENS * PIECES / 64; k++) {
                const int row = (k * 64 + lane) / PIECES, piece = lane % PIECES;
                const frag<T> v = *(const frag<T> *)(buf + row * WORDS + ((piece ^ (row & (PIECES - 1))) * 8));
                const int64_t n = n0 + wn + row, w = v0 + piece * 8;
                if (n < a.prob_rows && w < a.ld_prob) *(frag<T> *)(out + n * a.ld_prob + w) = v;
            }
            wave_fence();
        }
    }
}

// Large tiles of a last, incomplete round go in halves or quarters of their
// tokens: an epilogue follows the whole sum, so that they are not cut along K.
template <class T, class S, bool GRAD, bool TWO> __global__ __launch_bounds__(S::threads) void k_logits(LogitArgs a)
{
    TQ_STAGES(T, S, lds);
    __shared__ float2 join[GRAD ? 1 : std::max(S::WM * S::BN, Half::WM * Half::BN)];
    const Tile t = tile_of(a.p, (int)(a.first + block_of()));
    const int64_t m0 = t.m * S::BM, n0 = t.n * S::BN;
    if constexpr (std::is_same_v<S, Big>)
        if (t.split >= 0) {
            const int64_t n = n0 + t.split * (S::BN / a.p.splits);
            if (n >= (GRAD ? a.prob_rows : a.N)) return;
            if (a.p.splits == 4) logits_tile<T, Quarter, GRAD, TWO>(a, lds, join, m0, n);
            else logits_tile<T, Half, GRAD, TWO>(a, lds, join, m0, n);
            return;
        }
    logits_tile<T, S, GRAD, TWO>(a, lds, join, m0, n0);
}

// ------------------------------------------------------------ the products
// By kUpParts workgroups, over the rows with a target and a finite up that is not
// zero: the largest |up|; of fp32 rows the largest exponent of up times the row's
// scale (else -1000); of 16-bit rows the least and the largest digits of up.
constexpr int kUpParts = 64;
struct UpParts {
    float up[kUpParts];
    int bits[kUpParts];
    int least[kUpParts], most[kUpParts];  // of 16-bit rows
    int terms;  // of dweight's product of 16-bit rows, written with its hidden rows
};
// The largest |up| (1 if there is none), and the power of two that dweight's
// hidden rows are scaled by, 0 for 16-bit rows: it brings the largest of up
// times the scale to that of the largest up.
struct UpMax {
    float up;
    int bits;
};
__device__ __forceinline__ UpMax up_max_of(const UpParts *p)
{
    const int lane = threadIdx.x & 63;
    float u = p->up[lane];
    int e = p->bits[lane];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        u = fmaxf(u, __shfl_xor(u, d, 64));
        e = max(e, __shfl_xor(e, d, 64));
    }
    if (u == 0.f) return UpMax{1.f, 0};
    return UpMax{u, e > -1000 ? e - exponent(u) : 0};
}

// Whether two ups differ by more than a power of two: hidden rows times up over the
// largest up do not fit 16 bits then.
__device__ __forceinline__ bool up_varies(const UpParts *p)
{
    const int lane = threadIdx.x & 63;
    int least = p->least[lane], most = p->most[lane];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        least = min(least, __shfl_xor(least, d, 64));
        most = max(most, __shfl_xor(most, d, 64));
    }
    return least < most;
}

// What becomes of C: out = factor(row) C, or C is added up in fp32 over the
// pieces of the vocabulary (`sum`), or a part of a tile goes to its slab.
struct StoreArgs {
    ProductArgs p;
    int64_t M, N;
    float *slabs;  // [tile past `full`][split][BM BN]
    float *sum;    // NULL: write `out`
    bool add;      // to what `sum` holds
    void *out;
    int64_t ld_out;
    // factor: the row's up, or the largest one and the scale for all; and the
    // scale of the second operand
    const float *up;
    const uint64_t *targets;
    int64_t V;
    const UpParts *up_max;
    const float *w_max;
    const int *terms;  // NULL: p.terms
};

// The power of two that brings numbers of magnitude up to m into [2^13, 2^14).
__device__ __forceinline__ int scale_bits(float m)
{
    return max((int)((__float_as_uint(m) >> 23) & 255) - 127, -100) - 13;
}
__device__ __forceinline__ float two_to(int e) { return ldexpf(1.f, e); }

// The maximum of kMaxParts partial maxima, by one wavefront.
constexpr int kMaxParts = 256;
__device__ __forceinline__ float max_of(const float *part)
{
    const int lane = threadIdx.x & 63;
    float m = fmaxf(fmaxf(part[lane], part[lane + 64]), fmaxf(part[lane + 128], part[lane + 192]));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    return m;
}

struct Factor {
    const StoreArgs &a;
    int bits;
    float all;
    __device__ explicit Factor(const StoreArgs &s) : a(s), bits(-kProbBits), all(1.f)
    {
        if (a.w_max) bits += scale_bits(max_of(a.w_max));
        if (a.up_max) {
            const UpMax u = up_max_of(a.up_max);
            all = u.up;
            bits += u.bits;
        }
    }
    // c times the factor of row m; a row without a target is zero whatever the
    // weights hold
    __device__ float of(float c, int64_t m) const
    {
        if (!a.up) return ldexpf(c, bits) * all;
        return a.targets[m] < (uint64_t)a.V ? ldexpf(c, bits) * a.up[m] : 0.f;
    }
};

template <class T, class S, bool TA, class Out>
__device__ __forceinline__ void product_tile(const StoreArgs &a, const Stages<T> &lds, int blk)
{
    ProductArgs p = a.p;
    if (a.terms) p.terms = *a.terms;
    const Tile t = tile_of(p, blk);
    f32x16 acc[S::FM][S::FN];
    const int64_t m0 = t.m * S::BM, n0 = t.n * S::BN;
    const int all = p.terms * p.k_tiles;
    int k0 = 0, k1 = all;
    if (t.split >= 0) {
        k0 = (int)((int64_t)all * t.split / p.splits);
        k1 = (int)((int64_t)all * (t.split + 1) / p.splits);
    }
    product<T, S, TA, true>(p, lds, m0, n0, k0, k1, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / S::WN * S::FM * 32, wn = wave % S::WN * S::FN * 32;
    if (t.split >= 0) {
        float *slab = a.slabs + ((int64_t)(t.id - a.p.full) * a.p.splits + t.split) * (S::BM * S::BN);
#pragma unroll
        for (int j = 0; j < S::FN; j++)
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int e = 0; e < 16; e++)
                    slab[(wm + i * 32 + block_row(e, lane)) * S::BN + wn + j * 32 + (lane & 31)] = acc[i][j][e];
        return;
    }
    const Factor factor(a);
#pragma unroll
    for (int i = 0; i < S::FM; i++)
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const int64_t m = m0 + wm + i * 32 + block_row(e, lane);
            if (m >= a.M) continue;
#pragma unroll
            for (int j = 0; j < S::FN; j++) {
                const int64_t n = n0 + wn + j * 32 + (lane & 31);
                if (n >= a.N) continue;
                const float c = acc[i][j][e];
                if (a.sum) {
                    float *o = a.sum + m * a.N + n;
                    *o = a.add ? *o + c : c;
                } else ((Out *)a.out)[m * a.ld_out + n] = (Out)factor.of(c, m);
            }
        }
}

// dhidden's product in the first h_blocks workgroups and dweight's, whose tiles
// fill what the former's last round leaves free, in the others.  8192 x 65537 x 1024
// bf16, in two pieces: 1040 us each, 1060 TFLOP/s, the matrix units busy half of the time.
template <class T, class S, class Out>
__global__ __launch_bounds__(S::threads) void k_products(StoreArgs h, StoreArgs w, int h_blocks, uint32_t first)
{
    TQ_STAGES(T, S, lds);
    const int blk = (int)(first + block_of());
    if (blk < h_blocks) product_tile<T, S, false, Out>(h, lds, blk);
    else product_tile<T, S, true, Out>(w, lds, blk - h_blocks);
}

// The tiles that were cut along K: their slabs, added up in order.
template <class S, class Out> __global__ __launch_bounds__(256) void k_slabs(StoreArgs h, StoreArgs w, int h_tail)
{
    const StoreArgs &a = (int)blockIdx.x < h_tail ? h : w;
    const int tail = (int)blockIdx.x < h_tail ? blockIdx.x : blockIdx.x - h_tail;
    const ProductArgs &p = a.p;
    // the tile's place, as tile_of gives it
    const int id = p.full + tail;
    const int band = kGroup * p.n_tiles, g = id / band, rows = min(kGroup, p.m_tiles - g * kGroup);
    const int in = id - g * band;
    const int64_t m0 = (int64_t)(g * kGroup + in % rows) * S::BM, n0 = (int64_t)(in / rows) * S::BN;
    const float *slab = a.slabs + (int64_t)tail * p.splits * (S::BM * S::BN);
    const Factor factor(a);
    // four columns per thread
    const int at = (blockIdx.y * 256 + threadIdx.x) * 4, r = at / S::BN, c = at % S::BN;
    const int64_t m = m0 + r, n = n0 + c;
    if (m >= a.M) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int q = 0; q < p.splits; q++) s += *(const f32x4 *)(slab + (int64_t)q * (S::BM * S::BN) + at);
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if (n + j >= a.N) break;
        if (a.sum) {
            float *o = a.sum + m * a.N + n + j;
            *o = a.add ? *o + s[j] : s[j];
        } else ((Out *)a.out)[m * a.ld_out + n + j] = (Out)factor.of(s[j], m);
    }
}

// out = factor(row) sum; zeros without a sum.
template <class Out> __global__ __launch_bounds__(256) void k_finish(StoreArgs a)
{
    const int64_t n = (int64_t)blockIdx.y * 256 + threadIdx.x;
    const Factor factor(a);
    if (n >= a.N) return;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x)
        ((Out *)a.out)[m * a.ld_out + n] = (Out)(a.sum ? factor.of(a.sum[m * a.N + n], m) : 0.f);
}

// ------------------------------------------------------------ laying out
// Partial maxima of the finite magnitudes of src [rows, D], by kMaxParts
// workgroups.
__device__ __forceinline__ void max_part(const float *src, int64_t ld, int64_t rows, int64_t D, float *part, int blk)
{
    __shared__ float red[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float top = 0.f;
    for (int64_t r = (int64_t)blk * 4 + wave; r < rows; r += kMaxParts * 4)
        for (int64_t c = lane * 4; c < D; c += 256) {
            float f[4];
            load_part<4>(src + r * ld + c, (int)min((int64_t)4, D - c), f);
#pragma unroll
            for (int j = 0; j < 4; j++) top = fabsf(f[j]) < INFINITY ? fmaxf(top, fabsf(f[j])) : top;
        }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    if (lane == 0) red[wave] = top;
    __syncthreads();
    if (threadIdx.x == 0) part[blk] = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

struct PackArgs {
    const void *src;
    int64_t ld, rows, D;
    void *dst;          // [parts][rows, kp], zeros past D
    int64_t kp, part;
    float *scale;       // fp32: a power of two per row; written unless `all` alone is wanted
    void *all;          // fp32: a second copy with the scale of the maximum in w_max
    const float *w_max;
    // dst for dweight's product: zeros for rows without a target, other rows
    // times up, relative to the largest, and 2^-bits; of 16-bit rows a second part
    // with what the first one's rounding lost, unless it lost nothing
    const uint64_t *targets;
    int64_t V;
    const float *up;
    UpParts *up_max;
};

// One wavefront per row, four rows per workgroup.
template <class In, class T, bool TWO> __device__ __forceinline__ void pack_rows(const PackArgs &a, int blk)
{
    constexpr int VE = kVec<T>;
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blk * 4 + (threadIdx.x >> 6);
    const float w_max = TWO && a.all ? max_of(a.w_max) : 0.f;
    const UpMax largest = a.up ? up_max_of(a.up_max) : UpMax{1.f, 0};
    if (r >= a.rows) return;
    const In *src = (const In *)a.src + r * a.ld;
    int bits = 0, bits_all = 0;
    bool on = true;
    if constexpr (TWO) {
        bits_all = -scale_bits(w_max);
        float top = 0.f;
        for (int64_t c = lane * VE; c < a.D; c += 64 * VE) {
            float f[VE];
            load_part<VE>(src + c, (int)min((int64_t)VE, a.D - c), f);
            // a row with infinities is NaN in the products, by any scale
#pragma unroll
            for (int j = 0; j < VE; j++) top = fmaxf(top, fabsf(f[j]));
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
        bits = -scale_bits(top);
        if (a.scale && lane == 0) a.scale[r] = two_to(-bits);
    }
    float share = 1.f;
    bool second = false;
    if (a.up) {
        if constexpr (!TWO) {
            second = up_varies(a.up_max);
            if (r == 0 && lane == 0) a.up_max->terms = second ? 2 : 1;
        }
        on = a.targets[r] < (uint64_t)a.V;
        share = on ? a.up[r] / largest.up : 0.f;
        bits = -largest.bits;
    }
    for (int64_t c = lane * VE; c < a.kp; c += 64 * VE) {
        float f[VE], g[VE], lo[VE];
        const int n = on ? (int)max((int64_t)0, min((int64_t)VE, a.D - c)) : 0;
        load_part<VE>(src + (n ? c : 0), n, f);
        T *dst = (T *)a.dst + r * a.kp + c;
#pragma unroll
        for (int j = 0; j < VE; j++) {
            g[j] = TWO ? ldexpf(f[j] * share, bits) : f[j] * share;
            lo[j] = g[j] - (float)(T)g[j];
        }
        store_vec<VE>(dst, g);
        if (second) store_vec<VE>(dst + a.part, lo);
        if constexpr (TWO) {
            store_vec<VE>(dst + a.part, lo);
            if (a.all) {
                T *all = (T *)a.all + r * a.kp + c;
#pragma unroll
                for (int j = 0; j < VE; j++) {
                    g[j] = ldexpf(f[j], bits_all);
                    lo[j] = g[j] - (float)(T)g[j];
                }
                store_vec<VE>(all, g);
                store_vec<VE>(all + a.part, lo);
            }
        }
    }
}

struct UpArgs {
    const float *up, *scale;  // scale: of fp32 rows
    const uint64_t *targets;
    int64_t N, V;
    UpParts *out;
};
template <bool TWO> __device__ __forceinline__ void up_max(const UpArgs &a, int blk)
{
    __shared__ float reds[4];
    __shared__ int low[4], high[4];
    float top = 0.f;
    // fp32: the largest exponent, in `most`; 16 bits: the least and largest digits
    int least = INT_MAX, most = TWO ? -1000 : 0;
    for (int64_t i = (int64_t)blk * 256 + threadIdx.x; i < a.N; i += 256 * kUpParts) {
        const float u = fabsf(a.up[i]);
        const bool on = a.targets[i] < (uint64_t)a.V && u > 0.f && u < INFINITY;
        top = on ? fmaxf(top, u) : top;
        if constexpr (TWO) most = on ? max(most, exponent(u) + exponent(a.scale[i])) : most;
        else {
            const int digits = __float_as_int(u) & 0x7fffff;
            // numbers below the normal ones have their digits elsewhere
            least = on ? min(least, u < FLT_MIN ? -1 : digits) : least;
            most = on ? max(most, digits) : most;
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        top = fmaxf(top, __shfl_xor(top, d, 64));
        most = max(most, __shfl_xor(most, d, 64));
        if constexpr (!TWO) least = min(least, __shfl_xor(least, d, 64));
    }
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) reds[wave] = top, low[wave] = least, high[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 0; w < 4; w++) top = fmaxf(top, reds[w]), least = min(least, low[w]), most = max(most, high[w]);
        a.out->up[blk] = top;
        a.out->bits[blk] = TWO ? most : -1000;
        if constexpr (!TWO) a.out->least[blk] = least, a.out->most[blk] = most;
    }
}

struct LseArgs {
    const float2 *part;  // [N, tiles]
    int tiles;
    int64_t N, V;
    const uint64_t *targets;
    const float *z_target;
    float *loss, *lse;
};
// lse and loss of a token from its tiles' maxima and sums. One wavefront each.
__device__ __forceinline__ void lse_rows(const LseArgs &a, int blk)
{
    const int64_t n = (int64_t)blk * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (n >= a.N) return;
    const float2 *part = a.part + n * a.tiles;
    float top = -INFINITY;
    for (int k = lane; k < a.tiles; k += 64) top = fmaxf(top, part[k].x);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    float sum = 0.f;
    for (int k = lane; k < a.tiles; k += 64) sum += part[k].y * __expf(part[k].x - top);
    sum = group_sum<64>(sum);
    if (lane) return;
    const float l = top + logf(sum);
    a.lse[n] = l;
    a.loss[n] = a.targets[n] < (uint64_t)a.V ? l - a.z_target[n] : 0.f;
}

// Small steps that do not wait for one another share a launch.
//
// Before the logits: hidden's rows laid out, and what the weights' layout needs
// (their partial maxima).
template <class In, class T, bool TWO>
__global__ __launch_bounds__(256) void k_lay_hidden(PackArgs h, int h_blocks, const float *w, int64_t ld_w, int64_t V,
                                                   float *w_max, int max_blocks)
{
    const int blk = (int)block_of();
    if (blk < h_blocks) pack_rows<In, T, TWO>(h, blk);
    else if (blk - h_blocks < max_blocks) max_part(w, ld_w, V, h.D, w_max, blk - h_blocks);
}
// The weights' rows laid out, and the largest upstream.
template <class In, class T, bool TWO>
__global__ __launch_bounds__(256) void k_lay_weight(PackArgs w, int w_blocks, UpArgs u, int up_blocks)
{
    const int blk = (int)block_of();
    if (blk < w_blocks) pack_rows<In, T, TWO>(w, blk);
    else if (blk - w_blocks < up_blocks) up_max<TWO>(u, blk - w_blocks);
}
// After the logits: lse and loss, and hidden's rows laid out for dweight.
template <class In, class T, bool TWO>
__global__ __launch_bounds__(256) void k_lse(LseArgs l, int l_blocks, PackArgs h, int h_blocks)
{
    const int blk = (int)block_of();
    if (blk < l_blocks) lse_rows(l, blk);
    else if (blk - l_blocks < h_blocks) pack_rows<In, T, TWO>(h, blk - l_blocks);
}

// ------------------------------------------------------- a few tokens
// With few tokens the weights are what there is to read: wavefronts
// stream kFewRows x 16 words each from memory into 16 x 16 matrix instructions,
// no LDS, no packing; the few hidden rows come from the caches.  4 x 65537 x 512
// bf16 15 to 20 us, 3.3 to 4.5 TB/s (67 MB, partly from the last-level cache): the
// weights are all there is to read, but a wavefront waits for each step's reads
// before it asks for the next one's (the compiler does not unroll loops around
// matrix instructions whose trip count it does not know).  Up to 16 tokens of weights that the tiles can read where they
// are (23 us for 16, 41 us for 64; tiles 27 us for 65), else up to kFewTokens, since
// the tiles need the weights laid out first (fp32 of that size: 73 us for 64 tokens,
// tiles 111 us for 65; 65537 x 500 bf16 28 us for 33 tokens and 32 for 64, laid out
// 53; rows of 512 that lie 513 apart 41 us for 17 tokens, 45 for 32 and 56 for 64,
// laid out 50).
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
    float2 *part;  // [N, tiles]
    float *z_target;
    int tiles;
    uint32_t first;  // of the launch
};

template <class T, int NT> __global__ __launch_bounds__(64 * kFewWaves) void k_few(FewArgs a)
{
    constexpr int VE = kVec<T>, STEP = 4 * VE;
    __shared__ float2 join[kFewWaves][NT * 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tile = (int)(a.first + block_of());
    const int64_t v0 = ((int64_t)tile * kFewWaves + wave) * 16 * kFewRows;
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
        a.part[(int64_t)n * a.tiles + tile] = make_float2(top, sum);
    }
}

// ------------------------------------------------------------ plan
int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
int64_t ceil_div(int64_t n, int64_t m) { return (n + m - 1) / m; }

// How C [M, N] is cut into tiles.  Tiles go to the compute units in rounds (256
// large ones or 512 small ones, two to a compute unit, at a time); the tiles of
// a last, incomplete round are cut along K so that they fill it, those of logits,
// if large, in two or four along the tokens.
//
// What a cut costs is estimated in steps, a large tile's kBK of K (2.2 us): a small
// tile's count 5/8, half the work at four fifths of the rate; a tile begins and ends in
// three; writing and adding up the slabs of a round takes twelve.
struct Cut {
    bool big;
    int m_tiles, n_tiles, full, splits, tail;
    double work, slabs;        // steps of all tiles over the slots, and of the slabs
    double longest;            // of a tile of the last round
    int slots() const { return big ? 256 : 512; }
    // room: what the parts of the last round may take, up to slots
    template <class S> static Cut of(int64_t M, int64_t N, int64_t k_tiles, int room)
    {
        constexpr double kEnds = 3, kSlabs = 12;
        Cut c{};
        c.big = std::is_same_v<S, Big>;
        const int slots = c.slots();
        const double scale = c.big ? 1. : 0.625;
        c.m_tiles = (int)ceil_div(M, S::BM);
        c.n_tiles = (int)ceil_div(N, S::BN);
        const int tiles = c.m_tiles * c.n_tiles;
        c.tail = tiles % slots;
        c.splits = 1;
        auto slabs = [&](int q) { return q > 1 ? kSlabs * c.tail * q / slots : 0.; };
        auto last = [&](int q) { return (double)ceil_div(k_tiles, q) + kEnds + slabs(q); };
        for (int q = 2; q <= 16 && (int64_t)c.tail * q <= room && k_tiles / q >= 4; q++)
            if (last(q) < last(c.splits)) c.splits = q;
        c.work = scale * tiles / slots * (k_tiles + kEnds);
        c.slabs = scale * slabs(c.splits);
        c.longest = scale * (ceil_div(k_tiles, c.tail ? c.splits : 1) + kEnds);
        if (c.splits == 1) c.tail = 0;
        c.full = tiles - c.tail;
        return c;
    }
    // of logits
    template <class S> static Cut logits(int64_t M, int64_t N)
    {
        Cut c = of<S>(M, N, 1, 0);
        c.tail = c.full % c.slots();
        if (c.big && c.tail) c.splits = c.tail <= c.slots() / 4 ? 4 : c.tail <= c.slots() / 2 ? 2 : 1;
        const double rounds = c.full / c.slots() + (c.tail ? 1. / c.splits + (c.splits > 1 ? 0.1 : 0.) : 0.);
        c.work = rounds * (c.big ? 1. : 0.625);
        if (c.splits == 1) c.tail = 0;
        c.full -= c.tail;
        return c;
    }
    // steps of a launch of its own
    double steps() const { return slabs + (blocks() <= slots() ? longest : work + 0.5 * longest); }
    int blocks() const { return full + tail * splits; }
    size_t slab_bytes() const
    {
        const size_t tile = big ? Big::BM * Big::BN : Small::BM * Small::BN;
        return sizeof(float) * tile * tail * splits;
    }
    void put(ProductArgs &p) const
    {
        p.m_tiles = m_tiles;
        p.n_tiles = n_tiles;
        p.full = full;
        p.splits = splits;
    }
};

Cut cut_logits(int64_t M, int64_t N)
{
    const Cut b = Cut::logits<Big>(M, N), s = Cut::logits<Small>(M, N);
    return b.work <= s.work ? b : s;
}

// dhidden's and dweight's products.  Of one shape they share a launch, dhidden's
// tiles first, where one fills what the other leaves free of a round; else two more
// launches take as long as eight steps.
struct Cuts {
    Cut h, w;
    double steps() const
    {
        if (h.big != w.big) return h.steps() + w.steps() + 8;
        const double longest = std::max(h.longest, w.longest);
        if (h.blocks() + w.blocks() <= h.slots()) return h.slabs + w.slabs + longest;
        return h.slabs + w.slabs + std::max(longest, h.work + w.work + 0.5 * w.longest);
    }
};
Cuts cut_products(int64_t N, int64_t D, int64_t words, int64_t h_tiles, int64_t w_tiles)
{
    Cuts best{};
    double least = INFINITY;
    auto take = [&](const Cut &h, const Cut &w) {
        const Cuts c{h, w};
        if (c.steps() < least) least = c.steps(), best = c;
    };
    auto shape = [&](auto s) {
        using S = decltype(s);
        const int slots = std::is_same_v<S, Big> ? 256 : 512;
        const Cut h = Cut::of<S>(N, D, h_tiles, slots), w = Cut::of<S>(words, D, w_tiles, slots);
        take(h, w);
        // both in one round: what either leaves of it is the other's
        const Cut whole = Cut::of<S>(N, D, h_tiles, 0);
        take(Cut::of<S>(N, D, h_tiles, slots - w.blocks()), w);
        take(whole, Cut::of<S>(words, D, w_tiles, slots - whole.blocks()));
        const int share = (int)(slots * h.work / (h.work + w.work));
        take(Cut::of<S>(N, D, h_tiles, share), Cut::of<S>(words, D, w_tiles, slots - share));
        return Cuts{h, w};
    };
    const Cuts b = shape(Big{}), s = shape(Small{});
    take(b.h, s.w);
    take(s.h, b.w);
    return best;
}

// Sizes and workspace of a call.
struct XentPlan {
    bool two, few;
    int terms;
    int64_t N, V, D, kp, np;
    int64_t piece;  // words of a piece of the vocabulary
    size_t part, z_target, hp, wp, all, hs, h_scale, w_scale, w_max, up_max, prob, sum, slabs_h, slabs_w, bytes;

    Cuts cuts, last_cuts;  // of a piece's products, of the last one's
    Cuts cuts_of(int64_t words) const
    {
        return cut_products(N, D, words, terms * (up_to(words, kBK) / kBK), terms * (np / kBK));
    }

    // in_place: the products can read the weights where they are
    XentPlan(int32_t type, int64_t N_, int64_t V_, int64_t D_, bool grad, bool in_place)
        : two(type == TQ_F32), few(!grad && N_ <= (in_place ? 16 : kFewTokens)), terms(two ? 3 : 1), N(N_), V(V_), D(D_)
    {
        const size_t elem = 2 * (two ? 2 : 1);
        kp = std::max<int64_t>(up_to(D, kBK), kBK);
        np = up_to(N, kBK);
        // a piece's p takes up to about 2^28 elements
        const int64_t most = std::max<int64_t>(256, ((int64_t)1 << 28) / std::max<int64_t>(N, 1) / 256 * 256);
        piece = up_to(ceil_div(V, ceil_div(V, most * 9 / 8)), 256);
        Carver c;
        const int64_t tiles = few ? ceil_div(V, kFewWords) : ceil_div(V, Small::BM);
        part = c.take(sizeof(float2) * N * tiles);
        z_target = c.take(sizeof(float) * N);
        if (!few && N) {
            hp = c.take(elem * N * kp);
            wp = c.take(elem * V * kp);
            h_scale = c.take(two ? sizeof(float) * N : 0);
            w_scale = c.take(two ? sizeof(float) * up_to(V, 256) : 0);
        }
        if (grad && N) {
            const int64_t words = std::min(piece, up_to(V, kBK));
            all = c.take(two ? elem * V * kp : 0);
            w_max = c.take(sizeof(float) * kMaxParts);
            up_max = c.take(sizeof(UpParts));
            hs = c.take(sizeof(uint16_t) * 2 * N * kp);  // in two parts, 16-bit rows too
            prob = c.take(elem * np * words);
            sum = c.take(piece < V ? sizeof(float) * N * D : 0);
            size_t sh = 0, sw = 0;
            if (D) {
                const int64_t left = V - (V - 1) / piece * piece;
                last_cuts = cuts_of(left);
                cuts = left < V ? cuts_of(piece) : last_cuts;
                sh = std::max(cuts.h.slab_bytes(), last_cuts.h.slab_bytes());
                sw = std::max(cuts.w.slab_bytes(), last_cuts.w.slab_bytes());
            }
            slabs_h = c.take(sh);
            slabs_w = c.take(sw);
        }
        bytes = c.used;
    }
};

// Whether the products can read rows of D elements where they are: whole, aligned
// ones of 16 bits.
bool whole_rows(int32_t type, int64_t D) { return type != TQ_F32 && D > 0 && D % kBK == 0; }
bool in_place(int32_t type, const void *p, int64_t ld, int64_t D)
{
    return whole_rows(type, D) && ld % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

template <class T, bool GRAD, bool TWO> int run_logits(LogitArgs a, int64_t tokens, hipStream_t s)
{
    const Cut c = cut_logits(a.p.a.extent, tokens);
    c.put(a.p);
    launch_exactly(c.blocks(), [&](dim3 grid, uint32_t first) {
        a.first = first;
        if (c.big) k_logits<T, Big, GRAD, TWO><<<grid, Big::threads, 0, s>>>(a);
        else k_logits<T, Small, GRAD, TWO><<<grid, Small::threads, 0, s>>>(a);
    });
    return c.m_tiles;
}

// Both products of a piece, in one launch if their tiles have one shape.
template <class T, class Out> void run_products(StoreArgs h, StoreArgs w, const Cuts &c, hipStream_t s)
{
    const Cut &ch = c.h, &cw = c.w;
    ch.put(h.p);
    cw.put(w.p);
    auto go = [&](auto shape, int hb, int wb, int ht, int wt) {
        using S = decltype(shape);
        launch_exactly((int64_t)hb + wb, [&](dim3 grid, uint32_t first) {
            k_products<T, S, Out><<<grid, S::threads, 0, s>>>(h, w, hb, first);
        });
        if (ht + wt) k_slabs<S, Out><<<dim3((unsigned)(ht + wt), S::BM * S::BN / 1024), 256, 0, s>>>(h, w, ht);
    };
    auto by_shape = [&](bool big, int hb, int wb, int ht, int wt) {
        if (big) go(Big{}, hb, wb, ht, wt);
        else go(Small{}, hb, wb, ht, wt);
    };
    if (ch.big == cw.big) by_shape(ch.big, ch.blocks(), cw.blocks(), ch.tail, cw.tail);
    else {
        by_shape(ch.big, ch.blocks(), 0, ch.tail, 0);
        by_shape(cw.big, 0, cw.blocks(), 0, cw.tail);
    }
}

template <class Out> void run_finish(const StoreArgs &a, hipStream_t s)
{
    k_finish<Out><<<dim3((unsigned)std::min<int64_t>(a.M, kGridX), (unsigned)ceil_div(a.N, 256)), 256, 0, s>>>(a);
}

// In: type of the arrays; T: of the products' operands; TWO: in two parts.
template <class In, class T, bool TWO> hipError_t xent_t(int32_t type, const XentArgs &a, bool grad, hipStream_t s)
{
    const bool h_in_place = in_place(type, a.hidden, a.ld_hidden, a.D);
    const bool w_in_place = in_place(type, a.weight, a.ld_weight, a.D);
    const XentPlan p(type, a.N, a.V, a.D, grad, w_in_place);
    char *ws = (char *)a.ws;
    float2 *part = (float2 *)(ws + p.part);
    float *z_target = (float *)(ws + p.z_target);
    const unsigned token_blocks = (unsigned)ceil_div(a.N, 4);
    if (p.few) {
        const int tiles = (int)ceil_div(a.V, kFewWords);
        FewArgs f{a.hidden, a.weight, a.ld_hidden, a.ld_weight, a.N, a.V, a.D, a.targets, part, z_target, tiles, 0};
        launch_exactly(tiles, [&](dim3 grid, uint32_t first) {
            f.first = first;
            if (a.N <= 16) k_few<In, 1><<<grid, 64 * kFewWaves, 0, s>>>(f);
            else if (a.N <= 32) k_few<In, 2><<<grid, 64 * kFewWaves, 0, s>>>(f);
            else k_few<In, 4><<<grid, 64 * kFewWaves, 0, s>>>(f);
        });
        const LseArgs l{part, tiles, a.N, a.V, a.targets, z_target, a.loss, a.lse};
        k_lse<In, T, TWO><<<grid_of(token_blocks), 256, 0, s>>>(l, (int)token_blocks, PackArgs{}, 0);
        return hipGetLastError();
    }
    if (a.N == 0) {
        // no tokens: no gradient
        StoreArgs e{};
        e.M = a.V;
        e.N = a.D;
        e.out = a.dweight;
        e.ld_out = a.ld_dweight;
        if (a.D) run_finish<In>(e, s);
        return hipGetLastError();
    }
    float *h_scale = (float *)(ws + p.h_scale), *w_scale = (float *)(ws + p.w_scale), *w_max = (float *)(ws + p.w_max);
    Operand h{ws + p.hp, p.kp, a.N * p.kp, a.N, 0}, w{ws + p.wp, p.kp, a.V * p.kp, a.V, 0};
    Operand w_all = w;  // for dhidden's product
    const bool back = grad && a.D > 0;
    UpParts *up_max = (UpParts *)(ws + p.up_max);
    const UpArgs u{a.upstream, TWO ? h_scale : nullptr, a.targets, a.N, a.V, up_max};
    if (TWO && back) w_all.p = ws + p.all;
    PackArgs k{};
    k.D = a.D;
    k.kp = p.kp;
    if (h_in_place) h.p = a.hidden, h.ld = a.ld_hidden;
    else {
        k.src = a.hidden, k.ld = a.ld_hidden, k.rows = a.N;
        k.dst = ws + p.hp, k.part = h.part, k.scale = h_scale;
        const int parts = TWO && back ? kMaxParts : 0;
        k_lay_hidden<In, T, TWO><<<grid_of((int64_t)token_blocks + parts), 256, 0, s>>>(
            k, (int)token_blocks, (const float *)a.weight, a.ld_weight, a.V, w_max, parts);
    }
    unsigned word_blocks = 0;
    if (w_in_place) w.p = a.weight, w.ld = a.ld_weight;
    else {
        word_blocks = (unsigned)ceil_div(a.V, 4);
        k.src = a.weight, k.ld = a.ld_weight, k.rows = a.V;
        k.dst = ws + p.wp, k.part = w.part, k.scale = w_scale;
        if (TWO && back) k.all = ws + p.all, k.w_max = w_max;
    }
    const int up_parts = back ? kUpParts : 0;
    if (word_blocks + up_parts)
        k_lay_weight<In, T, TWO><<<grid_of((int64_t)word_blocks + up_parts), 256, 0, s>>>(k, (int)word_blocks, u, up_parts);
    if (!TWO) w_all = w;
    LogitArgs l{};
    l.p.a = w;
    l.p.b = h;
    l.p.terms = p.terms;
    l.p.k_tiles = (int)(p.kp / kBK);
    l.word_scale = w_scale;
    l.token_scale = h_scale;
    l.targets = a.targets;
    l.V = a.V;
    l.N = a.N;
    l.part = part;
    l.z_target = z_target;
    const int tiles = run_logits<T, false, TWO>(l, a.N, s);
    const LseArgs sums{part, tiles, a.N, a.V, a.targets, z_target, a.loss, a.lse};
    const Operand hs{ws + p.hs, p.kp, a.N * p.kp, p.kp, a.N};
    PackArgs v{};
    v.src = a.hidden, v.ld = a.ld_hidden, v.rows = a.N, v.D = a.D;
    v.dst = ws + p.hs, v.kp = p.kp, v.part = hs.part;
    v.targets = a.targets, v.V = a.V, v.up = a.upstream, v.up_max = up_max;
    const int hs_blocks = back ? (int)token_blocks : 0;
    k_lse<In, T, TWO><<<grid_of((int64_t)token_blocks + hs_blocks), 256, 0, s>>>(sums, (int)token_blocks, v, hs_blocks);
    if (!back) return hipGetLastError();

    StoreArgs d{};  // dhidden
    d.M = a.N, d.N = a.D;
    d.slabs = (float *)(ws + p.slabs_h);
    d.sum = p.piece < a.V ? (float *)(ws + p.sum) : nullptr;
    d.out = a.dhidden, d.ld_out = a.ld_dhidden;
    d.up = a.upstream, d.targets = a.targets, d.V = a.V;
    d.w_max = TWO ? w_max : nullptr;
    for (int64_t v0 = 0; v0 < a.V; v0 += p.piece) {
        const int64_t words = std::min(p.piece, a.V - v0), kv = up_to(words, kBK);
        l.p.a.p = (const T *)w.p + v0 * w.ld;
        l.p.a.extent = words;
        l.word_scale = w_scale + v0;
        l.v_base = v0;
        l.lse = a.lse;
        l.prob = ws + p.prob;
        l.ld_prob = kv;
        l.prob_rows = p.np;
        l.prob_part = p.np * kv;
        run_logits<T, true, TWO>(l, p.np, s);
        d.p.a = Operand{ws + p.prob, kv, l.prob_part, a.N, 0};
        d.p.b = Operand{(const T *)w_all.p + v0 * w_all.ld, w_all.ld, w_all.part, TWO || w_all.ld == p.kp ? p.kp : a.D, words};
        d.p.terms = p.terms;
        d.p.k_tiles = (int)(kv / kBK);
        d.add = v0 > 0;
        StoreArgs e{};  // dweight
        e.M = words, e.N = a.D;
        e.slabs = (float *)(ws + p.slabs_w);
        e.out = (In *)a.dweight + v0 * a.ld_dweight, e.ld_out = a.ld_dweight;
        e.up_max = up_max;
        e.p.a = Operand{ws + p.prob, kv, l.prob_part, kv, p.np};
        e.p.b = hs;
        e.p.terms = p.terms;
        e.terms = TWO ? nullptr : &up_max->terms;
        e.p.k_tiles = (int)(p.np / kBK);
        run_products<T, In>(d, e, v0 + words < a.V ? p.cuts : p.last_cuts, s);
    }
    if (d.sum) run_finish<In>(d, s);
    return hipGetLastError();
}

} // namespace

size_t xent_workspace(int32_t type, int64_t N, int64_t V, int64_t D, bool grad)
{
    // where the weights lie is not known here: what either way of a call with few tokens takes
    const size_t laid_out = XentPlan(type, N, V, D, grad, false).bytes;
    return whole_rows(type, D) ? std::max(laid_out, XentPlan(type, N, V, D, grad, true).bytes) : laid_out;
}

hipError_t launch_xent(int32_t type, const XentArgs &a, bool grad, hipStream_t s)
{
    if (type == TQ_F32) return xent_t<float, _Float16, true>(type, a, grad, s);
    if (type == TQ_BF16) return xent_t<__bf16, __bf16, false>(type, a, grad, s);
    return xent_t<_Float16, _Float16, false>(type, a, grad, s);
}

} // namespace tq
