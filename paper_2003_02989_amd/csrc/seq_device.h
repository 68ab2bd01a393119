// seq_device.h -- element types and vector access of the sequence kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace tq {

// A launch has fewer than 2^32 threads along x: from kGridX workgroups on (of at
// most 1024 threads) they go on along y.
constexpr unsigned kGridX = 1 << 21;

// In one launch, the last row of which may be past the end: the kernel returns in
// those workgroups before it reads or writes anything.
inline dim3 grid_of(int64_t blocks)
{
    if (blocks <= kGridX) return dim3((unsigned)blocks);
    return dim3(kGridX, (unsigned)((blocks + kGridX - 1) / kGridX));
}
// In whole rows and a rest, each calling go(grid, number of its first workgroup):
// no workgroup is past the end, which small kernels would wait for their arguments
// to find out (0.3 us).
template <class F> void launch_exactly(int64_t blocks, F &&go)
{
    const int64_t rows = blocks / kGridX, rest = blocks % kGridX;
    if (rows) go(dim3(kGridX, (unsigned)rows), (uint32_t)0);
    if (rest) go(dim3((unsigned)rest), (uint32_t)(rows * kGridX));
}

// The number of a workgroup within a launch of either kind, below 2^32.
__device__ __forceinline__ uint32_t block_of() { return blockIdx.y * kGridX + blockIdx.x; }

// Elements per 16-byte access.
template <class T> constexpr int kVec = 16 / (int)sizeof(T);

// N elements at p, which needs the alignment of one element only: gfx950 reads
// and writes global memory at any address, so that odd widths and strides take
// the same wide accesses as even ones.
template <int N, class T> __device__ __forceinline__ void load_vec(const T *p, float (&f)[N])
{
    T r[N];
    __builtin_memcpy(r, p, sizeof r);
#pragma unroll
    for (int i = 0; i < N; i++) f[i] = (float)r[i];
}

template <int N, class T> __device__ __forceinline__ void store_vec(T *p, const float (&f)[N])
{
    T r[N];
#pragma unroll
    for (int i = 0; i < N; i++) r[i] = (T)f[i];
    __builtin_memcpy(p, r, sizeof r);
}

// The first n (0..N) of N elements; the others read as zero.
template <int N, class T> __device__ __forceinline__ void load_part(const T *p, int n, float (&f)[N])
{
    if (n >= N) {
        load_vec<N>(p, f);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; i++) f[i] = i < n ? (float)p[i] : 0.f;
}

template <int N, class T> __device__ __forceinline__ void store_part(T *p, int n, const float (&f)[N])
{
    if (n >= N) {
        store_vec<N>(p, f);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; i++)
        if (i < n) p[i] = (T)f[i];
}

// Sum over the aligned group of L lanes (a power of two) a lane is in.
template <int L> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

} // namespace tq
