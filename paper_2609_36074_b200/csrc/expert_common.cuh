// Shared by the expert layer's memory-bound kernels: eight neighbouring elements of a row at a time.
#pragma once
#include "train_common.cuh"

namespace gemnlr {

// Eight elements from p, as FP32; `many` of them are there (the others read as 0).  WIDE: all eight are, on 16 bytes.
template <bool WIDE, typename T>
__device__ __forceinline__ void load8(const T* __restrict__ p, int many, float (&v)[8])
{
    if constexpr (WIDE) {
        uint4 w[sizeof(T) / 2];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
        const T* t = reinterpret_cast<const T*>(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < many ? to_f(p[i]) : 0.f;
    }
}

template <bool WIDE, typename T>
__device__ __forceinline__ void store8(T* __restrict__ p, int many, const float (&v)[8])
{
    if constexpr (WIDE) {
        uint4 w[sizeof(T) / 2];
        T* t = reinterpret_cast<T*>(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = from_f<T>(v[i]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < many) p[i] = from_f<T>(v[i]);
    }
}

// Blocks of up to 256 threads over the vectors of rows (x, in equal steps, whole warps where there are many) and over rows (y).
struct RowBlocks { dim3 grid, block; };
inline RowBlocks row_blocks(int64_t n, int vecs)
{
    int x = 4;
    if (vecs > 16) {
        const int steps = (vecs + 255) / 256;
        x = ((vecs + steps - 1) / steps + 31) / 32 * 32;
    } else {
        while (x < vecs) x *= 2;
    }
    const int rows = 256 / x;
    const int64_t steps = (n + rows - 1) / rows, most = (int64_t)kTrainSMs * 64;
    return {dim3((unsigned)(steps < most ? steps : most)), dim3(x, rows)};
}

// Lets a kernel have `bytes` of shared memory, once on each device.
template <auto kern> inline cudaError_t allow_shared(int bytes)
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t rc = cudaGetDevice(&dev);
    if (rc != cudaSuccess) return rc;
    const uint64_t bit = dev < kTrainDevices ? 1ull << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    rc = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (rc == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return rc;
}

// Whether every row of a matrix begins on 16 bytes (absent ones count as such).
inline bool wide_rows(const void* p, int64_t ld, int bytes) { return !p || (aligned_to(p, 16) && ld % (16 / bytes) == 0); }

}  // namespace gemnlr
