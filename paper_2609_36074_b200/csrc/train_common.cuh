// Shared by the training operators (layer norm, cross entropy, clipping): element types and argument checks.
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <atomic>
#include <type_traits>
#include "../../include/gem_nlr.h"
#include "device_utils.cuh"

namespace gemnlr {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

inline int type_bytes(int32_t type) { return type == GEM_NLR_F32 ? 4 : (type == GEM_NLR_F16 || type == GEM_NLR_BF16) ? 2 : 0; }
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Sums over a thread's terms of a row that a block of NT threads shares: in FP32 over 32 terms at a time, in FP64 beyond.
// (Terms that are alike round the same way: 2^17 of them in one FP32 sum are off by parts in a thousand.  Against one such sum,
// FP32: layer norm 64 x 70000 116 us and 118, its gradient 192 and 202, cross entropy 64 x 131073 173 and 198.)
template <int NT, int N, typename F>
__device__ __forceinline__ void thread_sums(int d, double (&sum)[N], F term)
{
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0;
    const auto strip = [&](int j, int terms) {
        float part[N] = {};
#pragma unroll 8
        for (int u = 0; u < terms; ++u) term(j + u * NT, part);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += (double)part[i];
    };
    int j = threadIdx.x;
    for (; j < d - 31 * NT; j += 32 * NT) strip(j, 32);
    if (j < d) strip(j, (d - j + NT - 1) / NT);
}

// Maximum over the block, the same value in every thread; sred: NT / 32 floats, reusable at once.
template <int NT>
__device__ __forceinline__ float block_max_f(float v, float* sred)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sred[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = sred[0];
#pragma unroll
    for (int w = 1; w < NT / 32; ++w) t = fmaxf(t, sred[w]);
    return t;
}

// Calls f with a value of the element type that `type` names (one of the three; checked before).
template <typename F> inline int by_type(int32_t type, F f)
{
    if (type == GEM_NLR_F32) return f(float{});
    if (type == GEM_NLR_F16) return f(__half{});
    return f(__nv_bfloat16{});
}

constexpr int kTrainSMs = 148, kTrainDevices = 64;

// Programmatic launches: the kernel before says that the next one may begin; that one waits for the kernel before to be
// complete (every block of it has to, or the kernel after it might begin before the first one is done).  What the kernel
// before writes is read through plain pointers: const __restrict__ says that nobody writes it while this kernel runs, and lets
// the compiler read it before the wait.
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_ready() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Columns of a row at most: int arithmetic on columns, steps included, stays far from its end.
constexpr int32_t kMaxColumns = 1 << 30;

inline int launched() { return cudaGetLastError() == cudaSuccess ? GEM_NLR_OK : GEM_NLR_E_CUDA; }

}  // namespace gemnlr
