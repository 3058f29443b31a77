// Rows of a matrix in registers: the layout that the layer norm and cross entropy kernels share.
//
// A row of `d` elements belongs to a group of TPR threads (8 or 16 of a warp, a warp, or several), EPL elements to a thread, taken as vectors of VB bytes: vector v of thread l holds elements (v TPR + l) N ... + N - 1, N = VB /
// sizeof(T), so that a group's loads are contiguous.  The row is read once and stays in registers, still in its own type.
#pragma once
#include "train_common.cuh"

namespace gemnlr {

template <int VB> struct RawOf;
template <> struct RawOf<2> { using type = uint16_t; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<16> { using type = uint4; };

template <typename T, int VB>
struct Vec {
    static constexpr int N = VB / (int)sizeof(T);
    union {
        typename RawOf<VB>::type raw;
        T e[N];
    };
    __device__ __forceinline__ Vec() {}
    __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const typename RawOf<VB>::type*>(p); }
    __device__ __forceinline__ void zero() { raw = typename RawOf<VB>::type{}; }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<typename RawOf<VB>::type*>(p) = raw; }
    __device__ __forceinline__ void store_streaming(T* p) const { __stcs(reinterpret_cast<typename RawOf<VB>::type*>(p), raw); }
    __device__ __forceinline__ float get(int i) const { return to_f(e[i]); }
    __device__ __forceinline__ void set(int i, float v) { e[i] = from_f<T>(v); }
};

__host__ __device__ constexpr int block_of(int tpr) { return tpr <= 256 ? 256 : tpr; }

// Floats of shared memory that group_all needs for R values at a time.
__host__ __device__ constexpr int group_floats(int tpr, int r) { return tpr <= 32 ? 1 : 2 * r * block_of(tpr) / 32; }

// Sums (or maxima) of R values over the TPR threads of a group; every thread gets the same bits.  Where a group is more than
// a warp, its warps meet at a barrier of their own (number 1 + group); `turn` alternates between the halves of the group's
// part of `buf`, so that one barrier a call is enough: a thread that writes a half has passed the barrier that followed
// every thread's last reads of it.
struct SumOp { __device__ __forceinline__ static float of(float a, float b) { return a + b; } };
struct MaxOp { __device__ __forceinline__ static float of(float a, float b) { return fmaxf(a, b); } };

template <typename Op, int TPR, int R>
__device__ __forceinline__ void group_all(float (&v)[R], float* buf, int& turn)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = Op::of(v[r], __shfl_xor_sync(0xffffffffu, v[r], o));
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32, NT = block_of(TPR);
        const int g = threadIdx.x / TPR, warp = (threadIdx.x % TPR) >> 5, l = threadIdx.x & 31;
        float* b = buf + (g * 2 + turn) * R * W;
        turn ^= 1;
        if (l == 0)
#pragma unroll
            for (int r = 0; r < R; ++r) b[r * W + warp] = v[r];
        if constexpr (TPR == NT) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "n"(TPR) : "memory");
        // a warp's lanes take the warps' values and join them, instead of every thread reading all of them
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float t = b[r * W + (l & (W - 1))];
#pragma unroll
            for (int o = W / 2; o > 0; o >>= 1) t = Op::of(t, __shfl_xor_sync(0xffffffffu, t, o));
            v[r] = t;
        }
    }
}

// How a row of d elements is spread: f(TPR, EPL) as constants, with TPR EPL >= d and no more than 24 elements (32 where a
// full block is all there is) to a thread, which is what 128 registers hold next to weights or sums.  Returns false for a row wider than TMAX threads can hold.
template <int V> struct Const { static constexpr int value = V; };
template <int TMAX, typename F>
bool by_width(int64_t d, F f)
{
    if (d <= 64) f(Const<8>{}, Const<8>{});
    else if (d <= 128) f(Const<8>{}, Const<16>{});
    else if (d <= 256) f(Const<16>{}, Const<16>{});
    else if (d <= 512) f(Const<32>{}, Const<16>{});
    else if (d <= 768) f(Const<32>{}, Const<24>{});
    else if (d <= 1024) f(Const<64>{}, Const<16>{});
    else if (d <= 1536) f(Const<64>{}, Const<24>{});
    else if (d <= 2048) f(Const<128>{}, Const<16>{});
    else if (d <= 4096) f(Const<256>{}, Const<16>{});
    else if (d <= 8192) f(Const<512>{}, Const<16>{});
    else {
        if constexpr (TMAX >= 1024) {
            if (d <= 16384) { f(Const<1024>{}, Const<16>{}); return true; }
            if (d <= 32768) { f(Const<1024>{}, Const<32>{}); return true; }
        }
        return false;
    }
    return true;
}

// f(T, VB) for an element type and a vector width (as vector_bytes gives it)
template <typename F>
void by_vector(int32_t type, int vb, F f)
{
    by_type(type, [&](auto t) {
        using T = decltype(t);
        if (vb == 16) f(t, Const<16>{});
        else if (vb == 4 || sizeof(T) == 4) f(t, Const<4>{});
        else if constexpr (sizeof(T) == 2) f(t, Const<2>{});
        return 0;
    });
}

// Blocks of kernel K that fit the GPU at once (looked up once).
template <auto K>
int resident_blocks(int threads)
{
    static const int blocks = [&] {
        int per_sm = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, K, threads, 0) != cudaSuccess || per_sm < 1) per_sm = 1;
        return per_sm * kTrainSMs;
    }();
    return blocks;
}

// The widest vector that every row of a matrix can be read in: its address, its row distance and its width are multiples.
inline int vector_bytes(const void* p, int64_t ld, int64_t d, int tb)
{
    const uintptr_t all = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * tb) | (uintptr_t)(d * tb);
    return (all & 15) == 0 ? 16 : (all & 3) == 0 ? 4 : 2;
}

// Launch behind `st`'s last kernel that may begin while it ends (it waits for its results with grid_ready()).
template <typename... P, typename... A>
cudaError_t launch_early(void (*k)(P...), dim3 grid, int threads, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    cudaLaunchAttribute at = {};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k, (P)args...);
}

}  // namespace gemnlr
