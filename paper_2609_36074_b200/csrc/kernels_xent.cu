// Softmax cross entropy against int32 cluster labels, loss and gradient, for any number of clusters.
//
//   row_loss_i = log sum_j exp(z_ij - m_i) - (z_i,label - m_i),  m_i = max_j z_ij
//   dz_ij      = s (exp(z_ij - m_i) / sum - [j = label]),        s = 1 or 1 / (rows that count)
#include "train_rows.cuh"

namespace gemnlr {
namespace {

constexpr int kRowThreads = 256;
constexpr int kCountBlocks = 64;

constexpr int kMaxBlocks = kTrainSMs * 16;
struct Scratch {
    int64_t  counts[kCountBlocks];
    double   sums[kMaxBlocks];       // each block's sum of row losses
    uint32_t done;                   // blocks that have written theirs; k_count_labels sets it to 0
};

__global__ void __launch_bounds__(256)
k_count_labels(const int32_t* __restrict__ labels, int64_t n, Scratch* __restrict__ sc)
{
    __shared__ double sred[8];
    double c = 0.0;                                  // whole numbers: exact
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) c += labels[i] >= 0;
    c = block_sum<256>(c, sred);
    if (threadIdx.x == 0) sc->counts[blockIdx.x] = (int64_t)c;
    if (threadIdx.x == 0 && blockIdx.x == 0) sc->done = 0;
    next_may_start();
}

__device__ __forceinline__ int64_t rows_that_count(const Scratch* sc)
{
    int64_t c = 0;
    for (int b = 0; b < kCountBlocks; ++b) c += sc->counts[b];
    return c;
}

// Called once by every thread of every block with the row losses that it has seen: the last block to arrive adds the
// blocks' sums in block order.
template <int NT>
__device__ __forceinline__ void finish_loss(double mine, int mean, Scratch* sc, float* loss)
{
    __shared__ double sred[NT / 32];
    __shared__ bool last;
    const double v = block_sum<NT>(mine, sred);
    if (threadIdx.x == 0) {
        sc->sums[blockIdx.x] = v;
        __threadfence();
        last = atomicAdd(&sc->done, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double t = 0.0;
    for (int b = threadIdx.x; b < (int)gridDim.x; b += NT) t += ((volatile double*)sc->sums)[b];
    t = block_sum<NT>(t, sred);
    if (threadIdx.x == 0) {
        const int64_t c = mean ? rows_that_count(sc) : 1;
        *loss = (float)(c > 0 ? t / (double)c : 0.0);
    }
}

// s of the loss: 1, or 1 / (rows that count).  One thread reads the counts for the block.
__device__ __forceinline__ float loss_scale(const Scratch* sc, int mean)
{
    __shared__ float scale;
    if (threadIdx.x < 32) {
        float s = 1.0f;
        if (mean) {
            double c = 0.0;
            for (int b = threadIdx.x; b < kCountBlocks; b += 32) c += (double)sc->counts[b];
            c = warp_sum(c);
            s = c > 0.0 ? (float)(1.0 / c) : 0.0f;
        }
        if (threadIdx.x == 0) scale = s;
    }
    __syncthreads();
    return scale;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
k_xent_any(const T* z, int64_t ld, const int32_t* __restrict__ labels, int64_t n, int k, int mean,
           Scratch* sc, float* __restrict__ loss, float* __restrict__ row_loss, T* dz, int64_t ldd)
{
    __shared__ float sred[kRowThreads / 32];
    grid_ready();
    const float scale = loss_scale(sc, mean);
    double sum = 0.0;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* zr = z + row * ld;
        T* dr = dz ? dz + row * ldd : nullptr;
        const int lab = labels[row];
        if (lab < 0) {
            if (threadIdx.x == 0) row_loss[row] = 0.0f;
            if (dr) for (int j = threadIdx.x; j < k; j += kRowThreads) dr[j] = from_f<T>(0.0f);
            continue;
        }
        float m = -INFINITY;
        for (int j = threadIdx.x; j < k; j += kRowThreads) m = fmaxf(m, to_f(zr[j]));
        m = block_max_f<kRowThreads>(m, sred);
        const float base = m == -INFINITY ? 0.0f : m;           // nothing but -inf (or NaN): no -inf - -inf below
        float s = 0.0f;
        for (int j = threadIdx.x; j < k; j += kRowThreads) s += expf(to_f(zr[j]) - base);
        s = block_sum_f<kRowThreads>(s, sred);
        const float nan = __int_as_float(0x7fffffff);
        const float zl = lab < k ? to_f(zr[lab]) : nan;
        if (threadIdx.x == 0) {
            const float v = s == 0.0f ? (lab < k ? INFINITY : nan) : logf(s) - (zl - base);
            row_loss[row] = v;
            sum += (double)v;
        }
        if (!dr) continue;
        __syncthreads();                                         // every thread has the label's logit: dz may be z
        const float q = lab < k ? (s == 0.0f ? 0.0f : 1.0f / s) : nan;
        for (int j = threadIdx.x; j < k; j += kRowThreads) {
            float g = expf(to_f(zr[j]) - base) * q;
            if (j == lab && s != 0.0f) g -= 1.0f;
            dr[j] = from_f<T>(g * scale);
        }
    }
    finish_loss<kRowThreads>(sum, mean, sc, loss);
}

// ---- rows in registers -------------------------------------------------------------------------------------------

// Rows at a time per group: the exponentials (FP32) and the logits of all of them stay in registers.
__host__ __device__ constexpr int xent_rows(int tpr, int epl) { return tpr >= 512 ? 1 : epl <= 8 ? 4 : epl <= 16 ? 2 : 1; }

template <typename T, int VB, int TPR, int EPL>
__global__ void __launch_bounds__(block_of(TPR), TPR <= 256 ? 3 : TPR <= 512 ? 2 : 1)
k_xent_rows(const T* z, int64_t ld, const int32_t* __restrict__ labels, int64_t n, int k, int mean, Scratch* sc, float* __restrict__ loss,
            float* __restrict__ row_loss, T* dz, int64_t ldd)
{
    using V = Vec<T, VB>;
    constexpr int N = V::N, NV = EPL / N, R = xent_rows(TPR, EPL), NT = block_of(TPR), GROUPS = NT / TPR;
    constexpr float kLog2e = 1.4426950408889634f;
    __shared__ float sred[group_floats(TPR, R)];
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const float nan = __int_as_float(0x7fffffff);
    float scale = 0.0f;
    bool scaled = false;
    double sum = 0.0;
    for (int64_t base = (int64_t)blockIdx.x * GROUPS * R; base < n; base += (int64_t)gridDim.x * GROUPS * R) {
        V zv[R][NV];
        float m[R], s[R], zl[R];
        int lab[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = base + r * GROUPS + g;
            lab[r] = row < n ? labels[row] : -1;
            const T* zr = z + row * ld;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * TPR + l) * N;
                if (row < n && e < k) zv[r][v].load(zr + e);
            }
            zl[r] = lab[r] >= 0 && lab[r] < k ? to_f(zr[lab[r]]) : nan;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -INFINITY;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if ((v * TPR + l) * N < k) {
#pragma unroll
                    for (int i = 0; i < N; ++i) m[r] = fmaxf(m[r], zv[r][v].get(i));
                }
        }
        group_all<MaxOp, TPR>(m, sred, turn);
        float e_[R][NV][N];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (m[r] == -INFINITY) m[r] = 0.0f;              // nothing but -inf (or NaN): no -inf - -inf below
            s[r] = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if ((v * TPR + l) * N < k) {
#pragma unroll
                    for (int i = 0; i < N; ++i) { e_[r][v][i] = exp2f((zv[r][v].get(i) - m[r]) * kLog2e); s[r] += e_[r][v][i]; }
                }
        }
        group_all<SumOp, TPR>(s, sred, turn);
        if (!scaled) {                                        // the first rows are read while the labels are counted
            grid_ready();
            scale = loss_scale(sc, mean);
            scaled = true;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = base + r * GROUPS + g;
            if (row >= n) continue;
            const bool counts = lab[r] >= 0, known = lab[r] < k, empty = s[r] == 0.0f;
            if (l == 0) {
                const float v = !counts ? 0.0f : !known ? nan : empty ? INFINITY : logf(s[r]) - (zl[r] - m[r]);
                row_loss[row] = v;
                sum += (double)v;
            }
            if (!dz) continue;
            const float q = !known ? nan : empty ? 0.0f : 1.0f / s[r];
            const int hot = empty ? -1 : lab[r];
            T* dr = dz + row * ldd;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * TPR + l) * N;
                if (e < k) {
                    V o;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float p = e_[r][v][i] * q - (e + i == hot ? 1.0f : 0.0f);
                        o.set(i, counts ? p * scale : 0.0f);
                    }
                    o.store(dr + e);
                }
            }
        }
    }
    if (!scaled) grid_ready();
    finish_loss<NT>(sum, mean, sc, loss);
}

}  // namespace
}  // namespace gemnlr

using namespace gemnlr;

extern "C" size_t gem_nlr_label_cross_entropy_scratch_bytes(int64_t n, int32_t k)
{
    return n < 0 || k < 1 ? 0 : sizeof(Scratch);
}

extern "C" int gem_nlr_label_cross_entropy(const void* logits_dev, int32_t type, int64_t ld, const int32_t* labels_dev, int64_t n,
                                           int32_t k, int32_t mean, float* loss_dev, float* row_loss_dev, void* dlogits_dev,
                                           int64_t ld_d, void* scratch_dev, size_t scratch_bytes, void* cuda_stream)
{
    const int tb = type_bytes(type);
    if (!tb || n < 0 || k < 1 || (mean != 0 && mean != 1) || !loss_dev || !aligned_to(loss_dev, 4)) return GEM_NLR_E_INVALID;
    if (n > 0 && (!logits_dev || !aligned_to(logits_dev, tb) || ld < 0 || !labels_dev || !aligned_to(labels_dev, 4) ||
                  !row_loss_dev || !aligned_to(row_loss_dev, 4) || !aligned_to(dlogits_dev, tb) || (dlogits_dev && ld_d < k) ||
                  (dlogits_dev == logits_dev && ld != ld_d)))
        return GEM_NLR_E_INVALID;
    if (!scratch_dev || !aligned_to(scratch_dev, 256) || scratch_bytes < sizeof(Scratch)) return GEM_NLR_E_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    Scratch* sc = (Scratch*)scratch_dev;
    k_count_labels<<<kCountBlocks, 256, 0, st>>>(labels_dev, n, sc);
    if (launched() != GEM_NLR_OK) return GEM_NLR_E_CUDA;
    int vb_all = vector_bytes(logits_dev, ld, k, tb);
    const int vd = dlogits_dev ? vector_bytes(dlogits_dev, ld_d, k, tb) : 16;
    if (vd < vb_all) vb_all = vd;
    cudaError_t rc = cudaSuccess;
    by_vector(type, vb_all, [&](auto t, auto vb) {
        using T = decltype(t);
        const bool held = by_width<1024>(k, [&](auto tpr, auto epl) {
            constexpr auto kern = k_xent_rows<T, vb.value, tpr.value, epl.value>;
            constexpr int nt = block_of(tpr.value);
            constexpr int64_t rows = (int64_t)(nt / tpr.value) * xent_rows(tpr.value, epl.value);
            int64_t blocks = resident_blocks<kern>(nt);
            if (blocks > kMaxBlocks) blocks = kMaxBlocks;
            if (blocks > (n + rows - 1) / rows) blocks = (n + rows - 1) / rows;
            rc = launch_early(kern, dim3((unsigned)(blocks < 1 ? 1 : blocks)), nt, st, (const T*)logits_dev, ld, labels_dev, n, k, mean, sc,
                              loss_dev, row_loss_dev, (T*)dlogits_dev, ld_d);
        });
        if (!held) {
            const int64_t blocks = n < kTrainSMs * 8 ? n : kTrainSMs * 8;
            rc = launch_early(k_xent_any<T>, dim3((unsigned)(blocks < 1 ? 1 : blocks)), kRowThreads, st, (const T*)logits_dev, ld, labels_dev, n,
                              k, mean, sc, loss_dev, row_loss_dev, (T*)dlogits_dev, ld_d);
        }
    });
    return rc == cudaSuccess ? GEM_NLR_OK : GEM_NLR_E_CUDA;
}
