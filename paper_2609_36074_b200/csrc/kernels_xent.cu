// Softmax cross entropy against int32 cluster labels, loss and gradient, for any number of clusters.
//
//   row_loss_i = log sum_j exp(z_ij - m_i) - (z_i,label - m_i),  m_i = max_j z_ij
//   dz_ij      = s (exp(z_ij - m_i) / sum - [j = label]),        s = 1 or 1 / (rows that count)
#include "train_common.cuh"

namespace gemnlr {
namespace {

constexpr int kRowThreads = 256;
constexpr int kCountBlocks = 64;

struct Scratch {
    int64_t counts[kCountBlocks];
};

__global__ void __launch_bounds__(256)
k_count_labels(const int32_t* __restrict__ labels, int64_t n, Scratch* __restrict__ sc)
{
    __shared__ double sred[8];
    double c = 0.0;                                  // whole numbers: exact
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) c += labels[i] >= 0;
    c = block_sum<256>(c, sred);
    if (threadIdx.x == 0) sc->counts[blockIdx.x] = (int64_t)c;
}

__device__ __forceinline__ float loss_scale(const Scratch* sc, int mean)
{
    if (!mean) return 1.0f;
    int64_t c = 0;
    for (int b = 0; b < kCountBlocks; ++b) c += sc->counts[b];
    return c > 0 ? (float)(1.0 / (double)c) : 0.0f;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
k_xent_any(const T* z, int64_t ld, const int32_t* __restrict__ labels, int64_t n, int k, int mean,
           const Scratch* __restrict__ sc, float* __restrict__ row_loss, T* dz, int64_t ldd)
{
    __shared__ float sred[kRowThreads / 32];
    const float scale = loss_scale(sc, mean);
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
        if (threadIdx.x == 0) row_loss[row] = s == 0.0f ? (lab < k ? INFINITY : nan) : logf(s) - (zl - base);
        if (!dr) continue;
        __syncthreads();                                         // every thread has the label's logit: dz may be z
        const float q = lab < k ? (s == 0.0f ? 0.0f : 1.0f / s) : nan;
        for (int j = threadIdx.x; j < k; j += kRowThreads) {
            float g = expf(to_f(zr[j]) - base) * q;
            if (j == lab && s != 0.0f) g -= 1.0f;
            dr[j] = from_f<T>(g * scale);
        }
    }
}

__global__ void __launch_bounds__(1024)
k_xent_sum(const float* __restrict__ row_loss, int64_t n, int mean, const Scratch* __restrict__ sc, float* __restrict__ loss)
{
    __shared__ double sred[32];
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) v += (double)row_loss[i];
    v = block_sum<1024>(v, sred);
    if (threadIdx.x == 0) {
        int64_t c = 0;
        for (int b = 0; b < kCountBlocks; ++b) c += sc->counts[b];
        *loss = (float)(mean ? (c > 0 ? v / (double)c : 0.0) : v);
    }
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
    if (n > 0) {
        const int blocks = (int)(n < 148 * 8 ? n : 148 * 8);
        by_type(type, [&](auto t) {
            using T = decltype(t);
            k_xent_any<T><<<blocks, kRowThreads, 0, st>>>((const T*)logits_dev, ld, labels_dev, n, k, mean, sc, row_loss_dev,
                                                          (T*)dlogits_dev, ld_d);
            return 0;
        });
    }
    k_xent_sum<<<1, 1024, 0, st>>>(row_loss_dev, n, mean, sc, loss_dev);
    return launched();
}
