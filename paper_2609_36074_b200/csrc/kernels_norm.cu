// Layer norm, forward and backward, for any width and alignment.
//
//   forward   y_ij = (x_ij - mu_i) r_i w_j + b_j,  mu_i = mean_j x_ij,  r_i = 1 / sqrt(mean_j (x_ij - mu_i)^2 + eps)
//   backward  h = (x - mu) r, g = dy w:  dx = r (g - mean_j g - h mean_j (g h)),  dw = sum_i dy h,  db = sum_i dy
//
// The variance is taken about the mean (a second look at the row), so an offset far above the spread costs nothing.
#include "train_common.cuh"

namespace gemnlr {
namespace {

constexpr int kRowThreads = 256;

template <typename T, typename W>
__global__ void __launch_bounds__(kRowThreads)
k_norm_any(const T* __restrict__ x, int64_t ldx, const W* __restrict__ w, const W* __restrict__ b, int64_t n, int d,
           float eps, T* __restrict__ y, int64_t ldy, float* __restrict__ mean, float* __restrict__ rstd)
{
    __shared__ float sred[kRowThreads / 32];
    const float inv_d = 1.0f / (float)d;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* xr = x + row * ldx;
        T* yr = y + row * ldy;
        float s = 0.0f;
        for (int j = threadIdx.x; j < d; j += kRowThreads) s += to_f(xr[j]);
        const float mu = block_sum_f<kRowThreads>(s, sred) * inv_d;
        s = 0.0f;
        for (int j = threadIdx.x; j < d; j += kRowThreads) { const float c = to_f(xr[j]) - mu; s += c * c; }
        const float r = 1.0f / sqrtf(block_sum_f<kRowThreads>(s, sred) * inv_d + eps);
        for (int j = threadIdx.x; j < d; j += kRowThreads) {
            const float h = (to_f(xr[j]) - mu) * r;
            yr[j] = from_f<T>(h * (w ? to_f(w[j]) : 1.0f) + (b ? to_f(b[j]) : 0.0f));
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

template <typename T, typename W>
__global__ void __launch_bounds__(kRowThreads)
k_norm_dx_any(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, const float* __restrict__ mean,
              const float* __restrict__ rstd, const W* __restrict__ w, int64_t n, int d, T* __restrict__ dx, int64_t lddx)
{
    __shared__ float sred[kRowThreads / 32];
    const float inv_d = 1.0f / (float)d;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T *xr = x + row * ldx, *gr = dy + row * lddy;
        const float mu = mean[row], r = rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int j = threadIdx.x; j < d; j += kRowThreads) {
            const float g = to_f(gr[j]) * (w ? to_f(w[j]) : 1.0f);
            s1 += g;
            s2 += g * ((to_f(xr[j]) - mu) * r);
        }
        const float c1 = block_sum_f<kRowThreads>(s1, sred) * inv_d;
        const float c2 = block_sum_f<kRowThreads>(s2, sred) * inv_d;
        for (int j = threadIdx.x; j < d; j += kRowThreads) {
            const float g = to_f(gr[j]) * (w ? to_f(w[j]) : 1.0f);
            dx[row * lddx + j] = from_f<T>(r * (g - c1 - (to_f(xr[j]) - mu) * r * c2));
        }
    }
}

// Partial sums over the rows: block (bx, by) takes 32 columns and the rows by * 8 + ty, ... ; one FP32 record of 2 d
// values per by.
template <typename T>
__global__ void __launch_bounds__(256)
k_norm_dw_any(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, const float* __restrict__ mean,
              const float* __restrict__ rstd, int64_t n, int d, float* __restrict__ part)
{
    __shared__ float sw[8][32], sb[8][32];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, j = blockIdx.x * 32 + tx;
    float aw = 0.0f, ab = 0.0f;
    if (j < d)
        for (int64_t row = (int64_t)blockIdx.y * 8 + ty; row < n; row += (int64_t)gridDim.y * 8) {
            const float g = to_f(dy[row * lddy + j]);
            aw += g * ((to_f(x[row * ldx + j]) - mean[row]) * rstd[row]);
            ab += g;
        }
    sw[ty][tx] = aw;
    sb[ty][tx] = ab;
    __syncthreads();
    if (ty == 0 && j < d) {
        for (int t = 1; t < 8; ++t) { aw += sw[t][tx]; ab += sb[t][tx]; }
        part[(size_t)blockIdx.y * 2 * d + j] = aw;
        part[(size_t)blockIdx.y * 2 * d + d + j] = ab;
    }
}

// dw, db from the records, in record order, in FP64
template <typename W>
__global__ void __launch_bounds__(256)
k_norm_dw_sum(const float* __restrict__ part, int records, int d, W* __restrict__ dw, W* __restrict__ db)
{
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e >= 2 * d) return;
    W* out = e < d ? dw : db;
    if (!out) return;
    double v = 0.0;
    for (int c = 0; c < records; ++c) v += (double)part[(size_t)c * 2 * d + e];
    out[e < d ? e : e - d] = from_f<W>((float)v);
}

constexpr int kMaxRecords = 296;

int norm_records(int64_t n) { const int64_t r = (n + 7) / 8; return (int)(r < 1 ? 1 : r > kMaxRecords ? kMaxRecords : r); }

bool bad_rows(const void* p, int32_t type, int64_t ld) { return !p || !aligned_to(p, type_bytes(type)) || ld < 0; }

}  // namespace
}  // namespace gemnlr

using namespace gemnlr;

extern "C" int gem_nlr_layer_norm(const void* x_dev, int32_t type, int64_t ld_x, const void* weight_dev, const void* bias_dev,
                                  int32_t wtype, int64_t n, int32_t d, float eps, void* y_dev, int64_t ld_y, float* mean_dev,
                                  float* rstd_dev, void* cuda_stream)
{
    if (!type_bytes(type) || (wtype != type && wtype != GEM_NLR_F32) || n < 0 || d < 1 || !(eps >= 0.0f) || isinf(eps))
        return GEM_NLR_E_INVALID;
    if (n == 0) return GEM_NLR_OK;
    if (bad_rows(x_dev, type, ld_x) || bad_rows(y_dev, type, ld_y) || ld_y < d || x_dev == y_dev ||
        !aligned_to(weight_dev, type_bytes(wtype)) || !aligned_to(bias_dev, type_bytes(wtype)) || !aligned_to(mean_dev, 4) ||
        !aligned_to(rstd_dev, 4))
        return GEM_NLR_E_INVALID;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int blocks = (int)(n < 148 * 8 ? n : 148 * 8);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        if (wtype == GEM_NLR_F32)
            k_norm_any<T, float><<<blocks, kRowThreads, 0, st>>>((const T*)x_dev, ld_x, (const float*)weight_dev,
                (const float*)bias_dev, n, d, eps, (T*)y_dev, ld_y, mean_dev, rstd_dev);
        else
            k_norm_any<T, T><<<blocks, kRowThreads, 0, st>>>((const T*)x_dev, ld_x, (const T*)weight_dev,
                (const T*)bias_dev, n, d, eps, (T*)y_dev, ld_y, mean_dev, rstd_dev);
        return launched();
    });
}

extern "C" size_t gem_nlr_layer_norm_backward_scratch_bytes(int64_t n, int32_t d)
{
    if (n < 0 || d < 1) return 0;
    return (size_t)norm_records(n) * 2 * (size_t)d * sizeof(float);
}

extern "C" int gem_nlr_layer_norm_backward(const void* dy_dev, int64_t ld_dy, const void* x_dev, int64_t ld_x, int32_t type,
                                           const float* mean_dev, const float* rstd_dev, const void* weight_dev, int32_t wtype,
                                           int64_t n, int32_t d, void* dx_dev, int64_t ld_dx, void* dweight_dev, void* dbias_dev,
                                           void* scratch_dev, size_t scratch_bytes, void* cuda_stream)
{
    if (!type_bytes(type) || (wtype != type && wtype != GEM_NLR_F32) || n < 0 || d < 1 || (!dx_dev && !dweight_dev && !dbias_dev))
        return GEM_NLR_E_INVALID;
    if (n > 0 && (bad_rows(dy_dev, type, ld_dy) || bad_rows(x_dev, type, ld_x) || !mean_dev || !rstd_dev ||
                  !aligned_to(mean_dev, 4) || !aligned_to(rstd_dev, 4) || (dx_dev && ld_dx < d) ||
                  !aligned_to(dx_dev, type_bytes(type)) || (dx_dev && (dx_dev == dy_dev || dx_dev == x_dev))))
        return GEM_NLR_E_INVALID;
    if (!aligned_to(weight_dev, type_bytes(wtype)) || !aligned_to(dweight_dev, type_bytes(wtype)) ||
        !aligned_to(dbias_dev, type_bytes(wtype)))
        return GEM_NLR_E_INVALID;
    if (!scratch_dev || !aligned_to(scratch_dev, 256) || scratch_bytes < gem_nlr_layer_norm_backward_scratch_bytes(n, d))
        return GEM_NLR_E_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    float* part = (float*)scratch_dev;
    const int blocks = (int)(n < 148 * 8 ? n : 148 * 8), records = norm_records(n);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const T *dy = (const T*)dy_dev, *x = (const T*)x_dev;
        if (dx_dev && n > 0) {
            if (wtype == GEM_NLR_F32)
                k_norm_dx_any<T, float><<<blocks, kRowThreads, 0, st>>>(dy, ld_dy, x, ld_x, mean_dev, rstd_dev,
                    (const float*)weight_dev, n, d, (T*)dx_dev, ld_dx);
            else
                k_norm_dx_any<T, T><<<blocks, kRowThreads, 0, st>>>(dy, ld_dy, x, ld_x, mean_dev, rstd_dev,
                    (const T*)weight_dev, n, d, (T*)dx_dev, ld_dx);
        }
        if (dweight_dev || dbias_dev) {
            k_norm_dw_any<T><<<dim3((d + 31) / 32, records), 256, 0, st>>>(dy, ld_dy, x, ld_x, mean_dev, rstd_dev, n, d, part);
            const int fin = (int)((2 * (int64_t)d + 255) / 256);
            if (wtype == GEM_NLR_F32)
                k_norm_dw_sum<float><<<fin, 256, 0, st>>>(part, records, d, (float*)dweight_dev, (float*)dbias_dev);
            else
                k_norm_dw_sum<T><<<fin, 256, 0, st>>>(part, records, d, (T*)dweight_dev, (T*)dbias_dev);
        }
        return launched();
    });
}
