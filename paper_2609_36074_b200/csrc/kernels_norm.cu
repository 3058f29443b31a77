// Layer norm, forward and backward, for any width and alignment.
//
//   forward   y_ij = (x_ij - mu_i) r_i w_j + b_j,  mu_i = mean_j x_ij,  r_i = 1 / sqrt(mean_j (x_ij - mu_i)^2 + eps)
//   backward  h = (x - mu) r, g = dy w:  dx = r (g - mean_j g - h mean_j (g h)),  dw = sum_i dy h,  db = sum_i dy
//
// The variance is taken about the mean (a second look at the row), so an offset far above the spread costs nothing.
#include "train_rows.cuh"

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

// ---- rows in registers -------------------------------------------------------------------------------------------

template <typename T, int N>
__device__ __forceinline__ void load_weights(const void* w, int wtype_f32, int e, float (&out)[N], float none)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        out[i] = !w ? none : wtype_f32 ? ((const float*)w)[e + i] : to_f(((const T*)w)[e + i]);
}

// rows in flight per group: about 48 registers of row, next to the weights
template <typename T> __host__ __device__ constexpr int fwd_rows(int tpr, int epl)
{
    return tpr >= 512 ? 1 : epl <= 16 && tpr <= 32 ? 4 : 2;
}

template <typename T, int VB, int TPR, int EPL>
__global__ void __launch_bounds__(block_of(TPR), TPR <= 256 ? 2 : 1)
k_norm_rows(const T* __restrict__ x, int64_t ldx, const void* __restrict__ w, const void* __restrict__ b, int w32, int64_t n, int d,
            float eps, T* __restrict__ y, int64_t ldy, float* __restrict__ mean, float* __restrict__ rstd)
{
    using V = Vec<T, VB>;
    constexpr int N = V::N, NV = EPL / N, R = fwd_rows<T>(TPR, EPL), NT = block_of(TPR), GROUPS = NT / TPR;
    constexpr bool KEEP = TPR <= 256;                 // the weights stay in registers; wider blocks have no room
    __shared__ float sred[group_floats(TPR, R)];
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const float inv_d = 1.0f / (float)d;
    float wr[KEEP ? NV : 1][N], br[KEEP ? NV : 1][N];
    if constexpr (KEEP) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int e = (v * TPR + l) * N;
            if (e < d) { load_weights<T, N>(w, w32, e, wr[v], 1.0f); load_weights<T, N>(b, w32, e, br[v], 0.0f); }
        }
    }
    for (int64_t base = (int64_t)blockIdx.x * GROUPS * R; base < n; base += (int64_t)gridDim.x * GROUPS * R) {
        V xv[R][NV];
        float s[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = base + r * GROUPS + g;
            const T* xr = x + row * ldx;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * TPR + l) * N;
                if (row < n && e < d) xv[r][v].load(xr + e); else xv[r][v].zero();
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[r] = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) s[r] += xv[r][v].get(i);
        }
        group_all<SumOp, TPR>(s, sred, turn);
        float mu[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mu[r] = s[r] * inv_d;
            s[r] = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if ((v * TPR + l) * N < d) {
#pragma unroll
                    for (int i = 0; i < N; ++i) { const float c = xv[r][v].get(i) - mu[r]; s[r] += c * c; }
                }
        }
        group_all<SumOp, TPR>(s, sred, turn);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = base + r * GROUPS + g;
            const float rs = 1.0f / sqrtf(s[r] * inv_d + eps);
            if (row < n) {
                T* yr = y + row * ldy;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int e = (v * TPR + l) * N;
                    if (e < d) {
                        float ww[N], bb[N];
                        if constexpr (!KEEP) { load_weights<T, N>(w, w32, e, ww, 1.0f); load_weights<T, N>(b, w32, e, bb, 0.0f); }
                        V o;
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const float h = (xv[r][v].get(i) - mu[r]) * rs;
                            o.set(i, KEEP ? h * wr[KEEP ? v : 0][i] + br[KEEP ? v : 0][i] : h * ww[i] + bb[i]);
                        }
                        o.store(yr + e);
                    }
                }
                if (l == 0) {
                    if (mean) mean[row] = mu[r];
                    if (rstd) rstd[row] = rs;
                }
            }
        }
    }
}

// The gradient.  Every thread keeps its columns' sums of dy h and dy over the rows that it sees (FP32), the block joins its
// groups' sums and writes one record; k_norm_dw_join adds the records.
template <typename T, int VB, int TPR, int EPL>
__global__ void __launch_bounds__(block_of(TPR), TPR <= 256 ? 2 : 1)
k_norm_grad_rows(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, const float* __restrict__ mean,
                 const float* __restrict__ rstd, const void* __restrict__ w, int w32, int64_t n, int d, T* __restrict__ dx, int64_t lddx,
                 float* __restrict__ part)
{
    using V = Vec<T, VB>;
    constexpr int N = V::N, NV = EPL / N, NT = block_of(TPR), GROUPS = NT / TPR;
    __shared__ float sred[group_floats(TPR, 2)];
    __shared__ float sums[GROUPS > 1 ? NT * EPL : 1];          // first the weights (one row), then the groups' sums
    int turn = 0;
    const int l = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const float inv_d = 1.0f / (float)d;
    float aw[NV][N], ab[NV][N];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < N; ++i) aw[v][i] = ab[v][i] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    V xv[NV], gv[NV];
    float mu = 0.0f, rs = 0.0f;
    const auto fetch = [&](int64_t row) {
        const bool ok = row < n;
        const T *xr = x + row * ldx, *gr = dy + row * lddy;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int e = (v * TPR + l) * N;
            if (ok && e < d) { xv[v].load(xr + e); gv[v].load(gr + e); } else { xv[v].zero(); gv[v].zero(); }
        }
        mu = ok ? mean[row] : 0.0f;
        rs = ok ? rstd[row] : 0.0f;
    };
    for (int64_t base = (int64_t)blockIdx.x * GROUPS; base < n; base += step) {
        const int64_t row = base + g;
        fetch(row);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int e = (v * TPR + l) * N;
            if (e < d) {
                float ww[N];
                load_weights<T, N>(w, w32, e, ww, 1.0f);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float gd = gv[v].get(i), h = (xv[v].get(i) - mu) * rs;
                    aw[v][i] += gd * h;
                    ab[v][i] += gd;
                    s[0] += gd * ww[i];
                    s[1] += gd * ww[i] * h;
                }
            }
        }
        if (!dx) continue;
        group_all<SumOp, TPR>(s, sred, turn);
        if (row < n) {
            const float c1 = s[0] * inv_d, c2 = s[1] * inv_d;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * TPR + l) * N;
                if (e < d) {
                    float ww[N];
                    load_weights<T, N>(w, w32, e, ww, 1.0f);
                    V o;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float h = (xv[v].get(i) - mu) * rs;
                        o.set(i, rs * (gv[v].get(i) * ww[i] - c1 - h * c2));
                    }
                    o.store(dx + row * lddx + e);
                }
            }
        }
    }
    if (!part) return;
    next_may_start();
    float* rec = part + (size_t)blockIdx.x * 2 * d;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (GROUPS > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) sums[g * (TPR * EPL) + (v * TPR + l) * N + i] = which ? ab[v][i] : aw[v][i];
            __syncthreads();
            for (int e = threadIdx.x; e < d; e += NT) {
                float t = 0.0f;
#pragma unroll
                for (int q = 0; q < GROUPS; ++q) t += sums[q * (TPR * EPL) + e];
                rec[which * d + e] = t;
            }
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * TPR + l) * N;
                if (e < d) {
#pragma unroll
                    for (int i = 0; i < N; ++i) rec[which * d + e + i] = which ? ab[v][i] : aw[v][i];
                }
            }
        }
    }
}

// dw, db: 32 columns a block, the records split over its 32 warps' lanes' rows, joined in a fixed order in FP64.
template <typename W>
__global__ void __launch_bounds__(1024)
k_norm_dw_join(const float* __restrict__ part, int records, int d, W* __restrict__ dw, W* __restrict__ db)
{
    __shared__ double s[32][33];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, e = blockIdx.x * 32 + tx;
    grid_ready();
    double v = 0.0;
    if (e < 2 * d)
        for (int c = ty; c < records; c += 32) v += (double)part[(size_t)c * 2 * d + e];
    s[ty][tx] = v;
    __syncthreads();
    // warp ty adds column ty's 32 partial sums
    v = warp_sum(s[tx][ty]);
    const int o = blockIdx.x * 32 + ty;
    if (tx == 0 && o < 2 * d) {
        W* out = o < d ? dw : db;
        if (out) out[o < d ? o : o - d] = from_f<W>((float)v);
    }
}

constexpr int kMaxRecords = 296;

int norm_records(int64_t n) { const int64_t r = n; return (int)(r < 1 ? 1 : r > kMaxRecords ? kMaxRecords : r); }

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
    const int tb = type_bytes(type), vx = vector_bytes(x_dev, ld_x, d, tb), vy = vector_bytes(y_dev, ld_y, d, tb);
    const int w32 = wtype == GEM_NLR_F32;
    bool held = false;
    by_vector(type, vx < vy ? vx : vy, [&](auto t, auto vb) {
        using T = decltype(t);
        held = by_width<1024>(d, [&](auto tpr, auto epl) {
            constexpr auto k = k_norm_rows<T, vb.value, tpr.value, epl.value>;
            constexpr int nt = block_of(tpr.value);
            constexpr int64_t rows = (int64_t)(nt / tpr.value) * fwd_rows<T>(tpr.value, epl.value);
            const int64_t all = resident_blocks<k>(nt), need = (n + rows - 1) / rows;
            k<<<(int)(need < all ? need : all), nt, 0, st>>>((const T*)x_dev, ld_x, weight_dev, bias_dev, w32, n, d, eps, (T*)y_dev, ld_y,
                                                             mean_dev, rstd_dev);
        });
    });
    if (held) return launched();
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
    const int tb = type_bytes(type), w32 = wtype == GEM_NLR_F32;
    int vb_all = vector_bytes(dy_dev, ld_dy, d, tb);
    const int vx = vector_bytes(x_dev, ld_x, d, tb), vdx = dx_dev ? vector_bytes(dx_dev, ld_dx, d, tb) : 16;
    if (vx < vb_all) vb_all = vx;
    if (vdx < vb_all) vb_all = vdx;
    bool held = false;
    int rec = 0;
    if (n > 0)
        by_vector(type, vb_all, [&](auto t, auto vb) {
            using T = decltype(t);
            held = by_width<512>(d, [&](auto tpr, auto epl) {
                constexpr auto k = k_norm_grad_rows<T, vb.value, tpr.value, epl.value>;
                constexpr int nt = block_of(tpr.value), groups = nt / tpr.value;
                int64_t all = resident_blocks<k>(nt), need = (n + groups - 1) / groups;
                if (all > kMaxRecords) all = kMaxRecords;
                rec = (int)(need < all ? need : all);
                k<<<rec, nt, 0, st>>>((const T*)dy_dev, ld_dy, (const T*)x_dev, ld_x, mean_dev, rstd_dev, weight_dev, w32, n, d,
                                      (T*)dx_dev, ld_dx, dweight_dev || dbias_dev ? part : nullptr);
            });
        });
    if (held) {
        int rc = launched();
        if (rc == GEM_NLR_OK && (dweight_dev || dbias_dev))
            rc = by_type(wtype, [&](auto t) {
                using W = decltype(t);
                return launch_early(k_norm_dw_join<W>, dim3((unsigned)((2 * (int64_t)d + 31) / 32)), 1024, st, (const float*)part, rec, (int)d,
                                    (W*)dweight_dev, (W*)dbias_dev) == cudaSuccess ? GEM_NLR_OK : GEM_NLR_E_CUDA;
            });
        return rc;
    }
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
