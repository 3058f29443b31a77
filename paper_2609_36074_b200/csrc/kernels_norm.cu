// Layer norm, forward and backward, for any width and alignment.
//
//   forward   y_ij = (x_ij - mu_i) r_i w_j + b_j,  mu_i = mean_j x_ij,  r_i = 1 / sqrt(mean_j (x_ij - mu_i)^2 + eps)
//   backward  h = (x - mu) r, g = dy w:  dx = r (g - mean_j g - h mean_j (g h)),  dw = sum_i dy h,  db = sum_i dy
//
// The variance is taken about the mean (a second look at the row in registers), so an offset far above the spread costs
// nothing.  Statistics and sums are FP32 within a row and a block, FP64 across blocks; y, dx, dw, db are rounded once.
//
// Rows that eight blocks hold are streamed through shared memory and read from HBM once (train_rows.cuh): forward, up to 65536
// elements of 2 bytes and 49152 of 4, or 49152 of any type read element by element (mode 2); gradient, up to 49152 aligned
// ones of 2 bytes (mode 0), else 32768.  Rows that begin anywhere (mode 1) lose up to 7 of these.  Wider ones, and calls without
// rows, take the plain kernels that come first here, which read a row two to three times, from L2 but for the first.
#include "train_rows.cuh"

namespace gemnlr {
namespace {

constexpr int kRowThreads = 256;

template <typename T, typename W>
__global__ void __launch_bounds__(kRowThreads)
k_norm_any(const T* __restrict__ x, int64_t ldx, const W* __restrict__ w, const W* __restrict__ b, int64_t n, int d,
           float eps, T* __restrict__ y, int64_t ldy, float* __restrict__ mean, float* __restrict__ rstd)
{
    __shared__ double sred[kRowThreads / 32];
    const double inv_d = 1.0 / (double)d;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T* xr = x + row * ldx;
        T* yr = y + row * ldy;
        double s[1];
        thread_sums<kRowThreads>(d, s, [&](int j, float (&p)[1]) { p[0] += to_f(xr[j]); });
        const float mu = (float)(block_sum<kRowThreads>(s[0], sred) * inv_d);
        thread_sums<kRowThreads>(d, s, [&](int j, float (&p)[1]) { const float c = to_f(xr[j]) - mu; p[0] += c * c; });
        const float r = 1.0f / sqrtf((float)(block_sum<kRowThreads>(s[0], sred) * inv_d) + eps);
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
    __shared__ double sred[kRowThreads / 32];
    const double inv_d = 1.0 / (double)d;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const T *xr = x + row * ldx, *gr = dy + row * lddy;
        const float mu = mean[row], r = rstd[row];
        double s[2];
        thread_sums<kRowThreads>(d, s, [&](int j, float (&p)[2]) {
            const float g = to_f(gr[j]) * (w ? to_f(w[j]) : 1.0f);
            p[0] += g;
            p[1] += g * ((to_f(xr[j]) - mu) * r);
        });
        const float c1 = (float)(block_sum<kRowThreads>(s[0], sred) * inv_d);
        const float c2 = (float)(block_sum<kRowThreads>(s[1], sred) * inv_d);
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
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= 2 * (int64_t)d) return;
    W* out = e < d ? dw : db;
    if (!out) return;
    double v = 0.0;
    for (int c = 0; c < records; ++c) v += (double)part[(size_t)c * 2 * d + e];
    out[e < d ? e : e - d] = from_f<W>((float)v);
}

// ---- streamed rows -----------------------------------------------------------------------------------------------

// Rows that a group works on at a time, so that their sums over the group run side by side: as many as the registers hold
// next to the weights, up to a warp a row.
__host__ __device__ constexpr int fwd_rows(int mode, int tpr, int epl)
{
    return tpr > 32 || epl > 24 || (epl > 16 && mode != 0) ? 1 : epl <= 8 ? 4 : 2;
}

template <typename T, int MODE, int TPR, int EPL, int C>
struct NormShape {
    using S0 = Source<T, MODE, TPR, EPL, C>;
    static constexpr int ROWS = fwd_rows(MODE, TPR, EPL), ROW = S0::stage_bytes(), STAGE = ROWS * ROW;
    static constexpr int MASKS = S0::L::mask_bytes(), STAGES = ring_stages(STAGE, MASKS), SHARED = STAGE * STAGES + MASKS;
};

// Forward.  HBM bounds it: 2 x 2 bytes an element of bf16 leave an SM some 22 instructions for each, of which it issues 11
// (packed FP32 pairs; weights in registers).  More rows in flight than two blocks' registers hold come from the ring (four
// stages).  What is read once leaves L2 first (262144 x 768: 151 us without, 144 us with the hints).
// Measured, 262144 x 768 bf16: 144 us, 5.6 TB/s (a device copy of the same bytes: 126 us); 60000 x 1001 bf16, rows that begin
// anywhere: 50 us, 4.8 TB/s, bound by issue (530 instructions a row and warp, 360 where rows are aligned).
template <typename T, int MODE, int TPR, int EPL, int C>
__global__ void __launch_bounds__(kRowBlock, 2)
k_norm_rows(const T* __restrict__ x, int64_t ldx, const void* __restrict__ w, const void* __restrict__ b, int wtype, int64_t n, int d,
            float eps, T* __restrict__ y, int64_t ldy, float* __restrict__ mean, float* __restrict__ rstd)
{
    using L = Lane<T, MODE, TPR, EPL, C>;
    using H = NormShape<T, MODE, TPR, EPL, C>;
    constexpr int R = H::ROWS, N = L::N, S = H::STAGES;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ Join<L, TPR, C, (TPR > 32 ? 3 : R), S> jn;
    __shared__ Edges<L> ed;
    uint32_t turn = 0, phase = 0;
    int at = 0;
    jn.begin();
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(ring);
    const L ln(d, x, ldx, ldy, ring0 + H::STAGE * S);
    const Source<T, MODE, TPR, EPL, C> xs(x, ldx, n, d);
    const bool lead = L::BULK && (int)threadIdx.x % TPR == 0;
    const uint32_t usual = xs.window_bytes(ln);
    const float inv_d = 1.0f / (float)d;
    const float head_spares = ln.head_spares(), tail_spares = ln.tail_spares();
    float warp_n = (float)d;                         // the row's elements that this warp has, where it has not all of them
    if constexpr (TPR > 32) {
        float c[1] = {0.0f};
        for (int k = 0; k < L::NV; ++k)
            for (int i = 0; i < N; ++i) c[0] += ln.holds(k, i);
        warp_all<SumOp, TPR>(c);
        warp_n = c[0];
    }
    const float inv_n = warp_n > 0.0f ? 1.0f / warp_n : 0.0f;
    const int64_t step = ln.groups();
    // the rows of the iteration that begins at `base`
    const auto send = [&](int64_t base, int stage) {
        if constexpr (L::BULK) {
            if (lead && (phase & 6) == 0 && base + ln.g < n) {
                const uint32_t bar = jn.stage(ln, stage);
                int skip[R];
                uint32_t bytes[R], all = 0;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int64_t row = base + r * step + ln.g;
                    bytes[r] = row < n ? xs.window(ln, row, usual, skip[r]) : 0u;
                    all += bytes[r];
                }
                expect_bytes(bar, all);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    xs.template send_bulk<true>(ln, base + r * step + ln.g, skip[r], bytes[r], ring0 + (uint32_t)(stage * H::STAGE + r * H::ROW), bar);
            }
        } else if constexpr (MODE != 2) {
            if (base < n)
#pragma unroll
                for (int r = 0; r < R; ++r) xs.send_own(ln, base + r * step + ln.g, ring0 + (uint32_t)(stage * H::STAGE + r * H::ROW));
            copies_end();
        }
    };
    for (int i = 0; i < S; ++i) {
#pragma unroll
        for (int r = 0; r < R; ++r) xs.prepare(ln, ring0 + (uint32_t)(i * H::STAGE + r * H::ROW), 0u);
        if (L::BULK || i < S - 1) send(ln.first_group() + i * R * step, i);
    }
    float2 w2[L::PAIRS], b2[L::PAIRS];
    load_weights<T>(ln, w, wtype, 1.0f, w2);
    load_weights<T>(ln, b, wtype, 0.0f, b2);
    for (int64_t base = ln.first_group(); base < n; base += R * step) {
        Row<T, MODE, EPL> xv[R];
        float2 sp[R];
        float s[R], mu[R];
        bool here = true;
        if constexpr (L::BULK) {
            if (base + ln.g < n) here = jn.row_ready(ln, at, phase);
        } else if constexpr (MODE != 2) {
            send(base + (S - 1) * R * step, at == 0 ? S - 1 : at - 1);
            copies_wait<S - 1>();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            xs.take(ln, base + r * step + ln.g, ring0 + (uint32_t)(at * H::STAGE + r * H::ROW), 0u, xv[r]);
            xv[r].mend_own(ln);
            float2 a = f2(here ? 0.0f : __int_as_float(0x7fffffff));
#pragma unroll
            for (int q = 0; q < L::PAIRS; ++q) a = __fadd2_rn(a, xv[r].pair(q));
            s[r] = a.x + a.y;
            if constexpr (MODE == 1) {
                sp[r] = xv[r].spares(ln);
                s[r] -= head_spares * sp[r].x + tail_spares * sp[r].y;
            }
        }
        warp_all<SumOp, TPR>(s);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mu[r] = s[r] * inv_n;                    // of the group's, or the warp's, elements
            const float2 m2 = f2(-mu[r]);
            float2 a = f2(0.0f);
#pragma unroll
            for (int k = 0; k < (MODE == 2 ? L::PAIRS : L::NV); ++k) {
                float2 b = f2(0.0f);
#pragma unroll
                for (int i = 0; i < (MODE == 2 ? 1 : N / 2); ++i) {
                    const int q = MODE == 2 ? k : k * (N / 2) + i;
                    float2 c = __fadd2_rn(xv[r].pair(q), m2);
                    if (MODE == 2) {
                        if (!ln.any(2 * q)) c.x = 0.0f;
                        if (!ln.any(2 * q + 1)) c.y = 0.0f;
                    }
                    b = __ffma2_rn(c, c, b);
                }
                if (MODE != 2 && !ln.any(k)) b = f2(0.0f);
                a = __fadd2_rn(a, b);
            }
            s[r] = a.x + a.y;
            if constexpr (MODE == 1) {
                const float ch = sp[r].x - mu[r], ct = sp[r].y - mu[r];
                s[r] -= head_spares * (ch * ch) + tail_spares * (ct * ct);
            }
        }
        warp_all<SumOp, TPR>(s);
        if constexpr (TPR > 32) {
            // each warp's count, mean and sum of squares about it, to the row's: the squares about the row's mean are the
            // warp's own and count (warp's mean - mean)^2.  One meeting of the group a row, and no cancellation.
            float v[3][2];
            const float mine[3] = {warp_n, mu[0], s[0]};
            group_join<TPR, C>(mine, v, jn, turn, phase);
            float t = v[0][0] * v[1][0] + v[0][1] * v[1][1];
            join_all<SumOp, TPR, C>(t);
            mu[0] = t * inv_d;
            const float c0 = v[1][0] - mu[0], c1 = v[1][1] - mu[0];
            t = v[2][0] + v[0][0] * (c0 * c0) + (v[2][1] + v[0][1] * (c1 * c1));
            join_all<SumOp, TPR, C>(t);
            s[0] = t;
        }
        if constexpr (L::BULK) send(base + S * R * step, at);    // every thread of the group has its part of the rows
        if (++at == S) { at = 0; phase ^= 1; }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = base + r * step + ln.g;
            const float rs = rsqrtf(s[r] * inv_d + eps);
            const float2 m2 = f2(-mu[r]), r2 = f2(rs);
#pragma unroll
            for (int q = 0; q < L::PAIRS; ++q)
                xv[r].set_pair(q, __ffma2_rn(__fmul2_rn(__fadd2_rn(xv[r].pair(q), m2), r2), w2[q], b2[q]));
            xv[r].template store<true>(ln, y, row, ldy, row < n, n, ed);
            if (ln.l == 0 && ln.rank == 0 && row < n) {
                if (mean) mean[row] = mu[r];
                if (rstd) rstd[row] = rs;
            }
        }
    }
    jn.land(ln, phase);
    leave_cluster<C>();
}

// Floats from one record to the next: 2 d, rounded up so that every record begins at a multiple of 16 bytes.
__host__ __device__ inline int64_t record_stride(int d) { return (2 * (int64_t)d + 3) & ~(int64_t)3; }

// The gradient.  Every thread keeps its columns' sums of dy h and dy over the rows that it sees (FP32), the block joins its
// groups' sums and writes one record; k_norm_dw_join adds the records (small calls: the blocks of the one cluster read each
// other's).  A row's mean and rstd are read a row ahead.  With 24 elements a thread the row is read from the ring a second
// time instead of being kept: sums and weights fill the registers (262144 x 768 bf16: 246 us when it was kept and spilled).
// Measured: 262144 x 768 bf16 198 us, 6.1 TB/s, HBM; 1021 x 16384 FP32, clusters of four blocks a row: 41.5 us, of which the
// rows take 33 and the join of 71 records of 131 KB 8; 60000 x 1001 bf16 85 us, bound by issue.
template <typename T, int MODE, int TPR, int EPL, int C>
struct GradShape {
    using S0 = Source<T, MODE, TPR, EPL, C>;
    static constexpr bool OWN = MODE != 2 && TPR < 32;
    static constexpr int ROW = S0::stage_bytes(), STAGE = 2 * ROW + (OWN ? 2 * 4 * kRowBlock : 0), MASKS = S0::L::mask_bytes();
    static constexpr int STAGES = ring_stages(STAGE, MASKS);
    static constexpr int SUMS = kRowBlock * EPL * 4;                                 // the columns' sums, after the ring's last use
    static constexpr int OWN_SUMS = C == 1 ? 2 * TPR * EPL * 4 : 0;                  // a block's record, where blocks read each other's
    static constexpr int SHARED = STAGE * STAGES + MASKS > SUMS + OWN_SUMS ? STAGE * STAGES + MASKS : SUMS + OWN_SUMS;
};

template <typename T, int MODE, int TPR, int EPL, int C>
__global__ void __launch_bounds__(kRowBlock, 2)
k_norm_grad_rows(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, const float* __restrict__ mean,
                 const float* __restrict__ rstd, const void* __restrict__ w, int wtype, int64_t n, int d, T* __restrict__ dx, int64_t lddx,
                 float* __restrict__ part, int one, void* __restrict__ dw, void* __restrict__ db)
{
    using L = Lane<T, MODE, TPR, EPL, C>;
    using H = GradShape<T, MODE, TPR, EPL, C>;
    constexpr int N = L::N, S = H::STAGES;
    constexpr bool AGAIN = L::BULK && EPL > 16;      // the row is read from the ring a second time: its registers hold sums
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ Join<L, TPR, C, 2, S> jn;
    __shared__ Edges<L> ed;
    uint32_t turn = 0, phase = 0;
    int at = 0;
    jn.begin();
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(ring);
    const L ln(d, x, ldx, lddx, ring0 + H::STAGE * S);
    const Source<T, MODE, TPR, EPL, C> xs(x, ldx, n, d), gs(dy, lddy, n, d);
    const uint32_t slot4 = ring0 + 2 * H::ROW + threadIdx.x * 4;
    const bool lead = L::BULK && (int)threadIdx.x % TPR == 0;
    const uint32_t usual = xs.window_bytes(ln);
    const float inv_d = 1.0f / (float)d;
    const int64_t step = ln.groups();
    const auto send = [&](int64_t row, int stage) {
        const uint32_t o = ring0 + (uint32_t)(stage * H::STAGE);
        if constexpr (L::BULK) {
            if (lead && (phase & 6) == 0 && row < n) {
                int sx, sg;
                const uint32_t bx = xs.window(ln, row, usual, sx), bg = gs.window(ln, row, usual, sg), bar = jn.stage(ln, stage);
                expect_bytes(bar, bx + bg);
                xs.template send_bulk<MODE == 0>(ln, row, sx, bx, o, bar);
                gs.template send_bulk<MODE == 0>(ln, row, sg, bg, o + H::ROW, bar);
            }
        } else if constexpr (MODE != 2) {
            if (row - ln.g < n) {
                xs.send_own(ln, row, o);
                gs.send_own(ln, row, o + H::ROW);
                copy4_ahead(slot4 + (uint32_t)(stage * H::STAGE), row < n ? mean + row : mean, row < n);
                copy4_ahead(slot4 + (uint32_t)(stage * H::STAGE) + 4 * kRowBlock, row < n ? rstd + row : rstd, row < n);
            }
            copies_end();
        }
    };
    for (int i = 0; i < S; ++i) {
        xs.prepare(ln, ring0 + (uint32_t)(i * H::STAGE), 0u);
        gs.prepare(ln, ring0 + (uint32_t)(i * H::STAGE + H::ROW), 0u);
        if (L::BULK || i < S - 1) send(ln.group() + i * step, i);
    }
    float2 w2[L::PAIRS], aw[L::PAIRS], ab[L::PAIRS];
    load_weights<T>(ln, w, wtype, 1.0f, w2);
#pragma unroll
    for (int q = 0; q < L::PAIRS; ++q) aw[q] = ab[q] = f2(0.0f);
    float mu_next = 0.0f, rs_next = 0.0f;
    if (!H::OWN && ln.group() < n) { mu_next = mean[ln.group()]; rs_next = rstd[ln.group()]; }
    for (int64_t base = ln.first_group(); base < n; base += step) {
        const int64_t row = base + ln.g;
        const uint32_t o = (uint32_t)(at * H::STAGE);
        Row<T, MODE, EPL> xv, gv;
        float mu = mu_next, rs = rs_next;
        bool here = true;
        if constexpr (L::BULK) {
            if (row < n) here = jn.row_ready(ln, at, phase);
        } else if constexpr (MODE != 2) {
            send(row + (S - 1) * step, at == 0 ? S - 1 : at - 1);
            copies_wait<S - 1>();
            mu = __uint_as_float(read4(slot4 + o));
            rs = __uint_as_float(read4(slot4 + o + 4 * kRowBlock));
        }
        if (!H::OWN && row + step < n) { mu_next = mean[row + step]; rs_next = rstd[row + step]; }
        xs.take(ln, row, ring0 + o, 0u, xv);
        gs.take(ln, row, ring0 + o + H::ROW, 0u, gv);
        xv.mend(ln, 0u);
        gv.mend(ln, 0u);
        if (row >= n) { xv.zero(); gv.zero(); mu = rs = 0.0f; }
        const float2 m2 = f2(-mu), r2 = f2(rs);
        float2 s0 = f2(here ? 0.0f : __int_as_float(0x7fffffff)), s1 = f2(0.0f);
#pragma unroll
        for (int q = 0; q < L::PAIRS; ++q) {
            const float2 g = gv.pair(q), t = __fmul2_rn(g, __fadd2_rn(xv.pair(q), m2));          // dy (x - mu)
            aw[q] = __ffma2_rn(t, r2, aw[q]);
            ab[q] = __fadd2_rn(ab[q], g);
            s0 = __ffma2_rn(g, w2[q], s0);
            s1 = __ffma2_rn(t, w2[q], s1);
        }
        float s[2] = {s0.x + s0.y, (s1.x + s1.y) * rs};
        group_sum<TPR, C>(s, jn, turn, phase);
        // every thread of the group is done with this row's stage, or (where it reads it again) with the one before
        if constexpr (L::BULK && !AGAIN) send(row + S * step, at);
        if constexpr (AGAIN) {
            if (base != ln.first_group()) send(row + (S - 1) * step, at == 0 ? S - 1 : at - 1);
        }
        if (dx) {
            // dx = r dy w - r c1 - (x - mu) r^2 c2
            const float2 c1 = f2(-rs * (s[0] * inv_d)), c2 = f2(-rs * rs * (s[1] * inv_d));
            if constexpr (AGAIN) {
                xs.take(ln, row, ring0 + o, 0u, xv);
                gs.take(ln, row, ring0 + o + H::ROW, 0u, gv);        // (what lies outside the row is not stored)
            }
#pragma unroll
            for (int q = 0; q < L::PAIRS; ++q) {
                const float2 gw = __fmul2_rn(gv.pair(q), w2[q]);
                xv.set_pair(q, __ffma2_rn(__fadd2_rn(xv.pair(q), m2), c2, __ffma2_rn(gw, r2, c1)));
            }
            xv.template store<MODE != 0>(ln, dx, row, lddx, row < n, n, ed);
        }
        if (++at == S) { at = 0; phase ^= 1; }
    }
    jn.land(ln, phase);
    leave_cluster<C>();
    if (!part && !one) return;
    next_may_start();
    copies_wait<0>();
    float* sums = reinterpret_cast<float*>(ring);
    float* rec = one ? sums + kRowBlock * EPL : part + (int64_t)(blockIdx.x / C) * record_stride(d);
    // whether one of the block's rows never came (after a meeting of the block): its sums are NaN then
    const auto lost = [&] {
        if constexpr (L::BULK) return *(volatile uint32_t*)&jn.row_lost != 0;
        else return false;
    };
    const float nan = __int_as_float(0x7fffffff);
    // the records of a grid that is one cluster, joined by its blocks (in block order, FP64)
    const auto join_one = [&] {
        if constexpr (C == 1) {
            cluster_barrier();
            const int blocks = (int)gridDim.x;
            for (int e = (int)(blockIdx.x * kRowBlock + threadIdx.x); e < 2 * d; e += blocks * kRowBlock) {
                const double v = from_all_blocks(rec + e, blocks);
                void* out = e < d ? dw : db;
                const int j = e < d ? e : e - d;
                if (out) {
                    if (wtype == GEM_NLR_F32) ((float*)out)[j] = (float)v;
                    else ((T*)out)[j] = from_f<T>((float)v);
                }
            }
            __syncwarp();
            cluster_barrier();
        }
    };
    if constexpr (L::GROUPS == 1) {
        // one group: through shared memory only to store neighbouring columns together
        const int from = ln.rank * (kRowBlock * EPL) - ln.s;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int q = 0; q < L::PAIRS; ++q) {
                const int p = 2 * q / N * (kRowBlock * N) + (int)threadIdx.x * N + 2 * q % N;
                const float2 a = which ? ab[q] : aw[q];
                if constexpr (N > 1) *reinterpret_cast<float2*>(sums + p) = a;
                else { sums[p] = a.x; sums[p + kRowBlock] = a.y; }
            }
            __syncthreads();
            const bool none = lost();
            for (int p = threadIdx.x; p < kRowBlock * EPL; p += kRowBlock) {
                const int e = from + p;
                if (e >= 0 && e < d) rec[which * d + e] = none ? nan : sums[p];
            }
        }
        if (one) join_one();
        return;
    }
    constexpr int W = TPR * EPL;                     // places of a group in `sums`
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < L::PAIRS; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = (2 * q + h) / N, i = (2 * q + h) % N;
                const float2 a = which ? ab[q] : aw[q];
                if (ln.holds(k, i)) sums[ln.g * W + ln.first(k) + i] = h ? a.y : a.x;
            }
        // in two steps where a row is narrower than the block: its threads share a column's groups
        constexpr int SPLIT = W < kRowBlock ? kRowBlock / W : 1, EACH = L::GROUPS / SPLIT;
        __syncthreads();
        const bool none = lost();
        for (int e = threadIdx.x % W; e < W; e += kRowBlock) {
            const int q0 = SPLIT > 1 ? (int)threadIdx.x / W * EACH : 0;
            float t = 0.0f;
            if (e < d)
#pragma unroll
                for (int q = 0; q < EACH; ++q) t += sums[(q0 + q) * W + e];
            if constexpr (SPLIT > 1) sums[q0 * W + e] = t;               // (only this thread reads that place)
            else if (e < d) rec[which * d + e] = none ? nan : t;
        }
        if constexpr (SPLIT > 1) {
            __syncthreads();
            if ((int)threadIdx.x < d) {
                float t = 0.0f;
#pragma unroll
                for (int q = 0; q < SPLIT; ++q) t += sums[q * EACH * W + threadIdx.x];
                rec[which * d + threadIdx.x] = none ? nan : t;
            }
        }
    }
    if (one) join_one();
}

// dw, db: 128 columns a block, four to a lane; the block's 32 warps share the records out.  Fixed order, FP64.
template <typename W>
__global__ void __launch_bounds__(1024)
k_norm_dw_join(const float* part, int records, int d, W* __restrict__ dw, W* __restrict__ db)
{
    __shared__ double s[32][128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 128 + lane * 4;
    const int64_t stride = record_stride(d);
    grid_ready();
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    if (e < stride) {
#pragma unroll 4
        for (int c = warp; c < records; c += 32) {
            const float4 x = *reinterpret_cast<const float4*>(part + c * stride + e);
            v[0] += (double)x.x;
            v[1] += (double)x.y;
            v[2] += (double)x.z;
            v[3] += (double)x.w;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[warp][lane * 4 + i] = v[i];
    __syncthreads();
    // thread (j, p): rows 4 p ... of column j; then the eight parts
    const int j = threadIdx.x & 127, p = threadIdx.x >> 7, o = blockIdx.x * 128 + j;
    double t = s[4 * p][j] + s[4 * p + 1][j] + s[4 * p + 2][j] + s[4 * p + 3][j];
    __syncthreads();
    s[p][j] = t;
    __syncthreads();
    if (p == 0 && o < 2 * d) {
        t = 0.0;
#pragma unroll
        for (int q = 0; q < 8; ++q) t += s[q][j];
        W* out = o < d ? dw : db;
        if (out) out[o < d ? o : o - d] = from_f<W>((float)t);
    }
}

// Records of partial sums: at most one a block (or cluster) of the widest grid for the width, at least the eight that spread()
// may round up to.
int norm_records(int64_t n, int32_t d)
{
    const int most = d <= 6144 ? 2 * kTrainSMs : d <= 12288 ? kTrainSMs : kTrainSMs / 2;
    return n > most ? most : n < 8 ? 8 : (int)n;
}

bool bad_rows(const void* p, int32_t type, int64_t ld) { return !p || !aligned_to(p, type_bytes(type)) || ld < 0; }

}  // namespace
}  // namespace gemnlr

using namespace gemnlr;

extern "C" int gem_nlr_layer_norm(const void* x_dev, int32_t type, int64_t ld_x, const void* weight_dev, const void* bias_dev,
                                  int32_t wtype, int64_t n, int32_t d, float eps, void* y_dev, int64_t ld_y, float* mean_dev,
                                  float* rstd_dev, void* cuda_stream)
{
    if (!type_bytes(type) || (wtype != type && wtype != GEM_NLR_F32) || n < 0 || d < 1 || d > kMaxColumns || !(eps >= 0.0f) ||
        isinf(eps))
        return GEM_NLR_E_INVALID;
    if (n == 0) return GEM_NLR_OK;
    if (bad_rows(x_dev, type, ld_x) || bad_rows(y_dev, type, ld_y) || ld_y < d || x_dev == y_dev ||
        !aligned_to(weight_dev, type_bytes(wtype)) || !aligned_to(bias_dev, type_bytes(wtype)) || !aligned_to(mean_dev, 4) ||
        !aligned_to(rstd_dev, 4))
        return GEM_NLR_E_INVALID;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int tb = type_bytes(type);
    const Matrix ms[2] = {{x_dev, ld_x}, {y_dev, ld_y}};
    const Lying lie = lying(ms, 2, n, d, tb);
    bool held = false;
    cudaError_t rc = cudaSuccess;
    by_mode(type, lie.mode, [&](auto t, auto mode) {
        using T = decltype(t);
        held = by_width<mode.value != 2 && sizeof(T) == 2 ? 16 : 8, mode.value != 2 && sizeof(T) == 2 ? 24 : 16, mode.value != 2 && sizeof(T) == 2 ? 32 : 24>(lie.mode == 1 ? (int64_t)d + 16 / tb - 1 : d, [&](auto tpr, auto epl, auto c) {
            constexpr auto k = k_norm_rows<T, mode.value, tpr.value, epl.value, c.value>;
            constexpr int shared = NormShape<T, mode.value, tpr.value, epl.value, c.value>::SHARED;
            const int cl = spread(n, kRowBlock / tpr.value, fwd_rows(mode.value, tpr.value, epl.value), lie.period, resident_clusters<k, c.value>(shared));
            rc = launch_rows(k, cl * c.value, c.value, shared, false, st, (const T*)x_dev, ld_x, weight_dev, bias_dev, (int)wtype, n, (int)d, eps,
                             (T*)y_dev, ld_y, mean_dev, rstd_dev);
        });
    });
    if (held) return told(rc);
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
    if (n < 0 || d < 1 || d > kMaxColumns || (n > 0 && one_cluster(n, d))) return 0;
    return (size_t)norm_records(n, d) * (size_t)record_stride(d) * sizeof(float);
}

extern "C" int gem_nlr_layer_norm_backward(const void* dy_dev, int64_t ld_dy, const void* x_dev, int64_t ld_x, int32_t type,
                                           const float* mean_dev, const float* rstd_dev, const void* weight_dev, int32_t wtype,
                                           int64_t n, int32_t d, void* dx_dev, int64_t ld_dx, void* dweight_dev, void* dbias_dev,
                                           void* scratch_dev, size_t scratch_bytes, void* cuda_stream)
{
    if (!type_bytes(type) || (wtype != type && wtype != GEM_NLR_F32) || n < 0 || d < 1 || d > kMaxColumns ||
        (!dx_dev && !dweight_dev && !dbias_dev))
        return GEM_NLR_E_INVALID;
    if (n > 0 && (bad_rows(dy_dev, type, ld_dy) || bad_rows(x_dev, type, ld_x) || !mean_dev || !rstd_dev ||
                  !aligned_to(mean_dev, 4) || !aligned_to(rstd_dev, 4) || (dx_dev && ld_dx < d) ||
                  !aligned_to(dx_dev, type_bytes(type)) || (dx_dev && (dx_dev == dy_dev || dx_dev == x_dev))))
        return GEM_NLR_E_INVALID;
    if (!aligned_to(weight_dev, type_bytes(wtype)) || !aligned_to(dweight_dev, type_bytes(wtype)) ||
        !aligned_to(dbias_dev, type_bytes(wtype)))
        return GEM_NLR_E_INVALID;
    const size_t need = gem_nlr_layer_norm_backward_scratch_bytes(n, d);
    if (need > 0 && (!scratch_dev || !aligned_to(scratch_dev, 256) || scratch_bytes < need))
        return GEM_NLR_E_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    float* part = (float*)scratch_dev;
    const int tb = type_bytes(type);
    const Matrix ms[3] = {{dy_dev, ld_dy}, {x_dev, ld_x}, {dx_dev, ld_dx}};
    const Lying lie = lying(ms, dx_dev ? 3 : 2, n, d, tb);
    const bool one = n > 0 && one_cluster(n, d) && (dweight_dev || dbias_dev);
    bool held = false;
    int rec = 0;
    cudaError_t err = cudaSuccess;
    if (n > 0)
        by_mode(type, lie.mode, [&](auto t, auto mode) {
            using T = decltype(t);
            held = by_width<mode.value != 2 && sizeof(T) == 2 ? 16 : 8, mode.value != 2 && sizeof(T) == 2 ? 16 : 12, mode.value == 0 && sizeof(T) == 2 ? 24 : 16>(lie.mode == 1 ? (int64_t)d + 16 / tb - 1 : d, [&](auto tpr, auto epl, auto c) {
                constexpr auto k = k_norm_grad_rows<T, mode.value, tpr.value, epl.value, c.value>;
                constexpr int shared = GradShape<T, mode.value, tpr.value, epl.value, c.value>::SHARED;
                const int most = resident_clusters<k, c.value>(shared), room = norm_records(n, d);
                rec = spread(n, kRowBlock / tpr.value, 1, lie.period, one ? kOneBlocks : most < room ? most : room);
                err = launch_rows(k, rec * c.value, one ? rec : c.value, shared, false, st, (const T*)dy_dev, ld_dy, (const T*)x_dev, ld_x, mean_dev, rstd_dev,
                                  weight_dev, (int)wtype, n, (int)d, (T*)dx_dev, ld_dx, (dweight_dev || dbias_dev) && !one ? part : nullptr, (int)one, dweight_dev, dbias_dev);
            });
        });
    if (held) {
        int rc = told(err);
        if (rc == GEM_NLR_OK && (dweight_dev || dbias_dev) && !one)
            rc = by_type(wtype, [&](auto t) {
                using W = decltype(t);
                return told(launch_early(k_norm_dw_join<W>, dim3((unsigned)((2 * (int64_t)d + 127) / 128)), 1024, st, (const float*)part, rec,
                                         (int)d, (W*)dweight_dev, (W*)dbias_dev));
            });
        return rc;
    }
    const int blocks = (int)(n < 148 * 8 ? n : 148 * 8), records = norm_records(n, d);
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
