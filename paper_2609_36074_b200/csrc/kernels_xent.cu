// Softmax cross entropy against int32 cluster labels, loss and gradient, for any number of clusters.
//
//   row_loss_i = log sum_j exp(z_ij - m_i) - (z_i,label - m_i),  m_i = max_j z_ij
//   dz_ij      = s (exp(z_ij - m_i) / sum - [j = label]),        s = 1 or 1 / (rows that count)
//
// A row is read from HBM once and its gradient written once; its exponentials stay in registers (FP32).  A warp takes the
// exponentials about its own maximum, so that the warps of a wide row have to meet once, with a maximum and a sum each,
// and not once for the maximum and once for the sum.  The mean's divisor is counted by a small kernel before, whose end the
// first rows do not wait for; the loss is added up in FP64 by the last block, in block order.  Rows wider than eight blocks
// hold (65536 elements of 2 bytes, 49152 of 4 or of any type read element by element; rows that begin anywhere lose up to 7 of
// these) take the plain kernel, which reads them three times.
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

// The same in a grid that is one cluster; `slot`: the block's shared memory.
__device__ __forceinline__ void finish_loss_one(double mine, int mean, int64_t counted, double* slot, float* loss)
{
    __shared__ double sred[kRowBlock / 32];
    const double v = block_sum<kRowBlock>(mine, sred);
    if (threadIdx.x == 0) *slot = v;
    __syncwarp();
    cluster_barrier();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const double t = from_all_blocks(slot, (int)gridDim.x);
        *loss = (float)(!mean ? t : counted > 0 ? t / (double)counted : 0.0);
    }
    __syncwarp();
    cluster_barrier();
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
    __shared__ double dred[kRowThreads / 32];
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
        double total[1];
        thread_sums<kRowThreads>(k, total, [&](int j, float (&p)[1]) { p[0] += expf(to_f(zr[j]) - base); });
        const float s = (float)block_sum<kRowThreads>(total[0], dred);
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

// ---- streamed rows -----------------------------------------------------------------------------------------------

// Rows that a group works on at a time: two or four of the narrow ones.
__host__ __device__ constexpr int xent_rows(int tpr, int epl) { return tpr >= 32 ? 1 : epl <= 8 ? 4 : 2; }

template <typename T, int MODE, int TPR, int EPL, int C>
struct XentShape {
    using S0 = Source<T, MODE, TPR, EPL, C>;
    static constexpr bool OWN = MODE != 2 && TPR < 32;
    static constexpr int ROWS = xent_rows(TPR, EPL), ROW = S0::stage_bytes() + (OWN ? 4 * kRowBlock : 0);       // rows and, if OWN, labels
    static constexpr int STAGE = ROWS * ROW, MASKS = S0::L::mask_bytes(), STAGES = ring_stages(STAGE, MASKS), SHARED = STAGE * STAGES + MASKS;
};

// -inf in every element of a word
template <typename T> __device__ __forceinline__ uint32_t minus_infinity();
template <> __device__ __forceinline__ uint32_t minus_infinity<float>() { return 0xff800000u; }
template <> __device__ __forceinline__ uint32_t minus_infinity<__half>() { return 0xfc00fc00u; }
template <> __device__ __forceinline__ uint32_t minus_infinity<__nv_bfloat16>() { return 0xff80ff80u; }

// 2^x to 2 ulp, 0 below FP32's normal range: the exponentials are weights beside a largest one of 1
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// Largest element of a thread's part of a row (NaNs are passed over: they show in the sum); two at a time in 16-bit types.
template <typename T, int MODE, int EPL>
__device__ __forceinline__ float row_max(const Row<T, MODE, EPL>& z)
{
    using R = Row<T, MODE, EPL>;
    if constexpr (sizeof(T) == 2 && MODE != 2) {
        using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        T2 m = *reinterpret_cast<const T2*>(&z.v[0].w[0]);
#pragma unroll
        for (int k = 0; k < R::NV; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = __hmax2(m, *reinterpret_cast<const T2*>(&z.v[k].w[i]));
        return fmaxf(to_f(m.x), to_f(m.y));
    } else {
        float m = -INFINITY;
#pragma unroll
        for (int q = 0; q < EPL / 2; ++q) { const float2 p = z.pair(q); m = fmaxf(fmaxf(m, p.x), p.y); }
        return m;
    }
}

// Measured: 131072 x 1000 bf16 92 us, 5.7 TB/s (issue 60 %, 13 instructions an element); 2053 x 32768 f16, four blocks a row:
// 64.5 us, 4.2 TB/s, bound by the chain of a row (maximum, sum, meeting, output) at two blocks an SM: a block begins the
// next row before it ends one (67 us without); 16 x 100 FP32, one launch: 3.6 us on the device.
template <typename T, int MODE, int TPR, int EPL, int C>
__global__ void __launch_bounds__(kRowBlock, 2)
k_xent_rows(const T* z, int64_t ld, const int32_t* __restrict__ labels, int64_t n, int k, int mean, Scratch* sc, float* __restrict__ loss,
            float* __restrict__ row_loss, T* dz, int64_t ldd, int one)
{
    using L = Lane<T, MODE, TPR, EPL, C>;
    using H = XentShape<T, MODE, TPR, EPL, C>;
    constexpr int N = L::N, R = H::ROWS, S = H::STAGES;
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ Join<L, TPR, C, (TPR > 32 ? 2 : R), S, (C > 1 ? 4 : 2)> jn;
    __shared__ Edges<L> ed;
    uint32_t turn = 0, sent = 0, phase = 0;
    int at = 0;
    jn.begin();
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(ring);
    const L ln(k, z, ld, ldd, ring0 + H::STAGE * S);
    const Source<T, MODE, TPR, EPL, C> zs(z, ld, n, k);
    const uint32_t slot4 = ring0 + H::S0::stage_bytes() + threadIdx.x * 4;
    const bool lead = L::BULK && (int)threadIdx.x % TPR == 0;
    const uint32_t usual = zs.window_bytes(ln);
    const float nan = __int_as_float(0x7fffffff);
    const int64_t step = ln.groups();
    const auto send = [&](int64_t base, int stage) {
        if constexpr (L::BULK) {
            const int64_t row = base + ln.g;
            if (lead && (phase & 6) == 0 && row < n) {
                int skip;
                const uint32_t bytes = zs.window(ln, row, usual, skip), bar = jn.stage(ln, stage);
                expect_bytes(bar, bytes);
                zs.template send_bulk<false>(ln, row, skip, bytes, ring0 + (uint32_t)(stage * H::STAGE), bar);
            }
        } else if constexpr (MODE != 2) {
            if (base < n)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int64_t row = base + r * step + ln.g;
                    const uint32_t o = (uint32_t)(stage * H::STAGE + r * H::ROW);
                    zs.send_own(ln, row, ring0 + o);
                    copy4_ahead(slot4 + o, row < n ? labels + row : labels, row < n);
                }
            copies_end();
        }
    };
    for (int i = 0; i < S; ++i) {
#pragma unroll
        for (int r = 0; r < R; ++r) zs.prepare(ln, ring0 + (uint32_t)(i * H::STAGE + r * H::ROW), minus_infinity<T>());
        if (L::BULK || i < S - 1) send(ln.first_group() + i * R * step, i);
    }
    float scale = 1.0f;
    bool scaled = false;
    double sum = 0.0;
    int64_t counted = 0;
    __shared__ double slot, cred[kRowBlock / 32];
    if (C == 1 && one) {                             // a small call's blocks count the labels themselves
        scaled = true;
        if (mean) {
            double c = 0.0;
            for (int64_t i = threadIdx.x; i < n; i += kRowBlock) c += labels[i] >= 0;
            counted = (int64_t)block_sum<kRowBlock>(c, cred);
            scale = counted > 0 ? (float)(1.0 / (double)counted) : 0.0f;
        }
    }
    int next = -1;
    if (L::BULK && ln.group() < n) next = labels[ln.group()];
    // Rows between their two halves: begun when the warp's maximum and sum are known (and, in a cluster, sent to the other
    // blocks), ended when the row's are.
    struct Rows {
        float2  e[R][L::PAIRS];
        float   m[R], s[R], z_hot[R];
        int     lab[R];
        bool    owner[R], bare;
        int64_t base;
        int     at;
    };
    const auto begin = [&](Rows& w, int64_t base) {
        Row<T, MODE, EPL> zv[R];
        bool here = true;
        w.base = base;
        w.at = at;
        if constexpr (L::BULK) {
            w.lab[0] = base + ln.g < n ? next : -1;
            if (base + step + ln.g < n) next = labels[base + step + ln.g];
            if (base + ln.g < n) here = jn.row_ready(ln, at, phase);
        } else if constexpr (MODE != 2) {
            send(base + (S - 1) * R * step, at == 0 ? S - 1 : at - 1);
            copies_wait<S - 1>();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = base + r * step + ln.g;
            const uint32_t o = (uint32_t)(at * H::STAGE + r * H::ROW);
            if constexpr (H::OWN) w.lab[r] = row < n ? (int)read4(slot4 + o) : -1;
            if constexpr (MODE == 2) w.lab[r] = row < n ? labels[row] : -1;
            zs.take(ln, row, ring0 + o, minus_infinity<T>(), zv[r]);
            zv[r].mend(ln, minus_infinity<T>());
            // the label's logit, right in the thread that has it (and anything elsewhere)
            const int lab = w.lab[r], hot = lab + ln.s - ln.rank * (L::NV * TPR * N);
            w.owner[r] = row < n && lab >= 0 && lab < k && hot >= 0 && hot < L::NV * TPR * N && hot / N % TPR == ln.l;
            if constexpr (MODE == 2) w.z_hot[r] = w.owner[r] ? to_f(z[row * ld + lab]) : nan;
            else {
                const int v = w.owner[r] ? hot / N / TPR : 0;
                w.z_hot[r] = to_f(reinterpret_cast<const T*>(ring + o + ln.place(v) * 16)[hot & (N - 1)]);
                if (MODE == 1 && zs.near_end(row) && w.owner[r]) w.z_hot[r] = to_f(z[row * ld + lab]);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) w.m[r] = row_max<T, MODE, EPL>(zv[r]);
        warp_all<MaxOp, TPR>(w.m);                   // of the group's, or the warp's, elements
#pragma unroll
        for (int r = 0; r < R; ++r) {
            w.bare = w.m[r] == -INFINITY;            // nothing but -inf (or NaN): no -inf - -inf below
            if (w.bare) w.m[r] = 0.0f;
            const float2 m2 = f2(-w.m[r]);
            float2 a = f2(here ? 0.0f : nan);
#pragma unroll
            for (int q = 0; q < L::PAIRS; ++q) {
                const float2 t = __fmul2_rn(__fadd2_rn(zv[r].pair(q), m2), f2(kLog2e));
                w.e[r][q] = make_float2(exp2_fast(t.x), exp2_fast(t.y));
                a = __fadd2_rn(a, w.e[r][q]);
            }
            w.s[r] = a.x + a.y;
        }
        warp_all<SumOp, TPR>(w.s);
        if constexpr (C > 1) {
            const float mine[2] = {w.bare ? -INFINITY : w.m[0], w.s[0]};
            join_send<TPR, C>(mine, jn, sent++, phase);
        }
        if (++at == S) { at = 0; phase ^= 1; }
    };
    const auto end = [&](Rows& w) {
        float down[R];                               // to the row's maximum from the warp's
#pragma unroll
        for (int r = 0; r < R; ++r) down[r] = 1.0f;
        if constexpr (TPR > 32) {
            // each warp's maximum and sum to the row's, at one meeting of the group a row
            float v[2][2];
            const float mine[2] = {w.bare ? -INFINITY : w.m[0], w.s[0]}, m_warp = w.m[0];
            if constexpr (C > 1) join_wait(v, jn, turn++, phase);
            else group_join<TPR, C>(mine, v, jn, turn, phase);
            constexpr bool MANY = TPR / 32 * C == 64;
            float t = MANY ? fmaxf(v[0][0], v[0][1]) : v[0][0];
            join_all<MaxOp, TPR, C>(t);
            w.m[0] = t == -INFINITY ? 0.0f : t;
            t = v[1][0] * exp2_fast((v[0][0] - w.m[0]) * kLog2e);
            if (MANY) t += v[1][1] * exp2_fast((v[0][1] - w.m[0]) * kLog2e);
            join_all<SumOp, TPR, C>(t);
            w.s[0] = t;
            down[0] = exp2_fast((w.bare ? -INFINITY : m_warp - w.m[0]) * kLog2e);
        }
        if constexpr (L::BULK) send(w.base + S * step, w.at);    // every thread of the group has its part of the row
        if (!scaled) {                                        // the first rows are worked on while the labels are counted
            grid_ready();
            scale = loss_scale(sc, mean);
            scaled = true;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = w.base + r * step + ln.g;
            const float s = w.s[r];
            const bool counts = w.lab[r] >= 0, known = w.lab[r] < k, empty = s == 0.0f;
            const float q = !known ? nan : empty ? 0.0f : __fdividef(1.0f, s);       // (1 <= s <= k, or NaN)
            // the label's thread has the row's loss and its element's gradient (p - 1) s; the first thread where there is none
            const bool teller = counts && known ? w.owner[r] : row < n && ln.l == 0 && ln.rank == 0;
            const float t = w.z_hot[r] - w.m[r];
            const float v = !counts ? 0.0f : !known ? nan : empty ? INFINITY : logf(s) - t;
            const T one_hot = from_f<T>(empty ? 0.0f : (exp2_fast(t * kLog2e) * q - 1.0f) * scale);
            if (teller) {
                row_loss[row] = v;
                sum += (double)v;
            }
            if (!dz) continue;
            Row<T, MODE, EPL> o;
            const float2 q2 = f2(q * down[r] * scale);
#pragma unroll
            for (int p = 0; p < L::PAIRS; ++p) o.set_pair(p, __fmul2_rn(w.e[r][p], q2));
            if (!counts) o.zero();
            o.template store<true>(ln, dz, row, ldd, row < n, n, ed);       // (ends with the warp's lanes in step: no store of theirs comes after)
            if (w.owner[r]) dz[row * ldd + w.lab[r]] = one_hot;
        }
    };
    if constexpr (C > 1) {
        // the next row is begun before this one is ended: the messages of one travel while the other is worked on
        Rows a, b;
        int64_t base = ln.first_group();
        if (base < n) begin(a, base);
        for (; base < n; base += 2 * step) {
            const bool more = base + step < n;
            if (more) begin(b, base + step);
            end(a);
            if (base + 2 * step < n) begin(a, base + 2 * step);
            if (more) end(b);
        }
    } else {
        Rows a;
        for (int64_t base = ln.first_group(); base < n; base += R * step) {
            begin(a, base);
            end(a);
        }
    }
    if (!scaled) grid_ready();
    jn.land(ln, phase);
    leave_cluster<C>();
    if (C == 1 && one) finish_loss_one(sum, mean, counted, &slot, loss);
    else finish_loss<kRowBlock>(sum, mean, sc, loss);
}

}  // namespace
}  // namespace gemnlr

using namespace gemnlr;

extern "C" size_t gem_nlr_label_cross_entropy_scratch_bytes(int64_t n, int32_t k)
{
    return n < 0 || k < 1 || k > kMaxColumns || (n > 0 && one_cluster(n, k)) ? 0 : sizeof(Scratch);
}

extern "C" int gem_nlr_label_cross_entropy(const void* logits_dev, int32_t type, int64_t ld, const int32_t* labels_dev, int64_t n,
                                           int32_t k, int32_t mean, float* loss_dev, float* row_loss_dev, void* dlogits_dev,
                                           int64_t ld_d, void* scratch_dev, size_t scratch_bytes, void* cuda_stream)
{
    const int tb = type_bytes(type);
    if (!tb || n < 0 || k < 1 || k > kMaxColumns || (mean != 0 && mean != 1) || !loss_dev || !aligned_to(loss_dev, 4)) return GEM_NLR_E_INVALID;
    if (n > 0 && (!logits_dev || !aligned_to(logits_dev, tb) || ld < 0 || !labels_dev || !aligned_to(labels_dev, 4) ||
                  !row_loss_dev || !aligned_to(row_loss_dev, 4) || !aligned_to(dlogits_dev, tb) || (dlogits_dev && ld_d < k) ||
                  (dlogits_dev == logits_dev && ld != ld_d)))
        return GEM_NLR_E_INVALID;
    const bool one = n > 0 && one_cluster(n, k);
    if (!one && (!scratch_dev || !aligned_to(scratch_dev, 256) || scratch_bytes < sizeof(Scratch))) return GEM_NLR_E_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    Scratch* sc = (Scratch*)scratch_dev;
    if (!one) {
        k_count_labels<<<kCountBlocks, 256, 0, st>>>(labels_dev, n, sc);
        if (launched() != GEM_NLR_OK) return GEM_NLR_E_CUDA;
    }
    const Matrix ms[2] = {{logits_dev, ld}, {dlogits_dev, ld_d}};
    const Lying lie = lying(ms, dlogits_dev ? 2 : 1, n, k, tb);
    cudaError_t rc = cudaSuccess;
    by_mode(type, lie.mode, [&](auto t, auto mode) {
        using T = decltype(t);
        const bool held = by_width<mode.value != 2 && sizeof(T) == 2 ? 16 : 8, mode.value != 2 && sizeof(T) == 2 ? 24 : 16, mode.value != 2 && sizeof(T) == 2 ? 32 : 24>(lie.mode == 1 ? (int64_t)k + 16 / tb - 1 : k, [&](auto tpr, auto epl, auto c) {
            constexpr auto kern = k_xent_rows<T, mode.value, tpr.value, epl.value, c.value>;
            constexpr int shared = XentShape<T, mode.value, tpr.value, epl.value, c.value>::SHARED;
            const int most = resident_clusters<kern, c.value>(shared);
            const int room = kMaxBlocks / c.value;
            const int cl = spread(n, kRowBlock / tpr.value, one ? 1 : xent_rows(tpr.value, epl.value), lie.period, one ? kOneBlocks : most < room ? most : room);
            rc = launch_rows(kern, cl * c.value, one ? cl : c.value, shared, !one, st, (const T*)logits_dev, ld, labels_dev, n, (int)k, (int)mean, sc, loss_dev,
                             row_loss_dev, (T*)dlogits_dev, ld_d, (int)one);
        });
        if (!held) {
            const int64_t blocks = n < kTrainSMs * 8 ? n : kTrainSMs * 8;
            rc = launch_early(k_xent_any<T>, dim3((unsigned)(blocks < 1 ? 1 : blocks)), kRowThreads, st, (const T*)logits_dev, ld, labels_dev, n,
                              (int)k, (int)mean, sc, loss_dev, row_loss_dev, (T*)dlogits_dev, ld_d);
        }
    });
    return told(rc);
}
