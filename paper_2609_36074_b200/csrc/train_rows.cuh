// Rows of a matrix, streamed: the layout that the layer norm and cross entropy kernels share.
//
// A row of d elements belongs to a group of TPR threads of a block (part of a warp, a warp, or several), or of C whole
// blocks in a cluster; EPL elements to a thread, in NV vectors of N: vector k of thread l of block r of the group holds
// elements ((r NV + k) TPR + l) N - s ... + N - 1, so that a group's accesses are contiguous.  The row is read from HBM once.
//
// Three ways of reading a matrix (MODE):
//   0  every row begins and ends at a multiple of 16 bytes: vectors of 16 bytes, s = 0
//   1  rows begin anywhere: still vectors of 16 bytes at multiples of 16, beginning s elements before the row.  s depends on
//      the row's number modulo 16 bytes / element only, and a group's rows are that far apart (see spread()), so a thread's
//      columns are the same in all its rows.  The first and the last vector hold elements of the neighbouring rows (or of
//      the padding), which are replaced after loading and left alone in storing
//   2  element by element, where the matrices of one call lie differently to 16 bytes
//
// In modes 0 and 1 rows come through a ring of stages in shared memory, S rows ahead: registers alone hold too few bytes in
// flight for HBM.  From a warp a row on (BULK), one thread sends for the whole row by one bulk copy, which arrives at a
// barrier in shared memory; the threads of narrower rows copy 16 bytes each, the very vectors that they read themselves, and
// need no barrier.
#pragma once
#include "train_common.cuh"

namespace gemnlr {

// ---- a vector of elements ----------------------------------------------------------------------------------------

__device__ __forceinline__ float2 f2(float a) { return make_float2(a, a); }

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
template <typename T> __device__ __forceinline__ uint32_t pack2(float2 v);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float2 v)
{
    const __nv_bfloat162 t = __float22bfloat162_rn(v);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float2 v)
{
    const __half2 t = __float22half2_rn(v);
    return *reinterpret_cast<const uint32_t*>(&t);
}

template <int VB> struct RawOf;
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<16> { using type = uint4; };

// VB = 8 or 16 bytes of elements
template <typename T, int VB>
struct Vec {
    static constexpr int N = VB / (int)sizeof(T), P = N / 2;
    union {
        typename RawOf<VB>::type raw;
        uint32_t w[VB / 4];
    };
    __device__ __forceinline__ Vec() {}
    __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const typename RawOf<VB>::type*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<typename RawOf<VB>::type*>(p) = raw; }
    __device__ __forceinline__ void store_streaming(T* p) const { __stcs(reinterpret_cast<typename RawOf<VB>::type*>(p), raw); }
    __device__ __forceinline__ void fill(uint32_t x)
    {
#pragma unroll
        for (int i = 0; i < VB / 4; ++i) w[i] = x;
    }
    __device__ __forceinline__ float2 pair(int p) const
    {
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * p]), __uint_as_float(w[2 * p + 1]));
        else return unpack2<T>(w[p]);
    }
    __device__ __forceinline__ void set_pair(int p, float2 v)
    {
        if constexpr (sizeof(T) == 4) { w[2 * p] = __float_as_uint(v.x); w[2 * p + 1] = __float_as_uint(v.y); }
        else w[p] = pack2<T>(v);
    }
    __device__ __forceinline__ T at(int i) const
    {
        if constexpr (sizeof(T) == 4) return *reinterpret_cast<const T*>(&w[i]);
        else {
            const uint16_t h = (uint16_t)(w[i >> 1] >> ((i & 1) * 16));
            return *reinterpret_cast<const T*>(&h);
        }
    }
    __device__ __forceinline__ void set(int i, T v)
    {
        if constexpr (sizeof(T) == 4) w[i] = *reinterpret_cast<uint32_t*>(&v);
        else {
            const uint32_t h = *reinterpret_cast<uint16_t*>(&v);
            w[i >> 1] = (i & 1) ? (w[i >> 1] & 0xffffu) | (h << 16) : (w[i >> 1] & 0xffff0000u) | h;
        }
    }
};

// ---- a thread's part of a row ------------------------------------------------------------------------------------

constexpr int kRowBlock = 256;                       // threads of a block, whatever the shape

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// 16 bytes from global to shared memory, asynchronously: the first `bytes` of them, zeros behind
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// 4 bytes, or a zero
__device__ __forceinline__ void copy4_ahead(uint32_t to, const void* from, bool ok)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(ok ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint32_t read4(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// One contiguous piece from global to shared memory; arrives at the barrier.  16-byte aligned, a multiple of 16 bytes.
__device__ __forceinline__ void bulk_ahead(uint32_t to, const void* from, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

// Polls of one wait.  A healthy one ends within microseconds.  One that runs out raises the block's `late` flag: its row's
// results become NaN, and later waits poll a little only (their copies still have to land), so that the kernel ends whatever
// has happened.
constexpr uint32_t kPolls = 1u << 20, kLatePolls = 1u << 12;

__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile uint32_t* late)
{
    uint32_t limit = kPolls;
    for (uint32_t i = 0; i < limit; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if ((i & 63u) == 63u && *late) limit = kLatePolls;
    }
    *late = 1;
    return false;
}

template <typename T, int MODE, int TPR, int EPL, int C>
struct Lane {
    static constexpr int N = MODE == 2 ? 1 : 16 / (int)sizeof(T);
    static constexpr int NV = EPL / N, GROUPS = kRowBlock / TPR;
    static constexpr int PAIRS = EPL / 2;            // pair q holds the thread's elements 2 q and 2 q + 1
    static constexpr bool BULK = MODE != 2 && TPR >= 32;
    // Elements of cut vectors are stored one each by other lanes of the warp, through EDGES places of 16 bytes a warp; rows
    // of less than 8 threads have more ends than that pays for.
    static constexpr bool EDGED = MODE == 1 && TPR >= 8;
    static constexpr int ENDS = TPR >= 32 ? 2 : 2 * 32 / TPR, TURNS = EDGED ? (ENDS * N + 31) / 32 : 1;
    static_assert(C == 1 || TPR == kRowBlock, "");
    static_assert(EPL % N == 0 && EPL % 2 == 0, "");

    int l, g, s, d, rank;
    int last;                                        // k of the row's last vector, in the block that has it; else never reached
    uint32_t head[MODE == 1 ? 4 : 1], tail[MODE == 1 ? 4 : 1];   // the row's part of vector 0 and of vector `last`, as words
    uint32_t head_bits, tail_bits;                               // and as a bit an element
    int64_t edge[TURNS];                                         // elements that this lane stores for cut vectors: from its own row's
    int edge_group[TURNS];                                       // beginning, and of which group; -1: none

    __device__ __forceinline__ Lane(int d_, const T* base, int64_t ld, int64_t ld_out)
        : l((int)threadIdx.x % TPR), g((int)threadIdx.x / TPR), s(0), d(d_), rank(C > 1 ? (int)cluster_rank() : 0)
    {
        if constexpr (MODE == 1) {
            s = lies(base, ld, group());
            const int v_last = (s + d - 1) / N - rank * NV * TPR;
            last = v_last < 0 ? -1 : v_last / TPR;   // (NV and more: another block's)
            head_bits = tail_bits = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (first(0) + i >= 0 && (last != 0 || first(0) + i < d)) head_bits |= 1u << i;
                if (first(last) + i < d) tail_bits |= 1u << i;
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                constexpr int E = 4 / (int)sizeof(T);
                constexpr uint32_t ONE = E == 1 ? 0xffffffffu : 0xffffu;
                head[w] = tail[w] = 0;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (head_bits >> (w * E + j) & 1) head[w] |= ONE << (16 * j);
                    if (tail_bits >> (w * E + j) & 1) tail[w] |= ONE << (16 * j);
                }
            }
            if constexpr (EDGED) {
                const int lane = threadIdx.x & 31;
#pragma unroll
                for (int t = 0; t < TURNS; ++t) {
                    const int x = lane + 32 * t, end = x / N, i = x % N;        // element i of one of the warp's ends
                    edge[t] = 0;
                    edge_group[t] = -1;
                    if (end >= ENDS) continue;
                    const int first_group = (int)(threadIdx.x & ~31u) / TPR, gg = first_group + end / 2;
                    const int ss = lies(base, ld, group() + (gg - g));
                    const int v = end % 2 == 0 ? 0 : (ss + d - 1) / N, owner = v % TPR, e = v * N - ss + i;
                    const bool here = (v / TPR) / NV == rank && (TPR < 32 || owner / 32 == l / 32);
                    const bool cut = v * N - ss < 0 || v * N - ss + N > d;
                    if (here && cut && (end % 2 == 0 || v != 0) && e >= 0 && e < d) {
                        edge[t] = (gg - g) * ld_out + e;
                        edge_group[t] = gg;
                    }
                }
            }
        }
    }
    static __device__ __forceinline__ int lies(const T* base, int64_t ld, int64_t row)
    {
        return (int)((reinterpret_cast<uintptr_t>(base + row * ld) & 15) / sizeof(T));
    }
    // number of the group among all groups of the grid, and their count
    __device__ __forceinline__ int64_t group() const { return (int64_t)(blockIdx.x / C) * GROUPS + g; }
    __device__ __forceinline__ int64_t first_group() const { return (int64_t)(blockIdx.x / C) * GROUPS; }
    __device__ __forceinline__ int64_t groups() const { return (int64_t)(gridDim.x / C) * GROUPS; }
    __device__ __forceinline__ int first(int k) const { return ((rank * NV + k) * TPR + l) * N - (MODE == 1 ? s : 0); }
    __device__ __forceinline__ bool any(int k) const { return first(k) < d; }
    // whether vector k may be cut by an end of the row (the same for all lanes of the group)
    __device__ __forceinline__ bool end(int k) const { return MODE == 1 && ((k == 0 && rank == 0) || k == last); }
    __device__ __forceinline__ uint32_t bits(int k) const { return k == 0 && rank == 0 ? head_bits : tail_bits; }      // where end(k)
    __device__ __forceinline__ bool holds(int k, int i) const { return MODE == 1 ? first(k) + i >= 0 && first(k) + i < d : any(k); }
    // place of the thread's vector k in a stage, in vectors
    __device__ __forceinline__ int place(int k) const { return BULK ? (g * NV + k) * TPR + l : k * kRowBlock + (int)threadIdx.x; }
};

// Shared memory of cut vectors on their way out.
template <typename LN> struct Edges { uint4 v[LN::EDGED ? kRowBlock / 32 * LN::ENDS : 1]; };

// The thread's elements of one row.
template <typename T, int MODE, int EPL>
struct Row {
    static constexpr int N = MODE == 2 ? 1 : 16 / (int)sizeof(T), NV = EPL / N;
    using V = Vec<T, 16>;
    struct One { T e; };
    typename std::conditional<MODE == 2, One, V>::type v[NV];

    // By all lanes of the warp, `ok` or not.  (A lane's row is at most 31 rows from another's in its warp.)
    template <typename LN>
    __device__ __forceinline__ void store(const LN& ln, T* base, int64_t row, int64_t ld, bool ok, int64_t n, Edges<LN>& ed) const
    {
        T* p = base + row * ld;
        if (ok) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int e = ln.first(k);
                if constexpr (MODE == 2) {
                    if (ln.any(k)) p[e] = v[k].e;
                } else if (!ln.end(k)) {
                    if (ln.any(k)) v[k].store(p + e);
                } else {
                    const uint32_t b = ln.bits(k);
                    if (b == (1u << N) - 1) v[k].store(p + e);
                    else if constexpr (LN::EDGED) {
                        const int at = (int)threadIdx.x / 32 * LN::ENDS + (LN::ENDS > 2 ? ln.g % (LN::ENDS / 2) * 2 : 0) + (k == 0 && ln.rank == 0 && ln.l == 0 ? 0 : 1);
                        if (b) ed.v[at] = v[k].raw;
                    } else if (b) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (b & (1u << i)) p[e + i] = v[k].at(i);
                    }
                }
            }
        }
        if constexpr (LN::EDGED) {
            __syncwarp();
            const T* places = reinterpret_cast<const T*>(ed.v + threadIdx.x / 32 * LN::ENDS);
#pragma unroll
            for (int t = 0; t < LN::TURNS; ++t)
                if (ln.edge_group[t] >= 0 && row + (ln.edge_group[t] - ln.g) < n) p[ln.edge[t]] = places[(threadIdx.x & 31) + 32 * t];
            __syncwarp();
        }
    }
    __device__ __forceinline__ float2 pair(int q) const
    {
        if constexpr (MODE == 2) return make_float2(to_f(v[2 * q].e), to_f(v[2 * q + 1].e));
        else return v[2 * q / N].pair(2 * q % N / 2);
    }
    __device__ __forceinline__ void set_pair(int q, float2 x)
    {
        if constexpr (MODE == 2) { v[2 * q].e = from_f<T>(x.x); v[2 * q + 1].e = from_f<T>(x.y); }
        else v[2 * q / N].set_pair(2 * q % N / 2, x);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if constexpr (MODE == 2) v[k].e = from_f<T>(0.0f); else v[k].fill(0);
    }
};

// A matrix that is read row by row.  `none`: what stands for elements outside the row (its bits in every element of a word).
template <typename T, int MODE, int TPR, int EPL, int C>
struct Source {
    using L = Lane<T, MODE, TPR, EPL, C>;
    static constexpr int N = L::N, NV = L::NV;
    // bytes of a block's stage for one row of every group
    __host__ __device__ static constexpr int stage_bytes() { return MODE == 2 ? 0 : NV * 16 * kRowBlock; }
    const T* base;
    int64_t  ld, n, span;                            // span: elements from the matrix's first to its last
    __device__ __forceinline__ Source(const T* p, int64_t ld_, int64_t n_, int d) : base(p), ld(ld_), n(n_), span((n_ - 1) * ld_ + d) {}

    // Before the first send: what no copy will write reads as `none` (the vectors beyond the row).
    __device__ __forceinline__ void prepare(const L& ln, uint32_t stage, uint32_t none) const
    {
        if constexpr (MODE != 2) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (!ln.any(k))
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(stage + (uint32_t)ln.place(k) * 16), "r"(none) : "memory");
        }
    }
    // What one thread of a group (BULK) sends for: the bytes of the group's window that lie between the matrix's ends.
    __device__ __forceinline__ uint32_t window(const L& ln, int64_t row, int64_t& from) const
    {
        const int64_t begin = row * ld - ln.s + ln.rank * (NV * TPR * N);
        int64_t stop = row * ld - ln.s + (ln.s + ln.d + N - 1) / N * N;
        if (C > 1 && stop > begin + NV * TPR * N) stop = begin + NV * TPR * N;
        from = begin < 0 ? begin + N : begin;        // (only vectors that are whole: the rest is picked up by take())
        if (MODE == 1 && stop > span) stop -= N;
        return stop > from ? (uint32_t)(stop - from) * (uint32_t)sizeof(T) : 0u;
    }
    __device__ __forceinline__ void send_bulk(const L& ln, int64_t row, int64_t from, uint32_t bytes, uint32_t stage, uint32_t bar) const
    {
        const int64_t begin = row * ld - ln.s + ln.rank * (NV * TPR * N);
        if (bytes) bulk_ahead(stage + (uint32_t)(ln.g * NV * TPR * 16) + (uint32_t)(from - begin) * (uint32_t)sizeof(T), base + from, bytes, bar);
    }
    // What every thread of a narrower group sends for.
    __device__ __forceinline__ void send_own(const L& ln, int64_t row, uint32_t stage) const
    {
        const int64_t at = row * ld;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int e = ln.first(k);
            if (row < n && ln.any(k)) {
                if (!ln.end(k) || (at + e >= 0 && at + e + N <= span)) copy_ahead(stage + (uint32_t)ln.place(k) * 16, base + at + e, 16);
            }
        }
    }
    // The row that was sent for, once its copies are complete.
    __device__ __forceinline__ void take(const L& ln, int64_t row, uint32_t stage, uint32_t none, Row<T, MODE, EPL>& r) const
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int e = ln.first(k);
            if constexpr (MODE == 2) {
                const uint32_t x = none;
                if (row < n && ln.any(k)) r.v[k].e = base[row * ld + e]; else r.v[k].e = *reinterpret_cast<const T*>(&x);
            } else {
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(r.v[k].w[0]), "=r"(r.v[k].w[1]), "=r"(r.v[k].w[2]), "=r"(r.v[k].w[3])
                             : "r"(stage + (uint32_t)ln.place(k) * 16) : "memory");
                if (ln.end(k)) {
                    const int64_t at = row * ld + e;
                    if ((at < 0 || at + N > span) && row < n) {      // a vector that reaches over the matrix's own end
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (ln.holds(k, i)) r.v[k].set(i, base[at + i]);
                    }
                    const bool h = k == 0 && ln.rank == 0;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t m = h ? ln.head[w] : ln.tail[w];
                        r.v[k].w[w] = (r.v[k].w[w] & m) | (none & ~m);
                    }
                }
            }
        }
    }
};

// A thread's elements of a vector of d values (weights), as FP32 pairs; `none` where there is no vector, 0 outside the row.
template <typename T, typename LN>
__device__ __forceinline__ void load_weights(const LN& ln, const void* w, int wtype, float none, float2 (&out)[LN::PAIRS])
{
#pragma unroll
    for (int q = 0; q < LN::PAIRS; ++q) {
        float x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = (2 * q + h) / LN::N, i = (2 * q + h) % LN::N, e = ln.first(k) + i;
            x[h] = !ln.holds(k, i) ? 0.0f : !w ? none : wtype == GEM_NLR_F32 ? ((const float*)w)[e] : to_f(((const T*)w)[e]);
        }
        out[q] = make_float2(x[0], x[1]);
    }
}

// ---- sums over a group -------------------------------------------------------------------------------------------

struct SumOp { __device__ __forceinline__ static float of(float a, float b) { return a + b; } };
struct MaxOp { __device__ __forceinline__ static float of(float a, float b) { return fmaxf(a, b); } };

// Shared memory of group_all for R values at a time: two halves of a value for every warp of a group (or cluster); and the
// barriers of a ring of S stages, one a stage and group.
template <typename LN, int TPR, int C, int R, int S>
struct Join {
    static constexpr int W = TPR > 32 ? TPR / 32 * C : 1;        // values to join: one a warp
    static constexpr int FULLS = LN::BULK ? S * LN::GROUPS : 1;
    float    v[TPR <= 32 ? 1 : 2 * R * C * kRowBlock / 32];
    uint64_t bar[C > 1 ? 2 : 1];                                 // the halves' arrivals from the cluster's blocks
    uint64_t full[FULLS];                                        // the ring's stages
    uint32_t late;                                               // a wait has run out
    __device__ __forceinline__ uint32_t half(int h) { return (uint32_t)__cvta_generic_to_shared(&bar[h]); }
    __device__ __forceinline__ uint32_t stage(const LN& ln, int at) { return (uint32_t)__cvta_generic_to_shared(&full[at * LN::GROUPS + ln.g]); }
    // before the first use, by all threads
    __device__ __forceinline__ void begin()
    {
        if constexpr (LN::BULK || C > 1) {
            if (threadIdx.x == 0) {
                if constexpr (LN::BULK)
                    for (int i = 0; i < FULLS; ++i) barrier_init((uint32_t)__cvta_generic_to_shared(&full[i]), 1);
                if constexpr (C > 1) { barrier_init(half(0), 1); barrier_init(half(1), 1); }
                asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
                late = 0;
                if constexpr (C > 1)
#pragma unroll
                    for (int h = 0; h < 2; ++h) expect_bytes(half(h), W * R * (uint32_t)sizeof(float));
            }
            __syncwarp();
            if constexpr (C > 1) cluster_barrier(); else __syncthreads();
        }
    }
};

// Sums (or maxima) of R values over a group; every thread gets the same bits.  `turn` counts the calls.
// Where a group is more than a warp, its warps write their values to shared memory and meet at the group's barrier.  In a
// cluster every warp sends its values to every block, and a thread waits until its block has all of them; no block waits for
// a barrier of the cluster, whose release would wait for the rows' stores too.  Both use the halves of the buffer in turn:
// whoever writes a half has seen, in the call between, values that every warp sent after its last reads of that half.
template <typename Op, int TPR, int C, int R, typename J>
__device__ __forceinline__ void group_all(float (&v)[R], J& jn, uint32_t& turn)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = Op::of(v[r], __shfl_xor_sync(0xffffffffu, v[r], o));
    if constexpr (TPR > 32) {
        constexpr int W = J::W;
        const int g = threadIdx.x / TPR, warp = (threadIdx.x % TPR) >> 5, l = threadIdx.x & 31, half = turn & 1;
        float* b = jn.v + (g * 2 + half) * R * W;
        bool here = true;
        if constexpr (C > 1) {
            if (l < C) {
                const uint32_t mine = (uint32_t)__cvta_generic_to_shared(b + cluster_rank() * (TPR / 32) + warp);
                const uint32_t bar = jn.half(half);
                uint32_t there, there_bar;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(l));
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there_bar) : "r"(bar), "r"(l));
#pragma unroll
                for (int r = 0; r < R; ++r)
                    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];"
                                 ::"r"(there + (uint32_t)(r * W * sizeof(float))), "r"(__float_as_uint(v[r])), "r"(there_bar) : "memory");
            }
            __syncwarp();
            here = wait_for(jn.half(half), (turn >> 1) & 1, &jn.late);
            if (threadIdx.x == 0) expect_bytes(jn.half(half), W * R * (uint32_t)sizeof(float));      // for the call after the next
        } else {
            if (l == 0)
#pragma unroll
                for (int r = 0; r < R; ++r) b[r * W + warp] = v[r];
            if constexpr (TPR == kRowBlock) __syncthreads();
            else asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "n"(TPR) : "memory");
        }
        ++turn;
        // a warp's lanes take the warps' values and join them, instead of every thread reading all of them
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float t = b[r * W + (l & (W - 1))];
            if constexpr (W == 64) t = Op::of(t, b[r * W + 32 + l]);
#pragma unroll
            for (int o = (W < 32 ? W : 32) / 2; o > 0; o >>= 1) t = Op::of(t, __shfl_xor_sync(0xffffffffu, t, o));
            v[r] = here ? t : __int_as_float(0x7fffffff);
        }
    }
}

// A block of a cluster may not end while another one still writes to its shared memory.
template <int C> __device__ __forceinline__ void leave_cluster() { if constexpr (C > 1) cluster_barrier(); }

// ---- host: which shape, how many blocks ----------------------------------------------------------------------------

template <int V> struct Const { static constexpr int value = V; };

// f(TPR, EPL, C) as constants for rows of `width` elements (the window's s included), false if it is wider than eight blocks
// hold.  Few threads a row and many elements a thread keep the work per row (sums over the group, labels, statistics) small;
// what bounds EPL are 128 registers next to weights and sums: E1 or E2 elements from a warp a row on (E1 TPR > E2 TPR / 2).
// Rows wider than 256 E2 go to clusters of blocks, so that every SM still has two blocks, one of which loads while the
// other adds.
template <int E1, int E2, typename F>
bool by_width(int64_t width, F f)
{
    if (width <= 16) f(Const<1>{}, Const<16>{}, Const<1>{});
    else if (width <= 32) f(Const<2>{}, Const<16>{}, Const<1>{});
    else if (width <= 64) f(Const<4>{}, Const<16>{}, Const<1>{});
    else if (width <= 128) f(Const<8>{}, Const<16>{}, Const<1>{});
    else if (width <= 256) f(Const<16>{}, Const<16>{}, Const<1>{});
    else if (width <= 512) f(Const<32>{}, Const<16>{}, Const<1>{});
    else if (E2 > 16 && width <= 32 * E1) f(Const<32>{}, Const<(E2 > 16 ? E1 : 16)>{}, Const<1>{});
    else if (E2 > 16 && width <= 32 * E2) f(Const<32>{}, Const<(E2 > 16 ? E2 : 16)>{}, Const<1>{});
    else if (width <= 64 * E1) f(Const<64>{}, Const<E1>{}, Const<1>{});
    else if (width <= 64 * E2) f(Const<64>{}, Const<E2>{}, Const<1>{});
    else if (width <= 128 * E1) f(Const<128>{}, Const<E1>{}, Const<1>{});
    else if (width <= 128 * E2) f(Const<128>{}, Const<E2>{}, Const<1>{});
    else if (width <= 256 * E1) f(Const<256>{}, Const<E1>{}, Const<1>{});
    else if (width <= 256 * E2) f(Const<256>{}, Const<E2>{}, Const<1>{});
    else if (width <= 512 * E1) f(Const<256>{}, Const<E1>{}, Const<2>{});
    else if (width <= 512 * E2) f(Const<256>{}, Const<E2>{}, Const<2>{});
    else if (width <= 1024 * E1) f(Const<256>{}, Const<E1>{}, Const<4>{});
    else if (width <= 1024 * E2) f(Const<256>{}, Const<E2>{}, Const<4>{});
    else if (width <= 2048 * E1) f(Const<256>{}, Const<E1>{}, Const<8>{});
    else if (width <= 2048 * E2) f(Const<256>{}, Const<E2>{}, Const<8>{});
    else return false;
    return true;
}

// Stages of a ring whose stage takes `bytes`: up to four, within a half of an SM's shared memory (two blocks an SM).
__host__ __device__ constexpr int ring_stages(int bytes) { return bytes == 0 ? 1 : 98304 / bytes < 2 ? 2 : 98304 / bytes > 4 ? 4 : 98304 / bytes; }

// One matrix operand of a call.
struct Matrix {
    const void* p;
    int64_t     ld;
};

// How the matrices of a call can be read together, and the period of s in rows.
struct Lying {
    int mode;
    int period;
};
inline Lying lying(const Matrix* ms, int count, int64_t n, int64_t d, int tb)
{
    const auto begin = [&](const Matrix& m) { return (int)(reinterpret_cast<uintptr_t>(m.p) & 15); };
    const auto step = [&](const Matrix& m) { return n > 1 ? (int)((uint64_t)(m.ld * tb) & 15) : 0; };
    for (int i = 1; i < count; ++i)
        if (begin(ms[i]) != begin(ms[0]) || step(ms[i]) != step(ms[0])) return {2, 1};
    const int st = step(ms[0]);
    if (begin(ms[0]) == 0 && st == 0 && d * tb % 16 == 0) return {0, 1};
    int period = 1;
    while (st * period % 16 != 0) period *= 2;
    return {1, period};
}

// f(T, MODE) as a value and a constant
template <typename F>
void by_mode(int32_t type, int mode, F f)
{
    by_type(type, [&](auto t) {
        if (mode == 0) f(t, Const<0>{});
        else if (mode == 1) f(t, Const<1>{});
        else f(t, Const<2>{});
        return 0;
    });
}

// Groups of C blocks of kernel K, with `shared` bytes of dynamic shared memory, that fit the current device at once (looked up
// once a device, where the kernel is also allowed that much).
template <auto K, int C>
int resident_clusters(int shared)
{
    static std::atomic<int> found[kTrainDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kTrainDevices) return 1;
    int per = found[dev].load(std::memory_order_acquire);
    if (per) return per;
    if (shared > 0) cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if constexpr (C == 1) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, K, kRowBlock, (size_t)shared) != cudaSuccess || per < 1) per = 1;
        per *= kTrainSMs;
    } else {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(C);
        cfg.blockDim = dim3(kRowBlock);
        cfg.dynamicSmemBytes = (size_t)shared;
        cudaLaunchAttribute at = {};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = C;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&per, K, &cfg) != cudaSuccess || per < 1) per = 1;
    }
    found[dev].store(per, std::memory_order_release);
    return per;
}

// Clusters (or blocks) to launch for n rows, `at_once` of them handled by one at a time: no more than `most`, and a multiple
// of the period of s over the groups of one when rows come round again.
inline int spread(int64_t n, int groups, int at_once, int period, int64_t most)
{
    const int64_t need = (n + (int64_t)groups * at_once - 1) / ((int64_t)groups * at_once);
    if (need <= most && at_once == 1) return (int)(need < 1 ? 1 : need);
    int64_t c = need < most ? need : most;
    const int per = period > groups ? period / groups : 1;
    if (c > per) c -= c % per;
    else c = per;                                    // (a few more than there are rows for: they find none)
    return (int)c;
}

// Launch of `blocks` blocks of kRowBlock threads with `shared` bytes of dynamic shared memory in clusters of c; `early`: it may begin while the stream's last kernel ends
// (and waits for its results with grid_ready()).
template <typename... P, typename... A>
cudaError_t launch_rows(void (*k)(P...), int blocks, int c, int shared, bool early, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kRowBlock);
    cfg.dynamicSmemBytes = (size_t)shared;
    cfg.stream = st;
    cudaLaunchAttribute at[2] = {};
    int m = 0;
    if (early) {
        at[m].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[m++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (c > 1) {
        at[m].id = cudaLaunchAttributeClusterDimension;
        at[m].val.clusterDim.x = (unsigned)c;
        at[m].val.clusterDim.y = at[m].val.clusterDim.z = 1;
        ++m;
    }
    cfg.attrs = at;
    cfg.numAttrs = (unsigned)m;
    return cudaLaunchKernelEx(&cfg, k, (P)args...);
}

// Launch behind `st`'s last kernel that may begin while it ends.
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
