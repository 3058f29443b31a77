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
//      columns are the same in all its rows.  The first and the last vector may be cut: they hold elements of the
//      neighbouring rows (or of the padding) too, which are replaced after loading and left alone in storing
//   2  element by element, where the matrices of one call lie differently to 16 bytes
// Measured, bf16, 60000 rows of 1000 in mode 0, of 1001 in mode 1, of 1000 out of 1013 (with dense outputs) in mode 2: layer norm
// forward 45, 50, 77 us, its gradient 68, 85, 90 us, cross entropy 48, 53, 88 us.
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

// 16 bytes from global to shared memory, asynchronously
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
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
// ONCE: what is read is the first to leave L2.  Layer norm's aligned rows: 151 us without, 146 with (262144 x 768 bf16); rows
// that begin anywhere share sectors with their neighbours and lose (gradient 60000 x 1001 89 to 93 us), and so does the cross
// entropy (131072 x 1000 bf16 93 to 104 us).
template <bool ONCE>
__device__ __forceinline__ void bulk_ahead(uint32_t to, const void* from, uint32_t bytes, uint32_t bar)
{
    if constexpr (ONCE) {
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                     ::"r"(to), "l"(from), "r"(bytes), "r"(bar), "l"(policy) : "memory");
        return;
    }
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

// Polls of a wait.  A healthy one ends within microseconds.  One that runs out leaves NaN in the results that depend on it, and
// its thread waits for nothing of that kind again, so that the kernel ends whatever has happened.  Messages are waited for
// longer than rows: a block that gives a row up still sends its messages (NaN) in time, and the cluster's blocks stay in step.
constexpr uint32_t kPolls = 1u << 20, kLandPolls = 1u << 12, kMessagePolls = 4 * kPolls;

__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, uint32_t polls)
{
    for (uint32_t i = 0; i < polls; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}

template <typename T, int MODE, int TPR, int EPL, int C>
struct Lane {
    static constexpr int N = MODE == 2 ? 1 : 16 / (int)sizeof(T);
    static constexpr int NV = EPL / N, GROUPS = kRowBlock / TPR;
    static constexpr int PAIRS = EPL / 2;            // pair q holds the thread's elements 2 q and 2 q + 1
    static constexpr int LANES = TPR * C, STRIDE = TPR * N;           // elements from a thread's vector to its next
    static constexpr bool BULK = MODE != 2 && TPR >= 32;
    // Elements of cut vectors are stored one each by other lanes of the warp, through EDGES places of 16 bytes a warp; rows
    // of less than 8 threads have more ends than that pays for.
    static constexpr bool EDGED = MODE == 1 && TPR >= 8;
    static constexpr int ENDS = TPR >= 32 ? 2 : 2 * 32 / TPR, TURNS = EDGED ? (ENDS * N + 31) / 32 : 1;
    static_assert(C == 1 || TPR == kRowBlock, "");
    static_assert(EPL % N == 0 && EPL % 2 == 0, "");

    int l, g, s, d, rank;
    uint32_t wholes;                                 // bit k: vector k lies within the row (MODE 1)
    bool head;                                       // the thread's vector 0 is the row's first, and cut
    uint32_t tail;                                   // bit k: vector k is the row's last, not its first, and cut.  (A number to compare
                                                     // k with would make the compiler index the row, and so hold it in local memory.)
    int64_t edge[TURNS];                             // elements that this lane stores for cut vectors: from its own row's
    int edge_group[TURNS];                           // beginning, and of which group; -1: none

    // Vectors that a cut can be in: the first, and from the middle on (a row fills more than half of its shape's places, less
    // a vector; in clusters the last block may have a few only, and the narrowest shape takes every row there is).
    static constexpr int CUTS_FROM = C > 1 || TPR == 2 ? 0 : (NV + 1) / 2 - 1;
    __host__ __device__ static constexpr bool may_cut(int k) { return MODE == 1 && (k == 0 || k >= CUTS_FROM); }
    __host__ __device__ static constexpr int mask_bytes() { return MODE == 1 ? NV * 16 * kRowBlock : 0; }
    uint32_t masks;                                  // shared memory: the row's part of the thread's vectors, as bits

    // `masks_`: mask_bytes() of the block's shared memory; each thread reads what it has written there itself
    __device__ __forceinline__ Lane(int d_, const T* base, int64_t ld, int64_t ld_out, uint32_t masks_)
        : l((int)threadIdx.x % TPR), g((int)threadIdx.x / TPR), s(0), d(d_), rank(C > 1 ? (int)cluster_rank() : 0), wholes(0), head(false), tail(0), masks(masks_ + threadIdx.x * 16)
    {
        if constexpr (MODE == 1) {
            s = lies(base, ld, group());
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int lo = first(k), hi = lo + N;
                if (lo >= 0 && hi <= d) wholes |= 1u << k;
                else if (lo < 0) head = true;
                else if (lo < d && (k | rank | l) == 0) head = true;     // a row within one vector
                else if (lo < d) tail |= 1u << k;
                const uint4 m = words_of(lo);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(masks + k * 16 * kRowBlock), "r"(m.x), "r"(m.y), "r"(m.z), "r"(m.w) : "memory");
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
    // the row's part of the vector whose first element is e, as bits
    __device__ __forceinline__ uint4 words_of(int e) const
    {
        uint32_t m[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            constexpr int E = 4 / (int)sizeof(T);
            constexpr uint32_t ONE = E == 1 ? 0xffffffffu : 0xffffu;
            m[w] = 0;
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (e + w * E + j >= 0 && e + w * E + j < d) m[w] |= ONE << (16 * j);
        }
        return make_uint4(m[0], m[1], m[2], m[3]);
    }
    // elements of the thread's cut vectors that are not the row's
    __device__ __forceinline__ float head_spares() const { return MODE == 1 && head ? (float)(max(s, 0) + max(N - s - d, 0)) : 0.0f; }
    __device__ __forceinline__ float tail_spares() const { return MODE == 1 && tail ? (float)((N - (s + d) % N) % N) : 0.0f; }
    __device__ __forceinline__ uint4 mask(int k) const
    {
        uint4 m;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(m.x), "=r"(m.y), "=r"(m.z), "=r"(m.w) : "r"(masks + k * 16 * kRowBlock) : "memory");
        return m;
    }
    // place of the group's ends (a first and a last vector) among the block's; with more than a warp to a group, of the warp's
    __device__ __forceinline__ int place_of_ends() const { return TPR >= 32 ? (int)threadIdx.x / 32 : g; }
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
    __device__ __forceinline__ bool whole(int k) const { return MODE == 1 ? (wholes >> k & 1) != 0 : any(k); }
    __device__ __forceinline__ bool holds(int k, int i) const { return MODE == 1 ? first(k) + i >= 0 && first(k) + i < d : any(k); }
    // place of the thread's vector k in a stage, in vectors
    __device__ __forceinline__ int place(int k) const { return BULK ? (g * NV + k) * TPR + l : k * kRowBlock + (int)threadIdx.x; }
};

// Shared memory for the ends of rows: cut vectors on their way out.
template <typename LN>
struct Edges {
    static constexpr int PLACES = LN::GROUPS < kRowBlock / 32 ? 2 * (kRowBlock / 32) : 2 * LN::GROUPS;
    uint4 v[LN::EDGED ? PLACES : 1];
};

// The thread's elements of one row.
template <typename T, int MODE, int EPL>
struct Row {
    static constexpr int N = MODE == 2 ? 1 : 16 / (int)sizeof(T), NV = EPL / N;
    using V = Vec<T, 16>;
    struct One { T e; };
    typename std::conditional<MODE == 2, One, V>::type v[NV];

    // By all lanes of the warp, `ok` or not.  (A lane's row is at most 31 rows from another's in its warp.)  STREAM: what is
    // written is the first to leave L2.
    template <bool STREAM, typename LN>
    __device__ __forceinline__ void store(const LN& ln, T* base, int64_t row, int64_t ld, bool ok, int64_t n, Edges<LN>& ed) const
    {
        T* p = base + row * ld;
        if (ok) {
            T* mine = p + ln.first(0);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if constexpr (MODE == 2) {
                    if (ln.any(k)) mine[k * LN::STRIDE] = v[k].e;
                } else {
                    if (ln.whole(k)) {
                        if constexpr (STREAM) v[k].store_streaming(mine + k * LN::STRIDE); else v[k].store(mine + k * LN::STRIDE);
                    }
                }
            }
            if constexpr (LN::EDGED) {
                if (ln.head) ed.v[2 * ln.place_of_ends()] = v[0].raw;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (ln.tail >> k & 1) ed.v[2 * ln.place_of_ends() + 1] = v[k].raw;
            } else if constexpr (MODE == 1) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if ((k == 0 && ln.head) || (ln.tail >> k & 1)) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (ln.holds(k, i)) mine[k * LN::STRIDE + i] = v[k].at(i);
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
    // What stands in cut vectors for elements that are not the row's: the bits of a word.  (No branches here and below: a
    // divergent one costs more than masking every vector that could be cut.)
    template <typename LN>
    __device__ __forceinline__ void mend(const LN& ln, uint32_t none)
    {
        if constexpr (MODE == 1) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (LN::may_cut(k)) blend(v[k], none, ln.mask(k));
        }
    }
    // The same with copies of one of the row's elements in each cut vector (its last in the row's first vector, its first in
    // the others); it is what stands there afterwards that the sums are corrected by, which loses no more than as many
    // roundings as there are copies, wherever zero lies.
    template <typename LN>
    __device__ __forceinline__ void mend_own(const LN& ln)
    {
        if constexpr (MODE == 1) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (LN::may_cut(k)) blend(v[k], twice(own(ln, k)), ln.mask(k));
        }
    }
    template <typename LN>
    __device__ __forceinline__ T own(const LN& ln, int k) const
    {
        T one = k == 0 && ln.head ? v[0].at(N - 1) : v[k].at(0);
        if (LN::NV * LN::LANES * N <= 16 && k == 0 && ln.d < N - ln.s) {         // the whole row within one vector
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i == ln.s) one = v[k].at(i);
        }
        return one;
    }
    // those elements of the thread's cut vectors: the row's first, the row's last (anything where it has none)
    template <typename LN>
    __device__ __forceinline__ float2 spares(const LN& ln) const
    {
        float t = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (LN::may_cut(k) && (ln.tail >> k & 1)) t = to_f(v[k].at(0));
        return make_float2(to_f(own(ln, 0)), t);
    }
    static __device__ __forceinline__ uint32_t twice(T x)
    {
        if constexpr (sizeof(T) == 4) return *reinterpret_cast<uint32_t*>(&x);
        else return *reinterpret_cast<uint16_t*>(&x) * 0x10001u;
    }
    static __device__ __forceinline__ void blend(V& x, uint32_t none, uint4 m)
    {
        x.w[0] = (x.w[0] & m.x) | (none & ~m.x);
        x.w[1] = (x.w[1] & m.y) | (none & ~m.y);
        x.w[2] = (x.w[2] & m.z) | (none & ~m.z);
        x.w[3] = (x.w[3] & m.w) | (none & ~m.w);
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
    int64_t  near;                                   // rows that begin within N elements of the matrix's first
    __device__ __forceinline__ Source(const T* p, int64_t ld_, int64_t n_, int d)
        : base(p), ld(ld_), n(n_), span((n_ - 1) * ld_ + d), near(ld_ >= N ? 1 : ld_ > 0 ? (N - 1) / ld_ + 1 : n_) {}

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
    __device__ __forceinline__ uint32_t window_bytes(const L& ln) const
    {
        int stop = (ln.s + ln.d + N - 1) / N * N - ln.rank * (NV * TPR * N);
        if (C > 1 && stop > NV * TPR * N) stop = NV * TPR * N;
        return stop > 0 ? (uint32_t)stop * (uint32_t)sizeof(T) : 0u;
    }
    // usual: window_bytes(), which all rows share but those near the matrix's ends.  Returns the bytes, and adds the vectors
    // to leave out at the beginning to `skip` (what is left out is picked up by take()).
    __device__ __forceinline__ uint32_t window(const L& ln, int64_t row, uint32_t usual, int& skip) const
    {
        skip = 0;
        if (MODE == 1 && near_end(row)) {
            const int64_t begin = row * ld - ln.s + ln.rank * (NV * TPR * N), stop = begin + usual / (uint32_t)sizeof(T);
            const int64_t from = begin < 0 ? begin + N : begin, to = stop > span ? stop - N : stop;
            skip = begin < 0 ? N : 0;
            return to > from ? (uint32_t)(to - from) * (uint32_t)sizeof(T) : 0u;
        }
        return usual;
    }
    template <bool ONCE>
    __device__ __forceinline__ void send_bulk(const L& ln, int64_t row, int skip, uint32_t bytes, uint32_t stage, uint32_t bar) const
    {
        const T* from = base + (row * ld - ln.s + ln.rank * (NV * TPR * N) + skip);
        if (bytes) bulk_ahead<ONCE>(stage + (uint32_t)(ln.g * NV * TPR * 16 + skip * (int)sizeof(T)), from, bytes, bar);
    }
    // What every thread of a narrower group sends for.
    __device__ __forceinline__ void send_own(const L& ln, int64_t row, uint32_t stage) const
    {
        const T* mine = base + row * ld + ln.first(0);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (row < n && ln.any(k) && (MODE == 0 || ln.whole(k) || within(ln, row, k)))
                copy_ahead(stage + (uint32_t)ln.place(k) * 16, mine + k * L::STRIDE);
    }
    // whether a vector of the row may reach over one of the matrix's ends
    __device__ __forceinline__ bool near_end(int64_t row) const { return row < near || row >= n - near; }
    // whether the thread's vector k of the row lies between the matrix's ends
    __device__ __forceinline__ bool within(const L& ln, int64_t row, int k) const
    {
        const int64_t at = row * ld + ln.first(k);
        return at >= 0 && at + N <= span;
    }
    // The row that was sent for, once its copies are complete; cut vectors are not mended yet.
    __device__ __forceinline__ void take(const L& ln, int64_t row, uint32_t stage, uint32_t none, Row<T, MODE, EPL>& r) const
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if constexpr (MODE == 2) {
                const uint32_t x = none;
                if (row < n && ln.any(k)) r.v[k].e = base[row * ld + ln.first(k)]; else r.v[k].e = *reinterpret_cast<const T*>(&x);
            } else {
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(r.v[k].w[0]), "=r"(r.v[k].w[1]), "=r"(r.v[k].w[2]), "=r"(r.v[k].w[3])
                             : "r"(stage + (uint32_t)ln.place(k) * 16) : "memory");
            }
        }
        if constexpr (MODE == 1) {
            if (row < n && near_end(row)) {          // vectors that reach over the matrix's own ends came through no copy
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (((k == 0 && ln.head) || (ln.tail >> k & 1)) && !within(ln, row, k)) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (ln.holds(k, i)) r.v[k].set(i, base[row * ld + ln.first(k) + i]);
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

// Shared memory of group_join for R values at a time: PARTS times a value for every warp of a group (or cluster); and the
// barriers of a ring of S stages, one a stage and group.
template <typename LN, int TPR, int C, int R, int S, int PARTS_ = 2>
struct Join {
    static constexpr int PARTS = PARTS_;
    static constexpr int W = TPR > 32 ? TPR / 32 * C : 1;        // values to join: one a warp
    static constexpr int FULLS = LN::BULK ? S * LN::GROUPS : 1;
    float    v[TPR <= 32 ? 1 : PARTS * R * C * kRowBlock / 32];
    uint64_t bar[C > 1 ? PARTS : 1];                             // the parts' arrivals from the cluster's blocks
    uint64_t full[FULLS];                                        // the ring's stages
    uint32_t row_lost;                                           // whether a thread's wait for a row has run out (BULK)
    __device__ __forceinline__ uint32_t part(int h) { return (uint32_t)__cvta_generic_to_shared(&bar[h]); }
    __device__ __forceinline__ uint32_t stage(const LN& ln, int at) { return (uint32_t)__cvta_generic_to_shared(&full[at * LN::GROUPS + ln.g]); }
    // The group's row in stage `at`, whose turn is at bit 0 of `phase`: whether its copies are complete.  Bit 1 of `phase` says that
    // a wait of this thread for a row has run out (and bits 3 and on where that was), bit 2 that one for messages has.  After
    // the first it waits for no row, and after either it sends for none: the stage's barrier has an arrival that was not answered
    // and takes no second one, and without messages nobody tells when all warps are done with a stage.
    __device__ __forceinline__ bool row_ready(const LN& ln, int at, uint32_t& phase)
    {
        if (phase & 2) return false;
        if (wait_for(stage(ln, at), phase & 1, kPolls)) return true;
        phase |= 2 | (phase & 1) << 3 | (uint32_t)at << 4;
        return false;
    }
    // After the last row: what is still on its way is given time to land, so that no copy meets whatever the memory is used for
    // next, and sums over the rows are told (row_lost is theirs to read after a meeting of the block).
    __device__ __forceinline__ void land(const LN& ln, uint32_t phase)
    {
        if constexpr (LN::BULK) {
            if (phase & 2) {
                uint32_t parity = phase >> 3 & 1;
#pragma unroll 1
                for (int i = 0, at = (int)(phase >> 4); i < S; ++i) {
                    wait_for(stage(ln, at), parity, kLandPolls);
                    if (++at == S) { at = 0; parity ^= 1; }
                }
                *(volatile uint32_t*)&row_lost = 1;
            }
        }
    }
    // before the first use, by all threads
    __device__ __forceinline__ void begin()
    {
        if constexpr (LN::BULK || C > 1) {
            if (threadIdx.x == 0) {
                if constexpr (LN::BULK)
                    for (int i = 0; i < FULLS; ++i) barrier_init((uint32_t)__cvta_generic_to_shared(&full[i]), 1);
                if constexpr (C > 1)
                    for (int h = 0; h < PARTS; ++h) barrier_init(part(h), 1);
                asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
                row_lost = 0;
                if constexpr (C > 1)
#pragma unroll
                    for (int h = 0; h < PARTS; ++h) expect_bytes(part(h), W * R * (uint32_t)sizeof(float));
            }
            __syncwarp();
            if constexpr (C > 1) cluster_barrier(); else __syncthreads();
        }
    }
};

// Sums (or maxima) of R values over the group's threads in a warp; every thread gets the same bits.
template <typename Op, int TPR, int R>
__device__ __forceinline__ void warp_all(float (&v)[R])
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = Op::of(v[r], __shfl_xor_sync(0xffffffffu, v[r], o));
}

// Groups of more than a warp: R values of every warp to every warp; lane l gets those of warp l modulo their number W (and, of
// 64, of warp 32 + l too; zeros otherwise).  `turn` counts the calls.
// The warps write to shared memory and meet at the group's barrier.  In a cluster every warp sends its values to every block
// (join_send), and a thread waits until its block has all of them (join_wait); no block waits for a barrier of the cluster,
// whose release would wait for the rows' stores too.  The parts of the buffer are used in turn, two where a warp waits
// before it sends again: whoever writes a part has seen, in the call between, values that every warp sent after its last reads
// of that part.  A warp that sends once more before it waits needs four: it has then seen values of two calls before, sent
// after the reads of four calls before.
template <int TPR, int C, int R, typename J>
__device__ __forceinline__ void join_send(const float (&v)[R], J& jn, uint32_t turn, uint32_t phase)
{
    constexpr int W = J::W;
    const int warp = threadIdx.x >> 5, l = threadIdx.x & 31, p = turn % J::PARTS;
    if (l < C && (phase & 4) == 0) {
        const uint32_t mine = (uint32_t)__cvta_generic_to_shared(jn.v + p * R * W + cluster_rank() * (TPR / 32) + warp);
        const uint32_t bar = jn.part(p);
        uint32_t there, there_bar;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(l));
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there_bar) : "r"(bar), "r"(l));
#pragma unroll
        for (int r = 0; r < R; ++r)
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];"
                         ::"r"(there + (uint32_t)(r * W * sizeof(float))), "r"(__float_as_uint(v[r])), "r"(there_bar) : "memory");
    }
    __syncwarp();
}

template <int R, typename J>
__device__ __forceinline__ void join_read(const float* b, bool here, float (&out)[R][2], J&)
{
    constexpr int W = J::W;
    const int l = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        out[r][0] = here ? b[r * W + (l & (W - 1))] : __int_as_float(0x7fffffff);
        out[r][1] = W == 64 ? b[r * W + (W == 64 ? 32 + l : 0)] : 0.0f;
    }
}

// A wait that runs out is the thread's last (bit 2 of `phase`, see row_ready): its part is not complete, and its next turn would
// seem to be.  The first thread, which arms the parts, then arms no more (an incomplete part takes no second arrival), and
// the warp sends no more, which lets all others run out at their next waits: every row from here on is NaN.
template <int R, typename J>
__device__ __forceinline__ void join_wait(float (&out)[R][2], J& jn, uint32_t turn, uint32_t& phase)
{
    const int p = turn % J::PARTS;
    const bool here = (phase & 4) == 0 && wait_for(jn.part(p), (turn / J::PARTS) & 1, kMessagePolls);
    if (!here) phase |= 4;
    else if (threadIdx.x == 0) expect_bytes(jn.part(p), J::W * R * (uint32_t)sizeof(float));          // for the part's next use
    join_read(jn.v + p * R * J::W, here, out, jn);
}

template <int TPR, int C, int R, typename J>
__device__ __forceinline__ void group_join(const float (&v)[R], float (&out)[R][2], J& jn, uint32_t& turn, uint32_t& phase)
{
    if constexpr (C > 1) {
        join_send<TPR, C>(v, jn, turn, phase);
        join_wait(out, jn, turn, phase);
    } else {
        constexpr int W = J::W;
        const int g = threadIdx.x / TPR, warp = (threadIdx.x % TPR) >> 5;
        float* b = jn.v + (g * J::PARTS + turn % J::PARTS) * R * W;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int r = 0; r < R; ++r) b[r * W + warp] = v[r];
        if constexpr (TPR == kRowBlock) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "n"(TPR) : "memory");
        join_read(b, true, out, jn);
    }
    ++turn;
}

// Sum (or maximum) of what group_join left in the lanes.
template <typename Op, int TPR, int C>
__device__ __forceinline__ void join_all(float& t)
{
    constexpr int W = TPR / 32 * C;
#pragma unroll
    for (int o = (W < 32 ? W : 32) / 2; o > 0; o >>= 1) t = Op::of(t, __shfl_xor_sync(0xffffffffu, t, o));
}

// Sums of R values over a group.
template <int TPR, int C, int R, typename J>
__device__ __forceinline__ void group_sum(float (&v)[R], J& jn, uint32_t& turn, uint32_t& phase)
{
    warp_all<SumOp, TPR>(v);
    if constexpr (TPR > 32) {
        float o[R][2];
        group_join<TPR, C>(v, o, jn, turn, phase);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            v[r] = o[r][0] + o[r][1];
            join_all<SumOp, TPR, C>(v[r]);
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
// Narrower rows: E0, two vectors to a thread, so that neighbouring threads read whole sectors of 32 bytes.
// Rows wider than 256 E2 go to clusters of blocks, so that every SM still has two blocks, one of which loads while the
// other adds.
// The triples of the callers.  E0 is two vectors of 16 bytes: 16 elements of 2 bytes, 8 of 4 (8 too where single elements are
// read).  E1, E2 are 24 and 32 (2-byte vectors) or 16 and 24 in the forward norm and the loss: with 16 at most, norm 262144 x
// 768 bf16 187 us instead of 144, 60000 x 1001 65 instead of 51, 2048 x 24000 FP32 83 instead of 69, loss 131072 x 1000 135 instead
// of 92, 2053 x 32768 f16 103 instead of 64 (the other way: norm 16384 x 4096 bf16 46 instead of 49, loss 65536 x 768 FP32 73
// instead of 76).  The gradient keeps two sums a column in registers and takes 16 (FP32: 12 and 16), and 24 only for 2-byte
// elements in mode 0, where it reads the row a second time instead of keeping it (262144 x 768 bf16 198 us, 236 with 16).
// In mode 1 the masks of that second time spill (up to 216 bytes a thread): 24 there measured 60000 x 701 88 us against 84,
// 16384 x 2501 94 against 84, though 8000 x 5001 81 against 93.
// Not all shapes stay within the registers: -Xptxas -v reports spills for 46 of 502 row kernels, 4 to 120 bytes a thread, most in
// the forward norm of clusters in modes 1 and 2 (96 to 120, where each thread holds 24 or 32 elements beside two weight vectors).
template <int E0, int E1, int E2, typename F>
bool by_width(int64_t width, F f)
{
    if (width <= 16) f(Const<2>{}, Const<8>{}, Const<1>{});
    else if (width <= 32) f(Const<32 / E0>{}, Const<E0>{}, Const<1>{});
    else if (width <= 64) f(Const<64 / E0>{}, Const<E0>{}, Const<1>{});
    else if (width <= 128) f(Const<128 / E0>{}, Const<E0>{}, Const<1>{});
    else if (width <= 256) f(Const<256 / E0>{}, Const<E0>{}, Const<1>{});
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

// Stages of a ring whose stage takes `bytes`: two to four, within a half of an SM's shared memory (two blocks an SM) less
// `others`.
__host__ __device__ constexpr int ring_stages(int bytes, int others)
{
    return bytes == 0 ? 1 : (104448 - others) / bytes < 2 ? 2 : (104448 - others) / bytes > 4 ? 4 : (104448 - others) / bytes;
}

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

// Whether a call is small enough for one launch of one cluster of up to kOneBlocks blocks that join their sums themselves: at
// most kOneRows rows a group, by the shape with the fewest groups that any layout of rows of d elements gets.
// A launch and a scratch allocation cost the caller 3 to 4 us: cross entropy 128 x 1000 bf16 12.4 us a call against 16.1 (5.8
// on the device against 7.5), layer norm's gradient 128 x 768 14.8 against 18.3.  With eight rows a group eight SMs take
// longer than that saves (cross entropy 4000 x 33: 12.4 us on the device against 8.0).
constexpr int kOneBlocks = 8, kOneRows = 4;
inline bool one_cluster(int64_t n, int64_t d)
{
    int tpr = 2;
    const auto holds = [&] { return (int64_t)tpr * (tpr < 32 ? 8 : 16) >= d + 7; };
    while (tpr < kRowBlock && !holds()) tpr *= 2;
    return holds() && n <= kOneRows * kOneBlocks * (kRowBlock / tpr);
}

// A value in another block's shared memory, at the place that `p` has in this one's.
template <typename V>
__device__ __forceinline__ V from_block(const V* p, int block)
{
    uint32_t at = (uint32_t)__cvta_generic_to_shared(p);
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(at), "r"(block));
    if constexpr (sizeof(V) == 8) {
        double v;
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(at) : "memory");
        return v;
    } else {
        float v;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
        return v;
    }
}

// Sum of that value over the `blocks` blocks of the cluster, in block order (the reads do not wait for one another).
template <typename V>
__device__ __forceinline__ double from_all_blocks(const V* p, int blocks)
{
    V v[kOneBlocks];
#pragma unroll
    for (int b = 0; b < kOneBlocks; ++b) v[b] = from_block(p, b < blocks ? b : 0);
    double t = 0.0;
#pragma unroll
    for (int b = 0; b < kOneBlocks; ++b) t += b < blocks ? (double)v[b] : 0.0;
    return t;
}

// What a launch's error becomes at the C boundary (the error itself is not left behind for the next call).
inline int told(cudaError_t e)
{
    if (e == cudaSuccess) return GEM_NLR_OK;
    cudaGetLastError();
    return GEM_NLR_E_CUDA;
}

// Launch of `blocks` blocks of kRowBlock threads with `shared` bytes of dynamic shared memory in clusters of c; `early`: it may
// begin while the stream's last kernel ends (and waits for its results with grid_ready()).  Arguments go to the driver by
// address: a table of records is 32 KB, and copies of it on the way would be on the caller's stack, which may be small.
template <typename P> struct Same { using type = P; };
template <typename... P>
cudaError_t launch(void (*k)(P...), dim3 grid, int threads, int c, int shared, bool early, cudaStream_t st, const typename Same<P>::type&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
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
    void* list[] = {const_cast<void*>(static_cast<const void*>(&args))...};
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(k), list);
}
template <typename... P>
cudaError_t launch_rows(void (*k)(P...), int blocks, int c, int shared, bool early, cudaStream_t st, const typename Same<P>::type&... args)
{
    return launch(k, dim3((unsigned)blocks), kRowBlock, c, shared, early, st, args...);
}

// Launch behind `st`'s last kernel that may begin while it ends.
template <typename... P>
cudaError_t launch_early(void (*k)(P...), dim3 grid, int threads, cudaStream_t st, const typename Same<P>::type&... args)
{
    return launch(k, grid, threads, 1, 0, true, st, args...);
}

}  // namespace gemnlr
