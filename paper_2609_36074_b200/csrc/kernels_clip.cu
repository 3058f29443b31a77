// The norm of many gradient tensors, and clipping.
//
//   norm = sqrt(sum g^2),  c = min(1, max_norm / (norm + eps)),  out = c g
//
// The tensors' records travel in the kernel's parameters (up to kMaxRecords a launch), so a call needs no table on the
// device, no copy to it and no synchronization.  Every tensor is cut into chunks; a block takes a contiguous range of the
// chunks of all tensors of its launch, and goes through it backwards when it scales: what the first pass read last is
// still in L2 then.
//
// Squares are summed a vector at a time in FP32 where nothing can be lost at either end of its range, in FP64 otherwise, and
// the vectors' sums in FP64.  The norm needs every element before the first output, so what does not fit L2 is read twice:
// 84 million bf16 elements into FP32 cannot take less than (2 x 168 + 336) MB / 6.5 TB/s = 103 us; measured 120 us (squares 35,
// scaling 91 when run alone; one tensor's norm alone 30).  The caller pays for every tensor's checks and address, 1 us each:
// that bounds lists whose elements are few (61 tensors of 64-wide layers: 62 us a call, 6 on the device; a small head of 7
// tensors: 19.4 and 5.6), and larger ones hide it.
#include "train_rows.cuh"

namespace gemnlr {
namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = kTrainSMs * 4;
constexpr int kChunk = 2048;           // elements: the grain in which tensors are dealt out
constexpr int kOneChunks = 64;         // a call of no more is one launch of one cluster: 16384 elements a block.  (258 chunks that
                                       // way: 17 us on the device against 5.7 in two launches of the whole GPU)
constexpr int kMaxRecords = 1000;      // 32 bytes a record: within the 32764 bytes of a kernel's parameters

struct Record {
    const void* in;
    void*       out;
    int64_t     numel;
    uint32_t    first;                 // its first chunk's number
    uint16_t    type, out_type;
};

template <int CAP>
struct Table {
    int32_t  count;
    uint32_t chunks;
    Record   r[CAP];
};

// Sum of squares of `m` values: FP32 where nothing can have been lost at either end of its range, else FP64.
template <int M>
__device__ __forceinline__ double sum_squares(const float (&v)[M])
{
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < M; ++i) s = fmaf(v[i], v[i], s);
    if (s >= 1e-28f && s <= 1e37f) return (double)s;
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < M; ++i) t = fma((double)v[i], (double)v[i], t);
    return t;
}

constexpr int kAhead = 8;              // vectors that a thread loads before it uses the first: 128 KB an SM on their way

// Sum of squares of the thread's share of a span of m elements; vectors where it begins at a multiple of 16 bytes.
template <typename T>
__device__ __forceinline__ double span_squares(const T* p, int64_t m)
{
    constexpr int N = 16 / (int)sizeof(T);
    double acc = 0.0;
    int64_t e = 0;
    if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        const auto add = [&](const Vec<T, 16>& x) {
            float f[N];
#pragma unroll
            for (int i = 0; i < N; i += 2) { const float2 q = x.pair(i / 2); f[i] = q.x; f[i + 1] = q.y; }
            acc += sum_squares(f);
        };
        constexpr int STRIP = kThreads * kAhead * N;
        const T* mine = p + threadIdx.x * N;
        for (; e + STRIP <= m; e += STRIP) {
            Vec<T, 16> x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) x[u].load(mine + e + u * (kThreads * N));
#pragma unroll
            for (int u = 0; u < kAhead; ++u) add(x[u]);
        }
#pragma unroll 4
        for (; e + (int)(threadIdx.x + 1) * N <= m; e += kThreads * N) {
            Vec<T, 16> x;
            x.load(mine + e);
            add(x);
        }
        e = m / N * N;
    }
    for (e += threadIdx.x; e < m; e += kThreads) {
        const float f[1] = {to_f(p[e])};
        acc += sum_squares(f);
    }
    return acc;
}

// o = c p over a span, from its end to its beginning; vectors where both begin at a multiple of their bytes, 16-byte stores
template <typename T, typename O>
__device__ __forceinline__ void span_scale(const T* p, O* o, int64_t m, float c)
{
    constexpr int N = sizeof(O) == 4 ? 4 : 8;
    int64_t whole = 0;                               // elements in vectors
    if ((reinterpret_cast<uintptr_t>(p) & (N * sizeof(T) - 1)) == 0 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) whole = m / N * N;
    for (int64_t e = whole + threadIdx.x; e < m; e += kThreads) o[e] = from_f<O>(to_f(p[e]) * c);
    using In = Vec<T, N * (int)sizeof(T)>;
    const auto put = [&](const In& x, int64_t e) {
        Vec<O, 16> y;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) y.set_pair(i, __fmul2_rn(x.pair(i), f2(c)));
        y.store_streaming(o + e + threadIdx.x * N);
    };
    constexpr int STRIP = kThreads * kAhead * N;
    const T* mine = p + threadIdx.x * N;
    const int64_t strips = whole / STRIP;
#pragma unroll 4
    for (int64_t e = strips * STRIP; e + (int)(threadIdx.x + 1) * N <= whole; e += kThreads * N) {
        In x;
        x.load(mine + e);
        put(x, e);
    }
    for (int64_t e = (strips - 1) * STRIP; e >= 0; e -= STRIP) {
        In x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u].load(mine + e + u * (kThreads * N));
#pragma unroll
        for (int u = 0; u < kAhead; ++u) put(x[u], e + u * (kThreads * N));
    }
}

// The record that holds chunk number q: the last one with first <= q (records without elements hold none).
template <int CAP>
__device__ __forceinline__ int find_record(const Table<CAP>& tb, uint32_t q)
{
    int lo = 0, hi = tb.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tb.r[mid].first <= q) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// the thread's share of the squares of the chunks q0 ... q1 - 1
template <int CAP>
__device__ __forceinline__ double all_squares(const Table<CAP>& tb, uint32_t q0, uint32_t q1)
{
    double acc = 0.0;
    int t = q0 < q1 ? find_record(tb, q0) : 0;
    for (uint32_t q = q0; q < q1;) {                 // a span: the chunks of one tensor
        while (t + 1 < tb.count && tb.r[t + 1].first <= q) ++t;
        const uint32_t end = t + 1 < tb.count && tb.r[t + 1].first < q1 ? tb.r[t + 1].first : q1;
        const int64_t e0 = (int64_t)(q - tb.r[t].first) * kChunk, e1 = (int64_t)(end - tb.r[t].first) * kChunk;
        const int64_t m = (e1 < tb.r[t].numel ? e1 : tb.r[t].numel) - e0;
        if (tb.r[t].type == GEM_NLR_F32) acc += span_squares((const float*)tb.r[t].in + e0, m);
        else if (tb.r[t].type == GEM_NLR_F16) acc += span_squares((const __half*)tb.r[t].in + e0, m);
        else acc += span_squares((const __nv_bfloat16*)tb.r[t].in + e0, m);
        q = end;
    }
    return acc;
}

// the scaled outputs of the chunks q0 ... q1 - 1, from the last to the first
template <int CAP>
__device__ __forceinline__ void all_scaled(const Table<CAP>& tb, uint32_t q0, uint32_t q1, float c)
{
    int t = q0 < q1 ? find_record(tb, q1 - 1) : 0;
    for (uint32_t q = q1; q > q0;) {
        while (tb.r[t].first >= q) --t;
        const uint32_t begin = tb.r[t].first > q0 ? tb.r[t].first : q0;
        const int64_t e0 = (int64_t)(begin - tb.r[t].first) * kChunk, e1 = (int64_t)(q - tb.r[t].first) * kChunk;
        const int64_t m = (e1 < tb.r[t].numel ? e1 : tb.r[t].numel) - e0;
        const int type = tb.r[t].type, out = tb.r[t].out_type;
        const void* in = tb.r[t].in;
        void* to = tb.r[t].out;
        q = begin;
        if (in == to && c == 1.0f) continue;
        if (type == GEM_NLR_F32) span_scale((const float*)in + e0, (float*)to + e0, m, c);
        else if (type == GEM_NLR_F16) {
            if (out == GEM_NLR_F32) span_scale((const __half*)in + e0, (float*)to + e0, m, c);
            else span_scale((const __half*)in + e0, (__half*)to + e0, m, c);
        } else {
            if (out == GEM_NLR_F32) span_scale((const __nv_bfloat16*)in + e0, (float*)to + e0, m, c);
            else span_scale((const __nv_bfloat16*)in + e0, (__nv_bfloat16*)to + e0, m, c);
        }
    }
}

template <int CAP>
__device__ __forceinline__ uint32_t first_chunk(const Table<CAP>& tb, unsigned block) { return (uint32_t)((uint64_t)tb.chunks * block / gridDim.x); }

// c.  A NaN stays one; an infinite norm gives 0 whatever the limit (infinity by infinity would be a NaN of no tensor's).
__device__ __forceinline__ float clip_factor(double norm, float max_norm, float eps)
{
    const double below = norm + (double)eps, ratio = (double)max_norm / below;
    return norm == 0.0 || ratio >= 1.0 ? 1.0f : isinf(below) ? 0.0f : (float)ratio;
}

template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
k_clip_squares(const __grid_constant__ Table<CAP> tb, double* __restrict__ part)
{
    __shared__ double sred[kThreads / 32];
    const double acc = block_sum<kThreads>(all_squares(tb, first_chunk(tb, blockIdx.x), first_chunk(tb, blockIdx.x + 1)), sred);
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
    next_may_start();
}

// A small call in one launch: the grid is one cluster, its blocks read each other's sums.
template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
k_clip_one(const __grid_constant__ Table<CAP> tb, int scale, float max_norm, float eps, float* __restrict__ norm_out)
{
    __shared__ double sred[kThreads / 32], slot, norm;
    const uint32_t q0 = first_chunk(tb, blockIdx.x), q1 = first_chunk(tb, blockIdx.x + 1);
    const double acc = block_sum<kThreads>(all_squares(tb, q0, q1), sred);
    if (threadIdx.x == 0) slot = acc;
    __syncwarp();
    cluster_barrier();
    if (threadIdx.x == 0) {
        norm = sqrt(from_all_blocks(&slot, (int)gridDim.x));
        if (blockIdx.x == 0) *norm_out = (float)norm;
    }
    __syncthreads();
    cluster_barrier();                               // (no block ends while another one reads its sum)
    if (scale) all_scaled(tb, q0, q1, clip_factor(norm, max_norm, eps));
}

__device__ __forceinline__ double norm_of(const double* part, int parts, double* sred)
{
    double v = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) v += part[i];
    return sqrt(block_sum<kThreads>(v, sred));
}

__global__ void __launch_bounds__(kThreads)
k_clip_norm(const double* part, int parts, float* __restrict__ norm)
{
    __shared__ double sred[kThreads / 32];
    grid_ready();
    const double v = norm_of(part, parts, sred);
    if (threadIdx.x == 0) *norm = (float)v;
}

template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
k_clip_scale(const __grid_constant__ Table<CAP> tb, const double* part, int parts, float max_norm, float eps,
             float* __restrict__ norm_out)
{
    __shared__ double sred[kThreads / 32];
    grid_ready();
    const double norm = norm_of(part, parts, sred);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    all_scaled(tb, first_chunk(tb, blockIdx.x), first_chunk(tb, blockIdx.x + 1), clip_factor(norm, max_norm, eps));
}

int clip_launches(int32_t count) { return (count + kMaxRecords - 1) / kMaxRecords; }

// One launch's records; false if their chunks' number passes 32 bits.
template <int CAP>
bool fill(Table<CAP>& tb, const gem_nlr_tensor* ts, int count)
{
    uint64_t chunks = 0;
    tb.count = count;
    for (int i = 0; i < count; ++i) {
        tb.r[i] = Record{ts[i].in_dev, ts[i].out_dev, ts[i].numel, (uint32_t)chunks, (uint16_t)ts[i].type, (uint16_t)ts[i].out_type};
        chunks += (uint64_t)(ts[i].numel / kChunk) + (ts[i].numel % kChunk != 0);
        if (chunks > 0xffffffffull) return false;
    }
    tb.chunks = (uint32_t)chunks;
    return true;
}

template <int CAP>
int clip_all(const gem_nlr_tensor* ts, int32_t count, bool scale, float max_norm, float eps, float* norm, double* part, cudaStream_t st)
{
    static thread_local Table<CAP> tb;               // 32 KB: not on the caller's stack, nor copied there by the launches
    const int launches = clip_launches(count) < 1 ? 1 : clip_launches(count);
    int parts = 0;
    if (launches == 1) {
        if (!fill(tb, ts, count)) return GEM_NLR_E_INVALID;
        if (tb.chunks <= (uint32_t)kOneChunks) {
            const int blocks = tb.chunks < 1 ? 1 : tb.chunks < (uint32_t)kOneBlocks ? (int)tb.chunks : kOneBlocks;
            return told(launch_rows(k_clip_one<CAP>, blocks, blocks, 0, false, st, tb, (int)scale, max_norm, eps, norm));
        }
    }
    for (int l = 0; l < launches; ++l) {
        const int first = l * kMaxRecords, m = count - first < kMaxRecords ? count - first : kMaxRecords;
        if (!fill(tb, ts + first, m)) return GEM_NLR_E_INVALID;
        const int blocks = tb.chunks < 1 ? 1 : tb.chunks < (uint32_t)kBlocks ? (int)tb.chunks : kBlocks;
        const int rc = told(launch(k_clip_squares<CAP>, dim3((unsigned)blocks), kThreads, 1, 0, false, st, tb, part + parts));
        if (rc != GEM_NLR_OK) return rc;
        parts += blocks;
    }
    if (!scale)
        return told(launch_early(k_clip_norm, dim3(1), kThreads, st, part, parts, norm));
    for (int l = launches - 1; l >= 0; --l) {
        const int first = l * kMaxRecords, m = count - first < kMaxRecords ? count - first : kMaxRecords;
        if (launches > 1) fill(tb, ts + first, m);
        const int blocks = tb.chunks < 1 ? 1 : tb.chunks < (uint32_t)kBlocks ? (int)tb.chunks : kBlocks;
        // only the first one may begin early: it waits for the squares, the others for it
        const bool early = l == launches - 1;
        const int rc = told(launch(k_clip_scale<CAP>, dim3((unsigned)blocks), kThreads, 1, 0, early, st, tb, part, parts, max_norm, eps,
                                   early ? norm : nullptr));
        if (rc != GEM_NLR_OK) return rc;
    }
    return GEM_NLR_OK;
}

}  // namespace
}  // namespace gemnlr

using namespace gemnlr;

extern "C" size_t gem_nlr_clip_grad_norm_scratch_bytes(int32_t count)
{
    if (count < 0) return 0;
    const int l = clip_launches(count);
    return sizeof(double) * (size_t)kBlocks * (l < 1 ? 1 : l);
}

extern "C" int gem_nlr_clip_grad_norm(const gem_nlr_tensor* tensors_host, int32_t count, float max_norm, float eps, float* norm_dev,
                                      void* scratch_dev, size_t scratch_bytes, void* cuda_stream)
{
    if (count < 0 || (count > 0 && !tensors_host) || !norm_dev || !aligned_to(norm_dev, 4)) return GEM_NLR_E_INVALID;
    bool scale = false;                              // an empty tensor may have no address
    for (int i = 0; i < count; ++i) scale |= tensors_host[i].out_dev != nullptr;
    if (scale && (!(max_norm >= 0.0f) || !(eps >= 0.0f))) return GEM_NLR_E_INVALID;
    for (int i = 0; i < count; ++i) {
        const gem_nlr_tensor& t = tensors_host[i];
        const int tb = type_bytes(t.type);
        if (!tb || t.numel < 0 || (t.numel > 0 && !t.in_dev) || !aligned_to(t.in_dev, tb)) return GEM_NLR_E_INVALID;
        if (scale) {
            if ((t.out_type != t.type && t.out_type != GEM_NLR_F32) || (t.numel > 0 && !t.out_dev) ||
                !aligned_to(t.out_dev, type_bytes(t.out_type)) || (t.out_dev == t.in_dev && t.out_type != t.type && t.numel > 0))
                return GEM_NLR_E_INVALID;
        }
    }
    if (!scratch_dev || !aligned_to(scratch_dev, 256) || scratch_bytes < gem_nlr_clip_grad_norm_scratch_bytes(count))
        return GEM_NLR_E_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    double* part = (double*)scratch_dev;
    if (count <= 64) return clip_all<64>(tensors_host, count, scale, max_norm, eps, norm_dev, part, st);
    return clip_all<kMaxRecords>(tensors_host, count, scale, max_norm, eps, norm_dev, part, st);
}
