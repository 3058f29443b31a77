// Routing rows to experts: scores, the choice, the weights, the order of the experts' rows, and the weights' gradient.
//
//   s = softmax(z) or 1 / (1 + exp(-z));  c = s + b;  the k largest c of the kept groups (without b: the k largest z)
//   w_j = scale s_j / sum_l s_l (or scale s_j)
//
// A warp a row, up to 16 logits a lane.  Scores become unsigned keys in their order, so that the largest of 32 lanes is one
// warp reduction and the lowest index among equals another; a round of the choice is those two.  FP32 scores are right to about 2^-20,
// which does not tell neighbours apart: where two scores that follow one another in the choice are nearer than that (and are
// not the same logit with the same bias, which are equal in any precision), the row is chosen again in FP64.  One row in a hundred
// is, at 128 experts with sigmoid scores.
//
// The order is a counting sort that keeps the rows of an expert in order, without atomics whose order shows: blocks own
// consecutive rows and count their experts; the second kernel adds the counts of the blocks before (each block reads all of
// them, 148 x experts numbers), takes sums over the experts, and gives out places in order, a warp's 32 entries at a time by
// matching equal experts.  Few rows are one block and one launch.
#include "train_common.cuh"

namespace gemnlr {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBlocks = kTrainSMs * 2;
constexpr int kMaxChosen = 32, kMaxGroups = 32;
constexpr unsigned kAll = 0xffffffffu;

struct Route {
    const void* z;
    int64_t ld;
    const float* bias;
    int64_t n;
    int experts, k, score, groups, kept, best, renorm;
    float scale;
    int32_t* expert;
    float* weight;
    int32_t* offset;
    int32_t* row;
    int32_t* place;
    int32_t* counts;        // blocks x experts
    int64_t rows_per_warp;
};

// Keys: whole numbers in the order of the scores; 0 is no candidate.
__device__ __forceinline__ uint32_t key_of(float c)
{
    const uint32_t u = __float_as_uint(c + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float score_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ uint64_t key_of(double c)
{
    const uint64_t u = (uint64_t)__double_as_longlong(c + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double score_of(uint64_t k) { return __longlong_as_double((long long)(k >> 63 ? k & ~(1ull << 63) : ~k)); }
constexpr uint32_t kNone32 = 0x007fffffu;                   // -inf
constexpr uint64_t kNone64 = 0x000fffffffffffffull;
__device__ __forceinline__ bool is_none(uint32_t k) { return k <= kNone32; }
__device__ __forceinline__ bool is_none(uint64_t k) { return k <= kNone64; }

__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(kAll, k); }
__device__ __forceinline__ uint64_t warp_max(uint64_t k)
{
    const uint32_t hi = __reduce_max_sync(kAll, (uint32_t)(k >> 32));
    const uint32_t lo = __reduce_max_sync(kAll, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (uint64_t)hi << 32 | lo;
}

__device__ __forceinline__ float warp_top(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}

// The scores' margin in FP32: 2^-18 of a score (at most 1: exp to 2 units of its argument's rounding, x exp(-x) <= 0.37, a sum of
// 16 and 5 steps, a quotient and the sum with the bias make 30 units of 2^-24 at the most) and a rounding of the bias.
__device__ __forceinline__ float margin_of(float c) { return 0x1p-18f + 0x1p-21f * fabsf(c); }

template <int V, typename K> struct Candidates {
    K key[V];
    int lane;
    // The lane's best: the largest key, the lowest index first (indices grow with v).
    __device__ __forceinline__ void mine(K& top, int& at) const
    {
        top = key[0];
        at = 0;
#pragma unroll
        for (int v = 1; v < V; ++v)
            if (key[v] > top) { top = key[v]; at = v; }
    }
};

// The k best keys into `got` (lane j: the j-th's index, -1 for none).  near(key, index, key, index) is told of each two that follow one
// another, and of the last and the one after it.  Returns whether it ever said that they are too near.
template <int V, typename K, typename N>
__device__ __forceinline__ bool choose(Candidates<V, K>& c, int k, int& got, N near)
{
    const int lane = c.lane;
    K top, last = 0;
    int at, before = -1;
    bool unsure = false;
    got = -1;
    c.mine(top, at);
    for (int j = 0; j <= k; ++j) {
        const K best = warp_max(top);
        if (is_none(best)) break;
        const int index = (int)__reduce_min_sync(kAll, top == best ? (unsigned)(at * 32 + lane) : 0x7fffffffu);
        if (j > 0 && near(last, before, best, index)) unsure = true;
        if (j == k) break;
        if (lane == j) got = index;
        last = best;
        before = index;
        if ((index & 31) == lane) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v == index >> 5) c.key[v] = 0;
            c.mine(top, at);
        }
    }
    return unsure;
}

// Leaves only the kept groups' keys.  S: float or double; by(v): the score of the lane's v-th expert that its group is judged by (-inf: none).
template <int V, typename S, typename K, typename B, typename N>
__device__ __forceinline__ bool keep_groups(Candidates<V, K>& c, const Route& r, B by, N near)
{
    const int size = r.experts / r.groups, lane = c.lane;
    Candidates<1, K> group;
    group.lane = lane;
    group.key[0] = 0;
    K mine[V];
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v] = v * 32 + lane < r.experts ? key_of(by(v)) : K(0);
    for (int g = 0; g < r.groups; ++g) {
        const int first = g * size, end = first + size;
        K top = 0, second = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = v * 32 + lane;
            if (i >= first && i < end) {
                if (mine[v] > top) { second = top; top = mine[v]; }
                else if (mine[v] > second) second = mine[v];
            }
        }
        const K best = warp_max(top);
        S s = is_none(best) ? -(S)INFINITY : (S)score_of(best);
        if (r.best == 2 && !is_none(best)) {
            // the lane that holds the best gives its second; of several equal ones only the first does
            const unsigned holders = __ballot_sync(kAll, top == best);
            const K next = warp_max(lane == __ffs(holders) - 1 ? second : top);
            if (!is_none(next)) s += (S)score_of(next);
        }
        if (lane == g) group.key[0] = key_of(s);
    }
    int got;
    const bool unsure = choose(group, r.kept, got, near);
    const unsigned stays = __reduce_or_sync(kAll, got >= 0 ? 1u << got : 0u);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = v * 32 + lane;
        if (i < r.experts && !(stays >> (i / size) & 1u)) c.key[v] = 0;
    }
    return unsure;
}

// The choice in FP64, for rows whose FP32 scores do not decide it.
template <int V>
__device__ __noinline__ int choose_in_64_bits(const Route& r, const float (&z)[V], float m, int lane)
{
    double s[V], sum = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        s[v] = z[v] == -INFINITY ? 0.0 : r.score == GEM_NLR_SOFTMAX ? exp((double)z[v] - (double)m) : 1.0 / (1.0 + exp(-(double)z[v]));
        sum += s[v];
    }
    sum = warp_sum(sum);
    Candidates<V, uint64_t> c;
    c.lane = lane;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = v * 32 + lane;
        if (r.score == GEM_NLR_SOFTMAX) s[v] /= sum;
        double x = r.bias ? s[v] + (double)(i < r.experts ? __ldg(r.bias + i) : 0.f) : (double)z[v];
        if (z[v] == -INFINITY) x = -(double)INFINITY;
        c.key[v] = i < r.experts ? key_of(x) : 0;
        if (!r.bias && r.best == 1) s[v] = (double)z[v];
        else if (r.bias) s[v] = x;
        if (z[v] == -INFINITY) s[v] = -(double)INFINITY;
    }
    const auto never = [](uint64_t, int, uint64_t, int) { return false; };
    if (r.groups > 1) keep_groups<V, double>(c, r, [&](int v) { return s[v]; }, never);
    int got;
    choose(c, r.k, got, never);
    return got;
}

// One row by one warp.
template <int V, typename T>
__device__ __forceinline__ void route_row(const Route& r, int64_t row, int lane, int& chosen)
{
    const T* zr = reinterpret_cast<const T*>(r.z) + row * r.ld;
    float z[V], m = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = v * 32 + lane;
        z[v] = i < r.experts ? to_f(zr[i]) : -INFINITY;
        bad |= z[v] != z[v] || (r.score == GEM_NLR_SOFTMAX && z[v] == INFINITY);
        m = fmaxf(m, z[v]);
    }
    const bool scored = r.bias || (r.groups > 1 && r.best == 2);          // the choice needs the scores
    float sum = 0.0f;
    if (r.score == GEM_NLR_SOFTMAX && (scored || !r.renorm)) {
        m = warp_top(m);
#pragma unroll
        for (int v = 0; v < V; ++v) sum += z[v] == -INFINITY ? 0.0f : expf(z[v] - m);
        sum = warp_sum(sum);
    }
    Candidates<V, uint32_t> c;
    c.lane = lane;
    float by[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = v * 32 + lane;
        float x = z[v];
        by[v] = x;
        if (scored && x != -INFINITY) {
            float s = r.score == GEM_NLR_SOFTMAX ? expf(x - m) / sum : 1.0f / (1.0f + expf(-x));
            if (r.bias) {
                s += __ldg(r.bias + i);
                bad |= s != s;
                x = s;
            }
            if (r.bias || r.best == 2) by[v] = s;
        }
        c.key[v] = i < r.experts ? key_of(x) : 0;
    }
    int got = -1;
    bad = __any_sync(kAll, bad);
    if (!bad) {
        // the same logit with the same bias is equal in any precision; other neighbours within the margin are not decided
        const auto near = [&](uint32_t a, int i, uint32_t b, int j) {
            const float x = score_of(a), y = score_of(b);
            if (!r.bias || x - y > margin_of(x)) return false;
            return !(to_f(zr[i]) == to_f(zr[j]) && __ldg(r.bias + i) == __ldg(r.bias + j));
        };
        const auto near_groups = [&](uint32_t a, int, uint32_t b, int) {
            const float x = score_of(a), y = score_of(b);
            return scored && !(x - y > 2.0f * margin_of(x));
        };
        bool unsure = false;
        if (r.groups > 1) unsure = keep_groups<V, float>(c, r, [&](int v) { return by[v]; }, near_groups);
        unsure |= choose(c, r.k, got, near);
        if (unsure) got = choose_in_64_bits<V>(r, z, m, lane);
    }
    // weights: lane j has the j-th chosen expert
    float w = 0.0f;
    if (bad) {
        w = __uint_as_float(0x7fc00000u);
    } else {
        const float x = got >= 0 ? to_f(zr[got]) : -INFINITY;
        if (r.renorm) {
            // s_j / sum s as a softmax over log s of the chosen: neither underflows
            const float l = got < 0 ? -INFINITY : r.score == GEM_NLR_SOFTMAX ? x : fminf(x, 0.0f) - log1pf(expf(-fabsf(x)));
            const float top = warp_top(l);
            const float e = got >= 0 ? expf(l - top) : 0.0f;
            const float total = warp_sum(e);
            if (got >= 0) w = e / total * r.scale;
        } else if (got >= 0) {
            w = (r.score == GEM_NLR_SOFTMAX ? expf(x - m) / sum : 1.0f / (1.0f + expf(-x))) * r.scale;
        }
    }
    if (lane < r.k) {
        r.expert[row * r.k + lane] = got;
        r.weight[row * r.k + lane] = w;
    }
    chosen = got;
}

// Places for the rows of this block's warps.  at: kWarps x experts, each warp's counts, replaced by the place of its next row of
// each expert; first: the place of the block's first row of each expert.
__device__ __forceinline__ void give_places(const Route& r, int32_t* at, const int32_t* first, int64_t begin, int64_t end)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int e = threadIdx.x; e < r.experts; e += kThreads) {
        int32_t next = first[e];
        for (int w = 0; w < kWarps; ++w) {
            const int32_t c = at[w * r.experts + e];
            at[w * r.experts + e] = next;
            next += c;
        }
    }
    __syncthreads();
    int32_t* mine = at + warp * r.experts;
    const int64_t stop = end * r.k;
    for (int64_t i0 = begin * r.k; i0 < stop; i0 += 32) {
        const int64_t i = i0 + lane;
        const int e = i < stop ? r.expert[i] : -1;
        const unsigned same = __match_any_sync(kAll, e);
        const int rank = __popc(same & ((1u << lane) - 1));
        int32_t p = -1;
        if (e >= 0) p = mine[e] + rank;
        __syncwarp();
        if (e >= 0 && rank == 0) mine[e] += __popc(same);
        __syncwarp();
        if (i < stop) r.place[i] = p;
        if (e >= 0) r.row[p] = (int32_t)(i / r.k);
    }
}

// Exclusive sums of total[experts] into first[experts + 1], by one block.  (experts <= kThreads)
__device__ __forceinline__ void sums_over_experts(const int32_t* total, int32_t* first, int experts)
{
    __shared__ int32_t of_warp[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = threadIdx.x;
    const int32_t own = e < experts ? total[e] : 0;
    int32_t v = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t u = __shfl_up_sync(kAll, v, o);
        if (lane >= o) v += u;
    }
    if (lane == 31) of_warp[warp] = v;
    __syncthreads();
    int32_t base = 0;
    for (int w = 0; w < warp; ++w) base += of_warp[w];
    if (e < experts) first[e] = base + v - own;
    if (e == experts - 1) first[experts] = base + v;
    __syncthreads();
}

__device__ __forceinline__ void leave_rest(const Route& r, int32_t used)
{
    for (int64_t p = used + (int64_t)blockIdx.x * kThreads + threadIdx.x; p < r.n * r.k; p += (int64_t)gridDim.x * kThreads) r.row[p] = -1;
}

// Shared memory: kWarps x experts counts; ONE: and experts + 1 sums and experts totals.
template <int V, typename T, bool ONE>
__global__ void __launch_bounds__(kThreads)
k_route(const Route r)
{
    extern __shared__ int32_t at[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < kWarps * r.experts; i += kThreads) at[i] = 0;
    __syncthreads();
    const int64_t begin = min(r.n, ((int64_t)blockIdx.x * kWarps + warp) * r.rows_per_warp), end = min(r.n, begin + r.rows_per_warp);
    int32_t* mine = at + warp * r.experts;
    for (int64_t row = begin; row < end; ++row) {
        int got;
        route_row<V, T>(r, row, lane, got);
        if (got >= 0) mine[got] += 1;                    // a row's experts differ
        __syncwarp();
    }
    __syncthreads();
    int32_t* first = at + kWarps * r.experts;
    int32_t* total = ONE ? first + r.experts + 1 : r.counts + (int64_t)blockIdx.x * r.experts;
    for (int e = threadIdx.x; e < r.experts; e += kThreads) {
        int32_t c = 0;
        for (int w = 0; w < kWarps; ++w) c += at[w * r.experts + e];
        total[e] = c;
    }
    if constexpr (ONE) {
        __syncthreads();
        sums_over_experts(total, first, r.experts);
        for (int e = threadIdx.x; e <= r.experts; e += kThreads) r.offset[e] = first[e];
        give_places(r, at, first, begin, end);
        leave_rest(r, first[r.experts]);
    }
}

// Shared memory: kWarps x experts counts, then experts + 1 sums, experts totals, experts counts of the blocks before.
__global__ void __launch_bounds__(kThreads)
k_route_places(const Route r, int blocks)
{
    extern __shared__ int32_t at[];
    int32_t* first = at + kWarps * r.experts;
    int32_t* total = first + r.experts + 1;
    int32_t* before = total + r.experts;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < kWarps * r.experts + 3 * r.experts + 1; i += kThreads) at[i] = 0;
    __syncthreads();
    const int64_t begin = min(r.n, ((int64_t)blockIdx.x * kWarps + warp) * r.rows_per_warp), end = min(r.n, begin + r.rows_per_warp);
    for (int64_t i = begin * r.k + lane; i < end * r.k; i += 32) {
        const int e = r.expert[i];
        if (e >= 0) atomicAdd(at + warp * r.experts + e, 1);
    }
    // threads in pairs (expert, share of the blocks); whole numbers: the order of the additions does not show
    const int shares = max(1, kThreads / r.experts), share = threadIdx.x / r.experts;
    if (share < shares)
        for (int e = threadIdx.x % r.experts; e < r.experts; e += kThreads) {
            int32_t all = 0, low = 0;
#pragma unroll 8
            for (int b = share; b < blocks; b += shares) {
                const int32_t c = r.counts[(int64_t)b * r.experts + e];
                all += c;
                low += b < (int)blockIdx.x ? c : 0;
            }
            atomicAdd(total + e, all);
            atomicAdd(before + e, low);
        }
    __syncthreads();
    sums_over_experts(total, first, r.experts);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= r.experts; e += kThreads) r.offset[e] = first[e];
    for (int e = threadIdx.x; e < r.experts; e += kThreads) before[e] += first[e];
    __syncthreads();
    give_places(r, at, before, begin, end);
    leave_rest(r, first[r.experts]);
}

struct RouteGrad {
    const float* dweight;
    const void* z;
    int64_t ld;
    const int32_t* expert;
    int64_t n;
    int experts, k, score, renorm;
    float scale;
    void* dz;
    int64_t ldd;
};

// A warp a row; lane j holds the j-th chosen expert, then each lane its logits.
template <int V, typename T>
__global__ void __launch_bounds__(256)
k_route_backward(const RouteGrad r)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool soft = r.score == GEM_NLR_SOFTMAX;
    for (int64_t row = (int64_t)blockIdx.x * 8 + warp; row < r.n; row += (int64_t)gridDim.x * 8) {
        const T* zr = reinterpret_cast<const T*>(r.z) + row * r.ld;
        T* dr = reinterpret_cast<T*>(r.dz) + row * r.ldd;
        int e = lane < r.k ? __ldg(r.expert + row * r.k + lane) : -1;
        if (e >= r.experts) e = -1;
        const float v = e >= 0 ? __ldg(r.dweight + row * r.k + lane) * r.scale : 0.0f;
        const float x = e >= 0 ? to_f(zr[e]) : -INFINITY;
        float z[V], out[V], g;
        const bool whole = soft && !r.renorm;                  // every logit has a share
        float m = -INFINITY, sum = 0.0f;
        if (whole) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                z[i] = i * 32 + lane < r.experts ? to_f(zr[i * 32 + lane]) : -INFINITY;
                m = fmaxf(m, z[i]);
            }
            m = warp_top(m);
            // a NaN among the logits is lost in the maximum and comes back in the sum
#pragma unroll
            for (int i = 0; i < V; ++i) {
                z[i] = z[i] == -INFINITY ? 0.0f : expf(z[i] - m);
                sum += z[i];
            }
            sum = warp_sum(sum);
            const float s = e >= 0 && x != -INFINITY ? expf(x - m) / sum : 0.0f;
            const float t = warp_sum(s * v);
            const bool any = __any_sync(kAll, e >= 0);
            g = s * v;
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = any && i * 32 + lane < r.experts && sum > 0.0f ? -(z[i] / sum) * t : any && sum != sum ? sum : 0.0f;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = 0.0f;
            const float l = e < 0 ? -INFINITY : soft ? x : fminf(x, 0.0f) - log1pf(expf(-fabsf(x)));
            const float rest = soft ? 1.0f : 1.0f / (1.0f + expf(x));          // 1 - s
            if (r.renorm) {
                const float top = warp_top(l);
                const float p0 = e >= 0 && l != -INFINITY ? expf(l - top) : 0.0f;
                const float total = warp_sum(p0);
                const float p = total != 0.0f ? p0 / total : 0.0f;
                const float t = warp_sum(p * v);
                g = p * (v - t) * rest;
            } else {
                g = v * rest / (1.0f + expf(-x));
            }
            if (e < 0 || x == -INFINITY) g = 0.0f;
        }
        // the chosen experts' shares to the lanes that hold them
        for (int j = 0; j < r.k; ++j) {
            const int at = __shfl_sync(kAll, e, j);
            const float add = __shfl_sync(kAll, g, j);
            if (at >= 0 && (at & 31) == lane) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i == at >> 5) out[i] += add;
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i * 32 + lane < r.experts) dr[i * 32 + lane] = from_f<T>(out[i]);
    }
}

template <typename F> int by_experts(int experts, F f)
{
    if (experts <= 32) return f(std::integral_constant<int, 1>{});
    if (experts <= 64) return f(std::integral_constant<int, 2>{});
    if (experts <= 128) return f(std::integral_constant<int, 4>{});
    if (experts <= 256) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

// Up to this many rows one block routes and sorts: a row a warp.
constexpr int64_t kOneBlockRows = kWarps * 4;
bool one_block(int64_t n) { return n <= kOneBlockRows; }

template <typename F> cudaError_t launch_with_shared(F kern, int grid, int shared, cudaStream_t st, const Route& r, int blocks)
{
    void* args[] = {const_cast<Route*>(&r), &blocks};
    return cudaLaunchKernel((const void*)kern, dim3(grid), dim3(kThreads), args, shared, st);
}

bool ints(const void* p) { return p && aligned_to(p, 4); }
int told(cudaError_t rc)
{
    if (rc == cudaSuccess) return GEM_NLR_OK;
    cudaGetLastError();
    return GEM_NLR_E_CUDA;
}

}  // namespace
}  // namespace gemnlr

using namespace gemnlr;

extern "C" size_t gem_nlr_route_scratch_bytes(int64_t n, int32_t experts)
{
    return n < 0 || experts < 1 || experts > GEM_NLR_MAX_EXPERTS || one_block(n) ? 0 : (size_t)kBlocks * experts * 4;
}

extern "C" int gem_nlr_route(const void* logits_dev, int32_t type, int64_t ld, const float* bias_dev, int64_t n, int32_t experts, int32_t k,
                             int32_t score, int32_t groups, int32_t kept_groups, int32_t group_best, int32_t renormalize, float scale,
                             int32_t* expert_dev, float* weight_dev, int32_t* offset_dev, int32_t* row_dev, int32_t* place_dev, void* scratch_dev,
                             size_t scratch_bytes, void* cuda_stream)
{
    const int tb = type_bytes(type);
    if (!tb || n < 0 || experts < 1 || experts > GEM_NLR_MAX_EXPERTS || k < 1 || k > kMaxChosen || (score != GEM_NLR_SOFTMAX && score != GEM_NLR_SIGMOID) ||
        groups < 1 || groups > kMaxGroups || experts % groups || kept_groups < 1 || kept_groups > groups || k > kept_groups * (experts / groups) ||
        (group_best != 1 && group_best != 2) || (renormalize != 0 && renormalize != 1) || !isfinite(scale) || !aligned_to(bias_dev, 4) || !ints(offset_dev) ||
        n > INT32_MAX / k)
        return GEM_NLR_E_INVALID;
    if (n > 0 && (!logits_dev || !aligned_to(logits_dev, tb) || ld < 0 || !ints(expert_dev) || !ints(weight_dev) || !ints(row_dev) || !ints(place_dev)))
        return GEM_NLR_E_INVALID;
    const bool one = one_block(n);
    if (!one && (!scratch_dev || !aligned_to(scratch_dev, 256) || scratch_bytes < gem_nlr_route_scratch_bytes(n, experts))) return GEM_NLR_E_WORKSPACE;
    const int64_t per_warp = one ? (n + kWarps - 1) / kWarps : (n + (int64_t)kBlocks * kWarps - 1) / ((int64_t)kBlocks * kWarps);
    const int blocks = one ? 1 : (int)((n + per_warp * kWarps - 1) / (per_warp * kWarps));
    const Route r = {logits_dev, ld, bias_dev, n, experts, k, score, groups, groups == 1 ? 1 : kept_groups, group_best, renormalize, scale, expert_dev, weight_dev,
                     offset_dev, row_dev, place_dev, (int32_t*)scratch_dev, per_warp};
    const int counts = kWarps * experts * 4;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    return by_type(type, [&](auto t) {
        return by_experts(experts, [&](auto v) {
            using T = decltype(t);
            if (one) return told(launch_with_shared(k_route<v.value, T, true>, 1, counts + (2 * experts + 1) * 4, st, r, 0));
            cudaError_t rc = launch_with_shared(k_route<v.value, T, false>, blocks, counts, st, r, 0);
            if (rc == cudaSuccess) rc = launch_with_shared(k_route_places, blocks, counts + (3 * experts + 1) * 4, st, r, blocks);
            return told(rc);
        });
    });
}

extern "C" int gem_nlr_route_backward(const float* dweight_dev, const void* logits_dev, int32_t type, int64_t ld, const int32_t* expert_dev, int64_t n,
                                      int32_t experts, int32_t k, int32_t score, int32_t renormalize, float scale, void* dlogits_dev, int64_t ld_d,
                                      void* cuda_stream)
{
    const int tb = type_bytes(type);
    if (!tb || n < 0 || experts < 1 || experts > GEM_NLR_MAX_EXPERTS || k < 1 || k > kMaxChosen || (score != GEM_NLR_SOFTMAX && score != GEM_NLR_SIGMOID) ||
        (renormalize != 0 && renormalize != 1) || !isfinite(scale) || n > INT32_MAX / k)
        return GEM_NLR_E_INVALID;
    if (n == 0) return GEM_NLR_OK;
    if (!logits_dev || !aligned_to(logits_dev, tb) || ld < 0 || !ints(dweight_dev) || !ints(expert_dev) || !dlogits_dev || !aligned_to(dlogits_dev, tb) ||
        ld_d < experts || dlogits_dev == logits_dev)
        return GEM_NLR_E_INVALID;
    const RouteGrad r = {dweight_dev, logits_dev, ld, expert_dev, n, experts, k, score, renormalize, scale, dlogits_dev, ld_d};
    const int64_t blocks = (n + 7) / 8, most = (int64_t)kTrainSMs * 32;
    return by_type(type, [&](auto t) {
        return by_experts(experts, [&](auto v) {
            k_route_backward<v.value, decltype(t)><<<(unsigned)(blocks < most ? blocks : most), 256, 0, (cudaStream_t)cuda_stream>>>(r);
            return launched();
        });
    });
}
