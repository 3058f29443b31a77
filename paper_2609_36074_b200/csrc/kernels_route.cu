// Routing rows to experts: scores, the choice, the weights, the order of the experts' rows, and the weights' gradient.
//
//   s = softmax(z) or 1 / (1 + exp(-z));  c = s + b;  the k largest c of the kept groups (without b: the k largest z)
//   w_j = scale s_j / sum_l s_l (or scale s_j)
//
// A warp a row, up to 16 neighbouring logits a lane.  Scores become unsigned keys in their order, so that the largest of 32 lanes is
// one warp reduction; the lowest lane among equals, and in it the lowest logit, is the lowest index.  A round of the choice is that
// reduction, a vote and the owner's next best.  The FP32 scores of the choice are right to about 2^-20, which does not tell
// neighbours apart: where two scores that follow one another in the choice are nearer than that (and are not the same logit with
// the same bias, which are equal in any precision), the row is chosen again in FP64.  One row in a hundred is, at 128 experts with
// sigmoid scores.  Weights are taken from the chosen logits anew, one a lane.
//
// The order is a counting sort that keeps the rows of an expert in order, without atomics whose order shows: blocks own
// consecutive rows and count their experts; the second kernel adds the counts of the blocks before (each block reads all of
// them, 148 x experts numbers), takes sums over the experts, and gives out places in order, a warp's 32 entries at a time by
// matching equal experts.  Few rows are one block and one launch.
#include "expert_common.cuh"

namespace gemnlr {
namespace {

// Threads of a block: 1024 where 64 registers a thread suffice.  (Fewer, larger blocks: fewer counts to add.)
template <int V> constexpr int kBlockThreads = V <= 4 ? 1024 : 512;
constexpr int kBlocks = kTrainSMs * 2;             // at most
constexpr int kMaxChosen = 32, kMaxGroups = 32;
constexpr unsigned kAll = 0xffffffffu;

struct Route {
    const void* z;
    int64_t ld;
    const float* bias;
    int64_t n;
    int experts, k, score, groups, kept, best, renorm;
    int wide;               // a lane's logits are one vector
    int group_lanes;        // lanes that hold a group's experts; 0 where groups end inside a lane's or are not a power of two of lanes
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

// (NaNs are left out.)
__device__ __forceinline__ float warp_top(float v)
{
    float t;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(t) : "f"(v));
    return t;
}

// How far the choice's FP32 scores can be off: 2^-18 of a score that is at most 1 (the exponential is off by 2^-21 of itself and by
// its argument's rounding, x exp(-x) <= 0.37; a sum of 16 and 5 steps, a quotient and the sum with the bias add 30 units of 2^-24), and a
// rounding of the bias.
__device__ __forceinline__ float margin_of(float c) { return 0x1p-18f + 0x1p-21f * fabsf(c); }

// A lane's candidates: experts lane * V + v.  `at` are their v, in the order of `key` where they are kept sorted (the same v first
// among equals).
template <int V, typename K> struct Candidates {
    static constexpr bool SORTED = V <= 4;              // more are searched anew when the best is taken
    K key[V], top;
    int at[V], best;
    int lane;
    __device__ __forceinline__ void search()
    {
        top = key[0];
        best = 0;
#pragma unroll
        for (int v = 1; v < V; ++v)
            if (key[v] > top) { top = key[v]; best = v; }
    }
    __device__ __forceinline__ void begin()
    {
        if constexpr (SORTED) {
#pragma unroll
            for (int v = 0; v < V; ++v) at[v] = v;
#pragma unroll
            for (int round = 0; round < V; ++round)
#pragma unroll
                for (int v = round & 1; v + 1 < V; v += 2)
                    if (key[v + 1] > key[v]) {
                        const K k = key[v]; key[v] = key[v + 1]; key[v + 1] = k;
                        const int a = at[v]; at[v] = at[v + 1]; at[v + 1] = a;
                    }
            top = key[0];
            best = at[0];
        } else {
            search();
        }
    }
    __device__ __forceinline__ void take()
    {
        if constexpr (SORTED) {
#pragma unroll
            for (int v = 0; v + 1 < V; ++v) { key[v] = key[v + 1]; at[v] = at[v + 1]; }
            key[V - 1] = 0;
            top = key[0];
            best = at[0];
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v == best) key[v] = 0;
            search();
        }
    }
};

// The k best keys into `got` (lane j: the j-th's index, -1 for none).  near(key, index, key, index) is told of each two that follow one
// another, and of the last and the one after it.  Returns whether it ever said that they are too near.
template <int V, typename K, typename N>
__device__ __forceinline__ bool choose(Candidates<V, K>& c, int k, int& got, N near)
{
    const int lane = c.lane;
    K last = 0;
    int before = -1;
    bool unsure = false;
    got = -1;
    c.begin();
    for (int j = 0; j <= k; ++j) {
        const K best = warp_max(c.top);
        if (is_none(best)) break;
        const int owner = __ffs(__ballot_sync(kAll, c.top == best)) - 1;
        const int index = owner * V + __shfl_sync(kAll, c.best, owner);
        if (j > 0 && near(last, before, best, index)) unsure = true;
        if (j == k) break;
        if (lane == j) got = index;
        last = best;
        before = index;
        if (lane == owner) c.take();
    }
    return unsure;
}

// Leaves only the kept groups' keys.  S: float or double; by[v]: the score of the lane's v-th expert that its group is judged by
// (-inf: none).  Returns whether the border between kept groups and others is nearer than FP32 tells (`scored`).
template <int V, typename S, typename K>
__device__ __forceinline__ bool keep_groups(Candidates<V, K>& c, const Route& r, const S (&by)[V], bool scored)
{
    const int size = r.experts / r.groups, lane = c.lane;
    const S none = -(S)INFINITY;
    S mine = none;                                       // the score of the group `me`
    int me = r.groups, every = 1;                        // groups' scores are held by lanes 0, every, 2 every, ...
    if (r.group_lanes) {
        S first = none, second = none;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const S x = lane * V + v < r.experts ? by[v] : none;
            second = fmax(second, fmin(first, x));
            first = fmax(first, x);
        }
        for (int o = 1; o < r.group_lanes; o *= 2) {
            const S a = __shfl_xor_sync(kAll, first, o), b = __shfl_xor_sync(kAll, second, o);
            second = fmax(fmin(first, a), fmax(second, b));
            first = fmax(first, a);
        }
        every = r.group_lanes;
        if (lane / every < r.groups) {
            me = lane / every;
            mine = r.best == 2 && second != none ? first + second : first;
        }
    } else {
        for (int g = 0; g < r.groups; ++g) {
            S first = none, second = none;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = lane * V + v;
                const S x = i >= g * size && i < (g + 1) * size ? by[v] : none;
                second = fmax(second, fmin(first, x));
                first = fmax(first, x);
            }
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const S a = __shfl_xor_sync(kAll, first, o), b = __shfl_xor_sync(kAll, second, o);
                second = fmax(fmin(first, a), fmax(second, b));
                first = fmax(first, a);
            }
            if (lane == g) {
                me = g;
                mine = r.best == 2 && second != none ? first + second : first;
            }
        }
    }
    int rank = 0;
    for (int g = 0; g < r.groups; ++g) {
        const S other = __shfl_sync(kAll, mine, g * every);
        rank += other > mine || (other == mine && g < me);
    }
    const bool kept = me < r.groups && rank < r.kept;
    if (r.group_lanes) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (!kept) c.key[v] = 0;
    } else {
        const unsigned stays = __ballot_sync(kAll, kept);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int g = min((lane * V + v) / size, 31);
            if (!(stays >> g & 1u)) c.key[v] = 0;
        }
    }
    if (!scored) return false;
    // the lowest of those kept and the highest of the others
    const K low = ~warp_max((K)~key_of(kept ? mine : (S)INFINITY)), high = warp_max(key_of(me < r.groups && !kept ? mine : none));
    const float x = (float)score_of(low), y = (float)score_of(high);
    return !is_none(high) && !(x - y > 2.0f * margin_of(x));
}

// The choice in FP64, for rows whose FP32 scores do not decide it.
template <int V>
__device__ __noinline__ int choose_in_64_bits(const Route& r, const float (&z)[V], int lane)
{
    double s[V], sum = 0.0;
    float m = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) m = fmaxf(m, z[v]);
    m = warp_top(m);
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
        const int i = lane * V + v;
        if (r.score == GEM_NLR_SOFTMAX) s[v] /= sum;
        double x = r.bias ? s[v] + (double)(i < r.experts ? __ldg(r.bias + i) : 0.f) : (double)z[v];
        if (z[v] == -INFINITY) x = -(double)INFINITY;
        c.key[v] = i < r.experts ? key_of(x) : 0;
        if (!r.bias && r.best == 1) s[v] = (double)z[v];
        else if (r.bias) s[v] = x;
        if (z[v] == -INFINITY) s[v] = -(double)INFINITY;
    }
    if (r.groups > 1) keep_groups<V, double>(c, r, s, false);
    int got;
    choose(c, r.k, got, [](uint64_t, int, uint64_t, int) { return false; });
    return got;
}

// A lane's V logits.
template <int V, typename T>
__device__ __forceinline__ void load_logits(const T* zr, const Route& r, int lane, float (&z)[V])
{
    constexpr int BYTES = V * (int)sizeof(T);
    if (BYTES >= 4 && r.wide && lane * V + V <= r.experts) {
        uint32_t w[(BYTES + 3) / 4];
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) *reinterpret_cast<uint4*>(w + 4 * i) = *(reinterpret_cast<const uint4*>(zr + lane * V) + i);
        } else if constexpr (BYTES == 8) {
            *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(zr + lane * V);
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(zr + lane * V);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = to_f(reinterpret_cast<const T*>(w)[v]);
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = lane * V + v < r.experts ? to_f(zr[lane * V + v]) : -INFINITY;
    }
}

// One row by one warp.
template <int V, typename T>
__device__ __forceinline__ void route_row(const Route& r, int64_t row, int lane, const float (&bias)[V], int& chosen)
{
    const T* zr = reinterpret_cast<const T*>(r.z) + row * r.ld;
    const bool soft = r.score == GEM_NLR_SOFTMAX;
    float z[V], m = -INFINITY;
    load_logits<V>(zr, r, lane, z);
    bool bad = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bad |= z[v] != z[v] || (soft && z[v] == INFINITY);
        m = fmaxf(m, z[v]);
    }
    const bool scored = r.bias || (r.groups > 1 && r.best == 2);          // the choice needs the scores
    float sum = 0.0f;
    Candidates<V, uint32_t> c;
    c.lane = lane;
    float by[V];
    if (scored) {
        // exponentials to 2^-21: close neighbours are chosen in FP64
        float e[V];
        if (soft) {
            m = warp_top(m);
#pragma unroll
            for (int v = 0; v < V; ++v) { e[v] = z[v] == -INFINITY ? 0.0f : __expf(z[v] - m); sum += e[v]; }
            sum = warp_sum(sum);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float s = soft ? __fdividef(e[v], sum) : __fdividef(1.0f, 1.0f + __expf(-z[v]));
            const float x = s + bias[v];
            const bool there = z[v] != -INFINITY;
            bad |= there && x != x;
            c.key[v] = lane * V + v < r.experts ? key_of(!there ? -INFINITY : r.bias ? x : z[v]) : 0;
            by[v] = there ? x : -INFINITY;
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            c.key[v] = lane * V + v < r.experts ? key_of(z[v]) : 0;
            by[v] = z[v];
        }
    }
    int got = -1;
    bad = __any_sync(kAll, bad);
    if (!bad) {
        // the same logit with the same bias is equal in any precision; other neighbours within the margin are not decided
        const auto near = [&](uint32_t a, int i, uint32_t b, int j) {
            if (!r.bias) return false;
            const float x = score_of(a), y = score_of(b);
            if (x - y > margin_of(x)) return false;
            return !(to_f(zr[i]) == to_f(zr[j]) && __ldg(r.bias + i) == __ldg(r.bias + j));
        };
        bool unsure = false;
        if (r.groups > 1) unsure = keep_groups<V, float>(c, r, by, scored);
        unsure |= choose(c, r.k, got, near);
        if (unsure) got = choose_in_64_bits<V>(r, z, lane);
    }
    // weights: lane j has the j-th chosen expert
    float w = 0.0f;
    if (bad) {
        w = __uint_as_float(0x7fc00000u);
    } else {
        const float x = got >= 0 ? to_f(zr[got]) : -INFINITY;
        const auto logistic = [](float v) { return 1.0f / (1.0f + expf(-v)); };
        if (r.renorm) {
            float e = 0.0f, total;
            if (!soft) {
                if (got >= 0) e = logistic(x);
                total = warp_sum(e);
            }
            if (soft || total < 1e-30f) {
                // a softmax over the chosen logits, or the logarithms of their scores: neither underflows
                const float l = got < 0 ? -INFINITY : soft ? x : fminf(x, 0.0f) - log1pf(expf(-fabsf(x)));
                const float top = warp_top(l);
                e = got >= 0 ? expf(l - top) : 0.0f;
                total = warp_sum(e);
            }
            if (got >= 0) w = e / total * r.scale;
        } else if (soft) {
            m = warp_top(m);
            sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) sum += z[v] == -INFINITY ? 0.0f : expf(z[v] - m);
            sum = warp_sum(sum);
            if (got >= 0) w = expf(x - m) / sum * r.scale;
        } else if (got >= 0) {
            w = logistic(x) * r.scale;
        }
    }
    if (lane < r.k) {
        r.expert[row * r.k + lane] = got;
        r.weight[row * r.k + lane] = w;
    }
    chosen = got;
}

// Places for the rows of this block's warps.  at: warps x experts, each warp's counts, replaced by the place of its next row of
// each expert; first: the place of the block's first row of each expert.
template <int NT>
__device__ __forceinline__ void give_places(const Route& r, int32_t* at, const int32_t* first, int64_t begin, int64_t end)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int e = threadIdx.x; e < r.experts; e += NT) {
        int32_t next = first[e];
        for (int w = 0; w < (NT / 32); ++w) {
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

// Exclusive sums of total[experts] into first[experts + 1], by one block.  (experts <= NT)
template <int NT>
__device__ __forceinline__ void sums_over_experts(const int32_t* total, int32_t* first, int experts)
{
    __shared__ int32_t of_warp[(NT / 32)];
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

template <int NT>
__device__ __forceinline__ void leave_rest(const Route& r, int32_t used)
{
    for (int64_t p = used + (int64_t)blockIdx.x * NT + threadIdx.x; p < r.n * r.k; p += (int64_t)gridDim.x * NT) r.row[p] = -1;
}

// Shared memory: warps x experts counts; ONE: and experts + 1 sums and experts totals.
template <int V, typename T, bool ONE>
__global__ void __launch_bounds__(kBlockThreads<V>)
k_route(const __grid_constant__ Route r)
{
    constexpr int NT = kBlockThreads<V>;
    extern __shared__ int32_t at[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < (NT / 32) * r.experts; i += NT) at[i] = 0;
    __syncthreads();
    const int64_t begin = min(r.n, ((int64_t)blockIdx.x * (NT / 32) + warp) * r.rows_per_warp), end = min(r.n, begin + r.rows_per_warp);
    int32_t* mine = at + warp * r.experts;
    float bias[V];
#pragma unroll
    for (int v = 0; v < V; ++v) bias[v] = r.bias && lane * V + v < r.experts ? __ldg(r.bias + lane * V + v) : 0.0f;
    for (int64_t row = begin; row < end; ++row) {
        int got;
        route_row<V, T>(r, row, lane, bias, got);
        if (got >= 0) mine[got] += 1;                    // a row's experts differ
        __syncwarp();
    }
    __syncthreads();
    next_may_start();
    int32_t* first = at + (NT / 32) * r.experts;
    int32_t* total = ONE ? first + r.experts + 1 : r.counts + (int64_t)blockIdx.x * r.experts;
    for (int e = threadIdx.x; e < r.experts; e += NT) {
        int32_t c = 0;
        for (int w = 0; w < (NT / 32); ++w) c += at[w * r.experts + e];
        total[e] = c;
    }
    if constexpr (ONE) {
        __syncthreads();
        sums_over_experts<NT>(total, first, r.experts);
        for (int e = threadIdx.x; e <= r.experts; e += NT) r.offset[e] = first[e];
        give_places<NT>(r, at, first, begin, end);
        leave_rest<NT>(r, first[r.experts]);
    }
}

// Shared memory: warps x experts counts, then experts + 1 sums, experts totals, experts counts of the blocks before.
template <int NT>
__global__ void __launch_bounds__(NT)
k_route_places(const __grid_constant__ Route r, int blocks)
{
    extern __shared__ int32_t at[];
    int32_t* first = at + (NT / 32) * r.experts;
    int32_t* total = first + r.experts + 1;
    int32_t* before = total + r.experts;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < (NT / 32) * r.experts + 3 * r.experts + 1; i += NT) at[i] = 0;
    __syncthreads();
    const int64_t begin = min(r.n, ((int64_t)blockIdx.x * (NT / 32) + warp) * r.rows_per_warp), end = min(r.n, begin + r.rows_per_warp);
    grid_ready();
    for (int64_t i = begin * r.k + lane; i < end * r.k; i += 32) {
        const int e = r.expert[i];
        if (e >= 0) atomicAdd(at + warp * r.experts + e, 1);
    }
    // threads in pairs (expert, share of the blocks); whole numbers: the order of the additions does not show
    const int shares = max(1, NT / r.experts), share = threadIdx.x / r.experts;
    if (share < shares)
        for (int e = threadIdx.x % r.experts; e < r.experts; e += NT) {
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
    sums_over_experts<NT>(total, first, r.experts);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= r.experts; e += NT) r.offset[e] = first[e];
    for (int e = threadIdx.x; e < r.experts; e += NT) before[e] += first[e];
    __syncthreads();
    give_places<NT>(r, at, before, begin, end);
    leave_rest<NT>(r, first[r.experts]);
}

struct RouteGrad {
    const float* dweight;
    const void* z;
    int64_t ld;
    const int32_t* expert;
    int64_t n;
    int experts, k, score, renorm;
    int wide;               // rows of whole vectors of eight
    float scale;
    void* dz;
    int64_t ldd;
};

template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}
template <int LANES> __device__ __forceinline__ float lanes_top(float v)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}

// LANES lanes a row, V neighbouring logits a lane.  Slots are taken LANES at a time, a slot a lane; each lane then picks up the shares of
// its own experts.
template <int LANES, int V, typename T>
__global__ void __launch_bounds__(256)
k_route_backward(const __grid_constant__ RouteGrad r)
{
    constexpr int ROWS = 256 / LANES;
    const int lane = threadIdx.x & 31, me = lane % LANES;
    const bool soft = r.score == GEM_NLR_SOFTMAX;
    const bool whole = soft && !r.renorm;                  // every logit has a share
    const int64_t steps = (r.n + ROWS - 1) / ROWS;
    for (int64_t step = blockIdx.x; step < steps; step += gridDim.x) {
        const int64_t row = step * ROWS + threadIdx.x / LANES;
        const bool in = row < r.n;
        const T* zr = reinterpret_cast<const T*>(r.z) + (in ? row : 0) * r.ld;
        float z[V], m = -INFINITY, sum = 0.0f;
        if (whole) {
#pragma unroll
            for (int i = 0; i < V; ++i) z[i] = -INFINITY;
            if (in && me * V < r.experts) {
                if (r.wide) {
                    float v8[8];
#pragma unroll
                    for (int b = 0; b < V / 8; ++b) {
                        if (me * V + 8 * b >= r.experts) break;
                        load8<true>(zr + me * V + 8 * b, 8, v8);
#pragma unroll
                        for (int i = 0; i < 8; ++i) z[8 * b + i] = v8[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (me * V + i < r.experts) z[i] = to_f(zr[me * V + i]);
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) m = fmaxf(m, z[i]);
            m = lanes_top<LANES>(m);
            // a NaN among the logits is lost in the maximum and comes back in the sum
#pragma unroll
            for (int i = 0; i < V; ++i) {
                z[i] = z[i] == -INFINITY ? 0.0f : expf(z[i] - m);
                sum += z[i];
            }
            sum = lanes_sum<LANES>(sum);
        }
        // the slots: weights' shares first (their sum over all slots), then each lane's own
        const int rounds = (r.k + LANES - 1) / LANES;
        float top = -INFINITY, total = 0.0f, t = 0.0f;
        bool any = false;
        const auto slot = [&](int round, int& e, float& v, float& x) {
            const int j = round * LANES + me;
            e = in && j < r.k ? __ldg(r.expert + row * r.k + j) : -1;
            if (e >= r.experts) e = -1;
            v = e >= 0 ? __ldg(r.dweight + row * r.k + j) * r.scale : 0.0f;
            x = e >= 0 ? to_f(zr[e]) : -INFINITY;
            any |= e >= 0;
        };
        const auto log_score = [&](float x) { return soft || x == -INFINITY ? x : fminf(x, 0.0f) - log1pf(expf(-fabsf(x))); };
        float l0 = 0.0f, v0 = 0.0f, x0 = 0.0f;              // the first round's, which mostly is the only one
        int e0 = -1;
        if (r.renorm) {
            for (int q = 0; q < rounds; ++q) {
                int e; float v, x;
                slot(q, e, v, x);
                const float l = log_score(x);
                if (q == 0) { e0 = e; v0 = v; x0 = x; l0 = l; }
                top = fmaxf(top, l);
            }
            top = lanes_top<LANES>(top);
            for (int q = 0; q < rounds; ++q) {
                int e = e0; float v = v0, x = x0, l = l0;
                if (q > 0) { slot(q, e, v, x); l = log_score(x); }
                const float p = e >= 0 && x != -INFINITY ? expf(l - top) : 0.0f;
                total += p;
                t += p * v;
            }
            total = lanes_sum<LANES>(total);
            t = lanes_sum<LANES>(t);
            if (total != 0.0f) t /= total;
        } else {
            for (int q = 0; q < rounds; ++q) {
                int e; float v, x;
                slot(q, e, v, x);
                if (q == 0) { e0 = e; v0 = v; x0 = x; }
                if (whole && e >= 0 && x != -INFINITY) t += expf(x - m) / sum * v;
            }
            if (whole) t = lanes_sum<LANES>(t);
        }
        float out[V];
        if (whole) {
            unsigned has = __ballot_sync(kAll, any);
            any = has >> (lane - me) & (LANES == 32 ? kAll : (1u << (LANES & 31)) - 1u);
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = any && sum > 0.0f ? -(z[i] / sum) * t : any && sum != sum ? sum : 0.0f;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) out[i] = 0.0f;
        }
        for (int q = 0; q < rounds; ++q) {
            int e = e0; float v = v0, x = x0, l = l0;
            if (q > 0) { slot(q, e, v, x); l = r.renorm ? log_score(x) : 0.0f; }
            float g;
            if (whole) {
                g = expf(x - m) / sum * v;
            } else {
                const float rest = soft ? 1.0f : 1.0f / (1.0f + expf(x));          // 1 - s
                g = r.renorm ? (total != 0.0f ? expf(l - top) / total : 0.0f) * (v - t) * rest : v * rest / (1.0f + expf(-x));
            }
            if (e < 0 || x == -INFINITY) g = 0.0f;
            const int most = min(LANES, r.k - q * LANES);
            for (int j = 0; j < most; ++j) {
                const int at = __shfl_sync(kAll, e, j, LANES) - me * V;
                const float add = __shfl_sync(kAll, g, j, LANES);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i == at) out[i] += add;
            }
        }
        if (in) {
            T* dr = reinterpret_cast<T*>(r.dz) + row * r.ldd;
            if (r.wide) {
#pragma unroll
                for (int b = 0; b < V / 8; ++b) {
                    if (me * V + 8 * b >= r.experts) break;
                    float v8[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v8[i] = out[8 * b + i];
                    store8<true>(dr + me * V + 8 * b, 8, v8);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (me * V + i < r.experts) dr[me * V + i] = from_f<T>(out[i]);
            }
        }
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

// Up to this many rows one block routes and sorts.
constexpr int64_t kOneBlockRows = 64;
bool one_block(int64_t n) { return n <= kOneBlockRows; }

template <typename F, typename... Args>
cudaError_t launch_route(F kern, int grid, int threads, int shared, bool early, cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = early;
    return cudaLaunchKernelEx(&cfg, kern, args...);
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
    return by_type(type, [&](auto t) {
        return by_experts(experts, [&](auto v) {
            using T = decltype(t);
            constexpr int V = v.value, NT = kBlockThreads<V>, WARPS = NT / 32, BYTES = V * (int)sizeof(T) < 16 ? V * (int)sizeof(T) : 16;
            const int64_t slots = (int64_t)(kBlocks * 512 / NT) * WARPS, per_warp = one ? (n + WARPS - 1) / WARPS : (n + slots - 1) / slots;
            const int blocks = one ? 1 : (int)((n + per_warp * WARPS - 1) / (per_warp * WARPS));
            const int size = experts / groups, lanes = size % V ? 0 : size / V;
            const bool wide = aligned_to(logits_dev, BYTES) && ld * (int64_t)sizeof(T) % BYTES == 0;
            const Route r = {logits_dev, ld, bias_dev, n, experts, k, score, groups, kept_groups, group_best, renormalize, wide, lanes & (lanes - 1) ? 0 : lanes, scale,
                             expert_dev, weight_dev, offset_dev, row_dev, place_dev, (int32_t*)scratch_dev, per_warp};
            const int counts = WARPS * experts * 4;
            cudaStream_t st = (cudaStream_t)cuda_stream;
            if (one) return told(launch_route(k_route<V, T, true>, 1, NT, counts + (2 * experts + 1) * 4, false, st, r));
            cudaError_t rc = launch_route(k_route<V, T, false>, blocks, NT, counts, false, st, r);
            if (rc == cudaSuccess) rc = launch_route(k_route_places<NT>, blocks, NT, counts + (3 * experts + 1) * 4, true, st, r, blocks);
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
    const bool wide = experts % 8 == 0 && wide_rows(logits_dev, ld, tb) && wide_rows(dlogits_dev, ld_d, tb);
    const RouteGrad r = {dweight_dev, logits_dev, ld, expert_dev, n, experts, k, score, renormalize, wide, scale, dlogits_dev, ld_d};
    return by_type(type, [&](auto t) {
        const auto run = [&](auto lanes, auto v) {
            constexpr int ROWS = 256 / lanes.value;
            const int64_t blocks = (n + ROWS - 1) / ROWS, most = (int64_t)kTrainSMs * 64;
            k_route_backward<lanes.value, v.value, decltype(t)><<<(unsigned)(blocks < most ? blocks : most), 256, 0, (cudaStream_t)cuda_stream>>>(r);
            return launched();
        };
        using std::integral_constant;
        if (experts <= 32) return run(integral_constant<int, 4>{}, integral_constant<int, 8>{});
        if (experts <= 64) return run(integral_constant<int, 8>{}, integral_constant<int, 8>{});
        if (experts <= 128) return run(integral_constant<int, 16>{}, integral_constant<int, 8>{});
        if (experts <= 256) return run(integral_constant<int, 32>{}, integral_constant<int, 8>{});
        return run(integral_constant<int, 32>{}, integral_constant<int, 16>{});
    });
}
