// The experts' products on the tensor cores (tcgen05 + TMEM): FP16 or BF16 operands, FP32 accumulators.
//
//   rows      C_p = A_row(p) B_e  for the places p of expert e        (y = x W; dx = dy W^T)
//   weights   C_e = sum over e's places of A_row(p)^T B_row(p)          (dW = x^T dy)
//
// One persistent block an SM walks over tiles of 128 x BN of C; no tile spans two experts.  With `rows` an expert's rows are
// the M dimension (a tile's rows behind the expert's last are computed and not stored), with `weights` they are the K dimension
// (a stage's rows behind the last are zeros).  A stage holds 64 of K for both operands, in 128-byte rows with the 128-byte
// swizzle, K-major where the matrix is contiguous along K and MN-major where it is contiguous along M or N: nothing is transposed.
//
//   warp 0       loads by TMA, four to eight stages ahead; rows that are gathered come four at a time by their indices
//   warp 1       issues the MMAs
//   warps 4-7    epilogue: accumulators out of TMEM (double-buffered), rounded once, through shared memory into 128-byte
//                row pieces
//   warps 8-11   (matrices whose rows do not begin on 16 bytes) load instead of warp 0, by ordinary loads
//
// Every wait is bounded; after one that runs out the block issues nothing more and its remaining tiles are NaN.
#include <cuda.h>
#include <cudaTypedefs.h>
#include "train_common.cuh"
#include "pipeline.cuh"
#include "tc_common.cuh"

namespace gemnlr {
namespace {

constexpr int kTileM = 128;
constexpr int kChunk = 64;                        // of K a stage: 128 bytes
constexpr int kRow = kChunk * 2;                  // bytes of a row in shared memory
constexpr int kLoaders = 128;                     // threads of the ordinary loads

enum Mode { kRowsTimesPlain = 0, kRowsTimesTurned = 1, kWeights = 2 };

template <int BN> struct Shape {
    static constexpr int A = kTileM * kRow, B = BN * kRow, STAGE = A + B;
    static constexpr int STAGES = BN == 256 ? 4 : BN == 128 ? 6 : 8;
    static constexpr int STAGING = 4 * 2048;      // a warp's 32 rows of 32 columns
    static constexpr int BARRIERS = 2 * STAGES + 5;
    static constexpr int TABLES = (2 * GEM_NLR_MAX_EXPERTS + 4) * 4;
    static constexpr int SHARED = 1024 + STAGES * STAGE + STAGING + TABLES + BARRIERS * 8 + 16;
};

struct Operand {
    const uint16_t* p;
    int64_t ld, stride;       // elements from one row to the next, from one expert to the next (0: not the experts')
    int64_t rows;             // rows there are, of one expert where there are experts
    int columns;
    int gather;               // rows are named by row[]
    int wide;                 // rows begin on 16 bytes
};

struct Product {
    CUtensorMap ta, tb;       // boxes of rows
    CUtensorMap ra, rb;       // two SMs: single rows, for loads by index
    Operand a, b;
    const int32_t* offset;
    const int32_t* row;
    int64_t places;
    int experts, m, n, k;     // m: of C_e (weights); k: of the rows' products
    uint16_t* c;
    int64_t ldc, stride_c;
    int c_wide;
    uint32_t idesc;
    int bf16;
};

// (C is in memory, and a tile has at least 32 of its elements: tiles are counted in 32 bits.)
struct Tile {
    int expert;
    int c_row, stop;          // first row of C and the one behind the last (rows: places; weights: of C_e)
    int n0;
    int k_first;              // weights: first place
    int k;                    // length of the sum
};

__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile uint32_t* dead, uint32_t limit = kSpinLimit)
{
    for (uint32_t i = 0; i < limit; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63u) == 63u && *dead) return false;
    }
    *dead = 1u;
    return false;
}

__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
}

__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// 64 columns of four rows; rows outside the matrix are zeros.
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, int x, int4 y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(x), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w), "r"(bar) : "memory");
}

// first[e]: e's first place (falling or wild offsets cut to what is possible), tile0[e]: its first row of tiles; behind the
// experts the places without one.  HEIGHT: of a tile.  By one warp.
template <int HEIGHT>
__device__ __forceinline__ void make_tables(const Product& q, int32_t* first, int32_t* tile0, int lane)
{
    int32_t reached = 0, tiles = 0, before = 0;
    for (int e0 = 0; e0 <= q.experts + 1; e0 += 32) {
        const int e = e0 + lane;
        int32_t v = e == 0 ? 0 : e < q.experts + 1 ? __ldg(q.offset + e) : (int32_t)q.places;
        v = max(0, min(v, (int32_t)q.places));
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v = max(v, u);
        }
        v = max(v, reached);
        int32_t prev = __shfl_up_sync(0xffffffffu, v, 1);
        if (lane == 0) prev = before;
        int32_t t = e == 0 ? 0 : (int32_t)(((int64_t)v - prev + HEIGHT - 1) / HEIGHT);   // row tiles of e - 1
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t u = __shfl_up_sync(0xffffffffu, t, o);
            if (lane >= o) t += u;
        }
        t += tiles;
        if (e <= q.experts + 1) {
            first[e] = v;
            tile0[e] = t;
        }
        reached = before = __shfl_sync(0xffffffffu, v, 31);
        tiles = __shfl_sync(0xffffffffu, t, 31);
    }
}

template <int MODE, int BN, int HEIGHT = kTileM>
__device__ __forceinline__ Tile tile_at(const Product& q, const int32_t* first, const int32_t* tile0, int t)
{
    Tile w;
    const int nt = (q.n + BN - 1) / BN;
    const int row_tile = t / nt;
    w.n0 = (t - row_tile * nt) * BN;
    if (MODE == kWeights) {
        const int mt = (q.m + HEIGHT - 1) / HEIGHT;
        w.expert = row_tile / mt;
        w.c_row = (row_tile - w.expert * mt) * HEIGHT;
        w.stop = q.m;
        w.k_first = first[w.expert];
        w.k = first[w.expert + 1] - first[w.expert];
    } else {
        int lo = 0, hi = q.experts;                                  // the last with tile0[e] <= row_tile
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tile0[mid] <= row_tile) lo = mid; else hi = mid - 1;
        }
        w.expert = lo;
        w.c_row = first[lo] + (row_tile - tile0[lo]) * HEIGHT;
        w.stop = first[lo + 1];
        w.k_first = 0;
        w.k = lo == q.experts ? 0 : q.k;                             // places without an expert: zeros
    }
    return w;
}

// The row of operand o that stands for place p, -1 for none.
__device__ __forceinline__ int64_t row_of(const Operand& o, const int32_t* row, int64_t p)
{
    const int64_t r = o.gather ? (int64_t)__ldg(row + p) : p;
    return r >= 0 && r < o.rows ? r : -1;
}

// The rows of places p to p + 3, in the form that a gathered load takes: behind the last row, whose values are zeros, for none.
__device__ __forceinline__ int4 four_rows(const int32_t* row, int64_t p, int64_t stop, int64_t rows)
{
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = p + i < stop ? (uint32_t)__ldg(row + p + i) : 0x7fffffffu;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = r[i] < (uint32_t)rows ? r[i] : (uint32_t)rows;
    return make_int4((int)r[0], (int)r[1], (int)r[2], (int)r[3]);
}

// R rows of 128 bytes by ordinary loads.  K_MAJOR: row r is M or N index mn0 + r, its 64 columns the stage's K; else row r of box b is
// K index r, its columns 64 M or N indices from mn0 + 64 b.  place0 >= 0: the rows are places from there on, up to `stop`; else rows of the expert.
template <bool K_MAJOR, int R>
__device__ __forceinline__ void load_ordinary(const Operand& o, const int32_t* row, int expert, int64_t row0, int64_t stop, bool by_place, int column0,
                                              int columns, uint32_t dst, int thread)
{
    const uint16_t* base = o.p + expert * o.stride;
    constexpr int BATCH = R / 16 < 8 ? R / 16 : 8;
    const int c = thread & 7;
#pragma unroll 1
    for (int i0 = 0; i0 < R / 16; i0 += BATCH) {
        uint4 v[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int r = (thread >> 3) + 16 * (i0 + i);
            const int64_t at = row0 + (K_MAJOR ? r : r & 63);
            const int col = column0 + (K_MAJOR ? 0 : (r >> 6) * 64) + c * 8;
            const int many = columns - col;
            int64_t from = -1;
            if (at < stop && many > 0) from = by_place ? row_of(o, row, at) : at;
            v[i] = make_uint4(0, 0, 0, 0);
            if (from >= 0) {
                const uint16_t* p = base + from * o.ld + col;
                if (o.wide && many >= 8) {
                    v[i] = __ldg(reinterpret_cast<const uint4*>(p));
                } else {
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < many) w[j >> 1] |= (uint32_t)__ldg(p + j) << (16 * (j & 1));
                    v[i] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int r = (thread >> 3) + 16 * (i0 + i);
            sts128u(dst + (uint32_t)(r * kRow + ((c ^ (r & 7)) << 4)), v[i]);
        }
    }
}

// A warp's 32 rows of `steps` times 32 columns of a tile, from accumulator column `acc` (the warp's lanes) into C from (row0, col0) on;
// zeros where no sum was taken, NaN where a wait ran out.  32 columns at a time go through the warp's 2 KB of shared memory, so
// that rows are stored in pieces of 64 bytes.
template <int MODE>
__device__ __forceinline__ void store_tile(const Product& q, const Tile& w, int row0, int col0, int steps, uint32_t acc, uint32_t mine, int lane, bool on)
{
    uint16_t* c = q.c + (MODE == kWeights ? w.expert * q.stride_c : 0) + row0 * q.ldc;
    const int rows = min(32, w.stop - row0);
    const uint32_t to_stage = mine + (uint32_t)(lane * 64), phase = (uint32_t)(lane >> 1) & 3u;
    const uint32_t from_stage = mine + (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4));
#pragma unroll 1
    for (int g = 0; g < steps && col0 < q.n; ++g, col0 += 32) {
        float v[32];
        if (w.k && on) {
            tmem_ld32(acc + (uint32_t)(g * 32), v);
        } else {
            const float fill = on ? 0.0f : __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int x = 0; x < 32; ++x) v[x] = fill;
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            uint32_t h[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const float lo = v[x * 8 + 2 * y], hi = v[x * 8 + 2 * y + 1];
                if (q.bf16) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
                    h[y] = *reinterpret_cast<const uint32_t*>(&p);
                } else {
                    const __half2 p = __floats2half2_rn(lo, hi);
                    h[y] = *reinterpret_cast<const uint32_t*>(&p);
                }
            }
            sts128u(to_stage + (((uint32_t)x ^ phase) << 4), make_uint4(h[0], h[1], h[2], h[3]));
        }
        __syncwarp();
        const int col = col0 + (lane & 3) * 8;
        uint16_t* to = c + (int64_t)(lane >> 2) * q.ldc + col;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float4 f = lds128(from_stage + (uint32_t)(x * 512));
            if (8 * x + (lane >> 2) < rows && col < q.n) {
                uint16_t* at = to + (int64_t)(8 * x) * q.ldc;
                const uint32_t h[4] = {__float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(f.z), __float_as_uint(f.w)};
                if (q.c_wide && col + 8 <= q.n) {
                    *reinterpret_cast<uint4*>(at) = make_uint4(h[0], h[1], h[2], h[3]);
                } else {
#pragma unroll
                    for (int y = 0; y < 8; ++y)
                        if (col + y < q.n) at[y] = (uint16_t)(h[y >> 1] >> (16 * (y & 1)));
                }
            }
        }
        __syncwarp();
    }
}

template <int MODE, int BN, bool TMA>
__global__ void __launch_bounds__(TMA ? 256 : 384, 1)
k_expert(const __grid_constant__ Product q)
{
    using S = Shape<BN>;
    constexpr bool A_K = MODE != kWeights, B_K = MODE == kRowsTimesTurned;
    extern __shared__ unsigned char raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t stages = smem_u32(smem);
    unsigned char* staging = smem + S::STAGES * S::STAGE;
    int32_t* first = reinterpret_cast<int32_t*>(staging + S::STAGING);
    int32_t* tile0 = first + GEM_NLR_MAX_EXPERTS + 2;
    uint64_t* bars = reinterpret_cast<uint64_t*>(staging + S::STAGING + S::TABLES);
    volatile uint32_t* dead = reinterpret_cast<uint32_t*>(bars + S::BARRIERS);
    volatile uint32_t* tmem_at = dead + 1;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int s) { return bar0 + 8u * s; };
    const auto free_ = [&](int s) { return bar0 + 8u * (S::STAGES + s); };
    const auto acc_full = [&](int a) { return bar0 + 8u * (2 * S::STAGES + a); };
    const auto acc_free = [&](int a) { return bar0 + 8u * (2 * S::STAGES + 2 + a); };
    const uint32_t drained = bar0 + 8u * (2 * S::STAGES + 4);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init(full(s), TMA ? 1 : kLoaders);
            mbar_init(free_(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(acc_full(a), 1);
            mbar_init(acc_free(a), 4);
        }
        mbar_init(drained, 1);
        *dead = 0;
        fence_barrier_init();
    }
    if (warp == 2) tmem_alloc(smem_u32((const void*)tmem_at), 2 * BN);
    if (warp == 3) make_tables<kTileM>(q, first, tile0, lane);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_at;

    const int nt = (q.n + BN - 1) / BN;
    const int tiles = (MODE == kWeights ? q.experts * ((q.m + kTileM - 1) / kTileM) : tile0[q.experts + 1]) * nt;

    if (TMA && warp == 0) {
        int s = 0;
        uint32_t parity = 1;                                  // the first round finds every stage free
        int64_t issued = 0;
        bool on = true;
        for (int t = blockIdx.x; t < tiles && on; t += gridDim.x) {
            const Tile w = tile_at<MODE, BN>(q, first, tile0, t);
            const int chunks = (w.k + kChunk - 1) / kChunk;
            int4 named = make_int4(0, 0, 0, 0);
            if (A_K && q.a.gather && chunks) named = four_rows(q.row, w.c_row + 4 * lane, w.stop, q.a.rows);
            for (int c = 0; c < chunks; ++c) {
                const int p0 = w.k_first + c * kChunk;        // weights: the chunk's first place
                if (MODE == kWeights && (q.a.gather || q.b.gather))
                    named = four_rows(q.row, p0 + 4 * (lane & 15), w.k_first + w.k, q.a.gather ? q.a.rows : q.b.rows);
                on = wait_for(free_(s), parity, dead);
                on = __all_sync(0xffffffffu, on);
                if (!on) break;
                const uint32_t a = stages + (uint32_t)s * S::STAGE, b = a + S::A, bar = full(s);
                if (lane == 0) mbar_expect_tx(bar, S::STAGE);
                __syncwarp();
                if (A_K) {
                    if (q.a.gather) load_rows(a + lane * 512, &q.ta, c * kChunk, named, bar);
                    else if (lane == 0) tma_load_2d(a, &q.ta, c * kChunk, w.c_row, bar);
                } else if (q.a.gather) {
                    load_rows(a + lane * 512, &q.ta, w.c_row + 64 * (lane >> 4), named, bar);
                } else if (lane < 2) {
                    tma_load_2d(a + lane * 8192, &q.ta, w.c_row + 64 * lane, p0, bar);
                }
                if (MODE == kRowsTimesTurned) {
                    if (lane == 0) load_3d(b, &q.tb, c * kChunk, w.n0, w.expert, bar);
                } else if (MODE == kRowsTimesPlain) {
                    if (lane < BN / 64) load_3d(b + lane * 8192, &q.tb, w.n0 + 64 * lane, c * kChunk, w.expert, bar);
                } else if (q.b.gather) {
#pragma unroll
                    for (int i = 0; i < (BN + 127) / 128; ++i) {
                        const int box = 2 * i + (lane >> 4);
                        if (box < BN / 64) load_rows(b + box * 8192 + (lane & 15) * 512, &q.tb, w.n0 + 64 * box, named, bar);
                    }
                } else if (lane < BN / 64) {
                    tma_load_2d(b + lane * 8192, &q.tb, w.n0 + 64 * lane, p0, bar);
                }
                ++issued;
                if (++s == S::STAGES) { s = 0; parity ^= 1u; }
            }
        }
        if (!on) {
            // copies on their way land before the block ends: the last round's, stage by stage
            uint32_t none = 0;
            const int64_t from = issued > S::STAGES ? issued - S::STAGES : 0;
            for (int64_t i = from; i < issued; ++i) wait_for(full((int)(i % S::STAGES)), (uint32_t)(i / S::STAGES) & 1u, &none, kSpinLimit >> 4);
        }
    } else if (warp == 1) {
        int s = 0;
        uint32_t parity = 0;
        int64_t i = 0;                                        // accumulators handed over
        bool on = true;
        for (int t = blockIdx.x; t < tiles && on; t += gridDim.x) {
            const Tile w = tile_at<MODE, BN>(q, first, tile0, t);
            if (w.k == 0) continue;
            const int chunks = (w.k + kChunk - 1) / kChunk;
            const int a = (int)(i & 1);
            on = wait_for(acc_free(a), (uint32_t)((i >> 1) + 1) & 1, dead);
            on = __all_sync(0xffffffffu, on);
            const uint32_t acc = tmem + (uint32_t)(a * BN);
            for (int c = 0; c < chunks && on; ++c) {
                on = wait_for(full(s), parity, dead);
                on = __all_sync(0xffffffffu, on);
                if (!on) break;
                tc_fence_after();
                const int left = w.k - c * kChunk;
                const uint32_t sa = stages + (uint32_t)s * S::STAGE, sb = sa + S::A;
                if (MODE == kWeights && TMA && left < kChunk) {
                    // rows of the next expert behind the last one's: zeros up to the end of the last MMA's 16
                    const int rows = ((left + 15) & ~15) - left;
                    for (int x = lane; x < rows * 8 * (2 + BN / 64); x += 32) {
                        const int r = left + (x >> 3) % rows, box = (x >> 3) / rows;
                        sts128u(sa + box * 8192 + r * kRow + (x & 7) * 16, make_uint4(0, 0, 0, 0));
                    }
                    fence_proxy_async();
                    __syncwarp();
                }
                if (lane == 0) {
                    const uint64_t da = A_K ? umma_desc_sw128(sa, 16, 1024) : umma_desc_sw128(sa, 8192, 1024);
                    const uint64_t db = B_K ? umma_desc_sw128(sb, 16, 1024) : umma_desc_sw128(sb, 8192, 1024);
                    const int steps = left >= kChunk ? 4 : (left + 15) >> 4;
                    for (int x = 0; x < steps; ++x)
                        mma(acc, da + (uint64_t)(x * (A_K ? 2 : 128)), db + (uint64_t)(x * (B_K ? 2 : 128)), q.idesc, c || x);
                    umma_commit(free_(s));
                }
                __syncwarp();
                if (++s == S::STAGES) { s = 0; parity ^= 1u; }
            }
            if (lane == 0 && on) umma_commit(acc_full(a));
            __syncwarp();
            ++i;
        }
        if (!on) {
            uint32_t none = 0;
            if (lane == 0) umma_commit(drained);
            wait_for(drained, 0, &none, kSpinLimit >> 4);
        }
    } else if (warp >= 4 && warp < 8) {
        const int quarter = warp & 3;
        const uint32_t mine = smem_u32(staging) + (uint32_t)quarter * 2048u;
        int64_t i = 0;
        bool on = true;
        for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
            const Tile w = tile_at<MODE, BN>(q, first, tile0, t);
            const int a = (int)(i & 1);
            if (w.k && on) {
                on = wait_for(acc_full(a), (uint32_t)(i >> 1) & 1, dead);
                on = __all_sync(0xffffffffu, on);
                tc_fence_after();
            }
            store_tile<MODE>(q, w, w.c_row + quarter * 32, w.n0, BN / 32, tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(a * BN), mine, lane, on);
            if (w.k) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && on) mbar_arrive(acc_free(a));
                ++i;
            }
        }
    } else if (!TMA && warp >= 8) {
        const int thread = threadIdx.x - 256;
        int s = 0;
        uint32_t parity = 1;
        bool on = true;
        for (int t = blockIdx.x; t < tiles && on; t += gridDim.x) {
            const Tile w = tile_at<MODE, BN>(q, first, tile0, t);
            const int chunks = (w.k + kChunk - 1) / kChunk;
            for (int c = 0; c < chunks; ++c) {
                on = wait_for(free_(s), parity, dead);
                if (!on) break;
                const uint32_t a = stages + (uint32_t)s * S::STAGE, b = a + S::A;
                const int p0 = w.k_first + c * kChunk, end = w.k_first + w.k;
                if (MODE == kWeights) {
                    load_ordinary<false, kTileM>(q.a, q.row, 0, p0, end, true, w.c_row, q.a.columns, a, thread);
                    load_ordinary<false, BN>(q.b, q.row, 0, p0, end, true, w.n0, q.b.columns, b, thread);
                } else {
                    load_ordinary<true, kTileM>(q.a, q.row, 0, w.c_row, w.stop, true, c * kChunk, q.a.columns, a, thread);
                    if (B_K) load_ordinary<true, BN>(q.b, q.row, w.expert, w.n0, q.b.rows, false, c * kChunk, q.b.columns, b, thread);
                    else load_ordinary<false, BN>(q.b, q.row, w.expert, (int64_t)c * kChunk, q.b.rows, false, w.n0, q.b.columns, b, thread);
                }
                fence_proxy_async();
                mbar_arrive(full(s));
                if (++s == S::STAGES) { s = 0; parity ^= 1u; }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) tmem_dealloc(tmem, 2 * BN);
}

// ---- two SMs on one tile of 256 x 256 ------------------------------------------------------------------------------------------
// A stage costs 48 KB of loads a 128 x 256 tile of one SM, and 32 KB an SM here: each SM of a pair holds 128 rows of A and 128
// columns of B, the MMA reads both SMs' shared memory, and each keeps 128 rows of accumulators.  The first SM issues the MMAs for
// both; the second's loads and epilogue signal the first's barriers.
//
//   warps 0, 2      TMA loads of A and of B, each SM its own
//   warp 1         (first SM) issues the MMAs
//   warps 4-11     epilogue: a quarter of the rows and a half of the columns each
//   warps 12-15    (GATHER) rows that are named by index, four at a time: a box cannot; one thread each
// An expert's last, cut rows where they are the K dimension are loaded by warps 0 and 2 in the same way, rows behind the last as zeros.

constexpr int kPairN = 256;
struct Pair {
    static constexpr int A = kTileM * kRow, B = kTileM * kRow, STAGE = A + B;
    static constexpr int STAGES = 6;
    static constexpr int STAGING = 8 * 2048;
    static constexpr int BARRIERS = 2 * STAGES + 5;
    static constexpr int TABLES = (2 * GEM_NLR_MAX_EXPERTS + 4) * 4;
    static constexpr int SHARED = 1024 + STAGES * STAGE + STAGING + TABLES + BARRIERS * 8 + 16;
};

// One thread of a converged warp.  What it runs alone takes its operands from uniform registers, which the MMAs and TMA copies read.
__device__ __forceinline__ bool one_thread()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "elect.sync _|p, 0xffffffff;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

__device__ __forceinline__ uint32_t pair_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The address of the first SM's copy of a shared variable.
__device__ __forceinline__ uint32_t of_first(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void pair_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t bar)              // a barrier of either SM
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives at the barrier of this address in both SMs once the MMAs issued so far are complete.
__device__ __forceinline__ void pair_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load_rows(uint32_t dst, const CUtensorMap* map, int x, int4 y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(x), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w), "r"(bar) : "memory");
}

// The rows of places p to p + 3 of an operand, in the form that a load of rows takes: for none, the one behind the last.
__device__ __forceinline__ int4 rows_at(const Operand& o, const int32_t* row, int p, int stop)
{
    if (o.gather) return four_rows(row, p, stop, o.rows);
    const int none = (int)o.rows;
    return make_int4(p < stop ? p : none, p + 1 < stop ? p + 1 : none, p + 2 < stop ? p + 2 : none, p + 3 < stop ? p + 3 : none);
}

template <int MODE, bool GATHER>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GATHER ? 512 : 384, 1)
k_expert_pair(const __grid_constant__ Product q)
{
    using S = Pair;
    constexpr bool A_K = MODE != kWeights, B_K = MODE == kRowsTimesTurned;
    extern __shared__ unsigned char raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t stages = smem_u32(smem);
    unsigned char* staging = smem + S::STAGES * S::STAGE;
    int32_t* first = reinterpret_cast<int32_t*>(staging + S::STAGING);
    int32_t* tile0 = first + GEM_NLR_MAX_EXPERTS + 2;
    uint64_t* bars = reinterpret_cast<uint64_t*>(staging + S::STAGING + S::TABLES);
    volatile uint32_t* dead = reinterpret_cast<uint32_t*>(bars + S::BARRIERS);
    volatile uint32_t* tmem_at = dead + 1;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int s) { return bar0 + 8u * s; };                               // the first SM's count
    const auto free_ = [&](int s) { return bar0 + 8u * (S::STAGES + s); };                // each SM's own
    const auto acc_full = [&](int a) { return bar0 + 8u * (2 * S::STAGES + a); };         // each SM's own
    const auto acc_free = [&](int a) { return bar0 + 8u * (2 * S::STAGES + 2 + a); };     // the first SM's count
    const uint32_t drained = bar0 + 8u * (2 * S::STAGES + 4);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)pair_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init(full(s), 1);
            mbar_init(free_(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(acc_full(a), 1);
            mbar_init(acc_free(a), 16);
        }
        mbar_init(drained, 1);
        *dead = 0;
        fence_barrier_init();
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_at)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (warp == 3) make_tables<2 * kTileM>(q, first, tile0, lane);
    tc_fence_before();
    __syncthreads();
    pair_barrier();
    tc_fence_after();
    const uint32_t tmem = *tmem_at;

    const int nt = (q.n + kPairN - 1) / kPairN;
    const int tiles = (MODE == kWeights ? q.experts * ((q.m + 2 * kTileM - 1) / (2 * kTileM)) : tile0[q.experts + 1]) * nt;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const auto tile = [&](int t) { return tile_at<MODE, kPairN, 2 * kTileM>(q, first, tile0, t); };
    if (warp == 0 || warp == 2) {
        if (one_thread()) {
            const bool left_one = warp == 0;                // A; the other warp loads B
            const Operand& o = left_one ? q.a : q.b;
            const CUtensorMap* by_index = left_one ? &q.ra : &q.rb;
            const bool others = GATHER && o.gather;         // warps 12 to 15 load it
            int s = 0;
            uint32_t parity = 1, g = 0;
            bool on = true;
            for (int t = pair; t < tiles && on; t += pairs) {
                const Tile w = tile(t);
                const int a_row = w.c_row + rank * kTileM, b_col = w.n0 + rank * kTileM;
                const int x = left_one ? a_row : b_col;     // weights: the operand's first column
                int p0 = w.k_first;                         // weights: the chunk's first place
                for (int k = 0; k < w.k; k += kChunk, p0 += kChunk) {
                    on = wait_for(free_(s), parity, dead);
                    if (!on) break;
                    const uint32_t to = stages + (uint32_t)s * S::STAGE + (left_one ? 0 : S::A), bar = of_first(full(s));
                    if (MODE == kWeights && w.k - k < kChunk) {
                        // 16 rows an MMA; what is behind those stays
                        const int quads = (w.k - k + 15) / 16 * 4, end = w.k_first + w.k;
                        if (left_one && rank == 0) mbar_expect_tx(full(s), 8 * 512 * quads);
                        if (!others)
#pragma unroll 4
                            for (int i = 0; i < quads; ++i) {
                                const int4 named = rows_at(o, q.row, p0 + 4 * i, end);
                                pair_load_rows(to + i * 512, by_index, x, named, bar);
                                pair_load_rows(to + 8192 + i * 512, by_index, x + 64, named, bar);
                            }
                    } else {
                        if (left_one && rank == 0) mbar_expect_tx(full(s), 2 * S::STAGE);
                        if (!others) {
                            if (MODE == kWeights) {
                                pair_load_2d(to, left_one ? &q.ta : &q.tb, x, p0, bar);
                                pair_load_2d(to + 8192, left_one ? &q.ta : &q.tb, x + 64, p0, bar);
                            } else if (left_one) {
                                pair_load_2d(to, &q.ta, k, a_row, bar);
                            } else if (MODE == kRowsTimesTurned) {
                                pair_load_3d(to, &q.tb, k, b_col, w.expert, bar);
                            } else {
                                pair_load_3d(to, &q.tb, b_col, k, w.expert, bar);
                                pair_load_3d(to + 8192, &q.tb, b_col + 64, k, w.expert, bar);
                            }
                        }
                    }
                    ++g;
                    if (++s == S::STAGES) { s = 0; parity ^= 1u; }
                }
            }
            if (!on && rank == 0 && left_one) {
                // copies on their way land before the block ends
                uint32_t none = 0;
                for (uint32_t i = g > S::STAGES ? g - S::STAGES : 0; i < g; ++i) wait_for(full((int)(i % S::STAGES)), i / S::STAGES & 1u, &none, kSpinLimit);
            }
        }
    } else if (warp == 1 && rank == 0) {
        if (one_thread()) {
            const uint64_t da0 = A_K ? umma_desc_sw128(stages, 16, 1024) : umma_desc_sw128(stages, 8192, 1024);
            const uint64_t db0 = B_K ? umma_desc_sw128(stages + S::A, 16, 1024) : umma_desc_sw128(stages + S::A, 8192, 1024);
            int s = 0;
            uint32_t parity = 0, i = 0;
            bool on = true;
            for (int t = pair; t < tiles && on; t += pairs) {
                const int k = tile(t).k;
                if (k == 0) continue;
                const uint32_t acc = tmem + (i & 1u) * kPairN;
                on = wait_for(acc_free(i & 1), ((i >> 1) + 1) & 1, dead);
                for (int left = k; left > 0 && on; left -= kChunk) {
                    on = wait_for(full(s), parity, dead);
                    if (!on) break;
                    tc_fence_after();
                    const uint64_t da = da0 + (uint64_t)(uint32_t)(s * (S::STAGE >> 4)), db = db0 + (uint64_t)(uint32_t)(s * (S::STAGE >> 4));
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (x == 0 || x * 16 < left)
                            pair_mma(acc, da + (uint64_t)(x * (A_K ? 2 : 128)), db + (uint64_t)(x * (B_K ? 2 : 128)), q.idesc, x || left < k);
                    pair_commit(free_(s));
                    if (++s == S::STAGES) { s = 0; parity ^= 1u; }
                }
                if (on) pair_commit(acc_full(i & 1));
                ++i;
            }
            if (!on) {
                uint32_t none = 0;
                pair_commit(drained);
                wait_for(drained, 0, &none, kSpinLimit);
            }
        }
    } else if (warp >= 4 && warp < 12) {
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t mine = smem_u32(staging) + (uint32_t)(warp - 4) * 2048u;
        uint32_t i = 0;
        bool on = true;
        for (int t = pair; t < tiles; t += pairs) {
            const Tile w = tile(t);
            if (w.k && on) {
                on = wait_for(acc_full(i & 1), (i >> 1) & 1, dead);
                on = __all_sync(0xffffffffu, on);
                tc_fence_after();
            }
            store_tile<MODE>(q, w, w.c_row + rank * kTileM + quarter * 32, w.n0 + half * 128, 4,
                             tmem + ((uint32_t)(quarter * 32) << 16) + (i & 1u) * kPairN + (uint32_t)(half * 128), mine, lane, on);
            if (w.k) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && on) arrive_at(of_first(acc_free(i & 1)));
                ++i;
            }
        }
    } else if (GATHER && warp >= 12) {
        const int part = warp - 12;
        int s = 0;
        uint32_t parity = 1;
        bool on = true;
        for (int t = pair; t < tiles && on; t += pairs) {
            const Tile w = tile(t);
            const int a_row = w.c_row + rank * kTileM, b_col = w.n0 + rank * kTileM;
            if (A_K) {
                if (one_thread()) {
                    int4 named[8];                          // a quarter of A's rows
                    if (w.k)
#pragma unroll
                        for (int i = 0; i < 8; ++i) named[i] = rows_at(q.a, q.row, a_row + 32 * part + 4 * i, w.stop);
                    for (int k = 0; k < w.k; k += kChunk) {
                        on = wait_for(free_(s), parity, dead);
                        if (!on) break;
                        const uint32_t to = stages + (uint32_t)s * S::STAGE + (uint32_t)(32 * part * kRow), bar = of_first(full(s));
#pragma unroll
                        for (int i = 0; i < 8; ++i) pair_load_rows(to + (uint32_t)(4 * i * kRow), &q.ra, k, named[i], bar);
                        if (++s == S::STAGES) { s = 0; parity ^= 1u; }
                    }
                }
                on = __all_sync(0xffffffffu, on);
            } else {
                // A quarter of a chunk's places: lane i has the i-th's row, read four chunks ahead.
                constexpr int AHEAD = 4;
                const Operand& o = q.a.gather ? q.a : q.b;
                const CUtensorMap* map = q.a.gather ? &q.ra : &q.rb;
                const int x = q.a.gather ? a_row : b_col, end = w.k_first + w.k, mine = w.k_first + 16 * part + (lane & 15);
                int ahead[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) ahead[u] = mine + u * kChunk < end ? __ldg(q.row + mine + u * kChunk) : -1;
                for (int k0 = 0; k0 < w.k && on; k0 += AHEAD * kChunk) {
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) {
                        const int k = k0 + u * kChunk;
                        if (k >= w.k || !on) break;
                        on = wait_for(free_(s), parity, dead);
                        on = __all_sync(0xffffffffu, on);
                        if (!on) break;
                        const int r = (uint32_t)ahead[u] < (uint32_t)o.rows ? ahead[u] : (int)o.rows;
                        const int next = mine + k + AHEAD * kChunk;
                        ahead[u] = next < end ? __ldg(q.row + next) : -1;
                        int4 named[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            named[i] = make_int4(__shfl_sync(0xffffffffu, r, 4 * i), __shfl_sync(0xffffffffu, r, 4 * i + 1), __shfl_sync(0xffffffffu, r, 4 * i + 2),
                                                 __shfl_sync(0xffffffffu, r, 4 * i + 3));
                        if (one_thread() && 16 * part < w.k - k) {          // (a cut chunk has only the rows that an MMA takes)
                            const uint32_t to = stages + (uint32_t)s * S::STAGE + (q.a.gather ? 0 : S::A) + (uint32_t)(16 * part * kRow), bar = of_first(full(s));
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                pair_load_rows(to + (uint32_t)(i * 512), map, x, named[i], bar);
                                pair_load_rows(to + (uint32_t)(8192 + i * 512), map, x + 64, named[i], bar);
                            }
                        }
                        __syncwarp();
                        if (++s == S::STAGES) { s = 0; parity ^= 1u; }
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    pair_barrier();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

PFN_cuTensorMapEncodeTiled_v12000 encoder()
{
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult got;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &got) != cudaSuccess || got != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (PFN_cuTensorMapEncodeTiled_v12000)f;
    }();
    return fn;
}

// Boxes of box_rows rows of 128 bytes, 128-byte swizzle, zeros outside.
bool encode(CUtensorMap* map, const Operand& o, int experts, int box_rows, bool bf16)
{
    const auto fn = encoder();
    if (!fn) return false;
    const bool three = experts > 0;
    const cuuint64_t dims[3] = {(cuuint64_t)o.columns, (cuuint64_t)o.rows, (cuuint64_t)(three ? experts : 1)};
    const cuuint64_t strides[2] = {(cuuint64_t)(o.ld * 2), (cuuint64_t)(o.stride * 2)};
    const cuuint32_t box[3] = {kChunk, (cuuint32_t)box_rows, 1}, unit[3] = {1, 1, 1};
    return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, three ? 3 : 2, const_cast<uint16_t*>(o.p), dims, strides, box, unit,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, int BN, bool TMA>
int launch(const Product& q, int64_t tiles, cudaStream_t st)
{
    constexpr auto kern = k_expert<MODE, BN, TMA>;
    static_assert(Shape<BN>::SHARED <= 232448, "shared memory of a block");
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<BN>::SHARED) != cudaSuccess) {
        cudaGetLastError();
        return GEM_NLR_E_CUDA;
    }
    kern<<<(unsigned)(tiles < kTrainSMs ? tiles : kTrainSMs), TMA ? 256 : 384, Shape<BN>::SHARED, st>>>(q);
    return launched();
}

template <int MODE, int BN>
int prepare(Product& q, int64_t tiles, bool bf16, cudaStream_t st)
{
    constexpr bool A_K = MODE != kWeights, B_K = MODE == kRowsTimesTurned;
    if (q.a.wide && q.b.wide && encode(&q.ta, q.a, 0, q.a.gather ? 1 : A_K ? kTileM : kChunk, bf16) &&
        encode(&q.tb, q.b, MODE == kWeights ? 0 : q.experts, q.b.gather ? 1 : B_K ? BN : kChunk, bf16))
        return launch<MODE, BN, true>(q, tiles, st);
    return launch<MODE, BN, false>(q, tiles, st);
}

template <int MODE, bool GATHER>
int launch_pair(const Product& q, int64_t tiles, cudaStream_t st)
{
    constexpr auto kern = k_expert_pair<MODE, GATHER>;
    static_assert(Pair::SHARED <= 232448, "shared memory of a block");
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Pair::SHARED) != cudaSuccess) {
        cudaGetLastError();
        return GEM_NLR_E_CUDA;
    }
    kern<<<2 * (unsigned)(tiles < kTrainSMs / 2 ? tiles : kTrainSMs / 2), GATHER ? 512 : 384, Pair::SHARED, st>>>(q);
    return launched();
}

// The widest tile that gives every SM one: a narrower one reads its rows (or the left operand) more often.
template <int MODE>
int run(Product& q, bool bf16, cudaStream_t st)
{
    // row tiles there can be: an expert's last one may be almost empty, and places without an expert have one more
    const int64_t row_tiles = MODE == kWeights ? (int64_t)q.experts * ((q.m + kTileM - 1) / kTileM)
                                               : q.places / kTileM + (q.places < q.experts + 1 ? q.places : q.experts + 1);
    const auto tiles = [&](int bn) { return row_tiles * ((q.n + bn - 1) / bn); };
    const auto idesc = [&](int bn) {
        return umma_idesc_f16(kTileM, bn, MODE == kWeights, MODE != kRowsTimesTurned) | (bf16 ? 1u << 7 | 1u << 10 : 0u);
    };
    const int64_t tall_tiles = (MODE == kWeights ? (int64_t)q.experts * ((q.m + 255) / 256) : q.places / 256 + (q.places < q.experts + 1 ? q.places : q.experts + 1)) *
                               ((q.n + kPairN - 1) / kPairN);
    if (q.a.wide && q.b.wide && (MODE == kWeights ? q.m : q.places / q.experts) >= 256 && tall_tiles >= kTrainSMs / 2) {
        constexpr bool A_K = MODE != kWeights, B_K = MODE == kRowsTimesTurned;
        q.idesc = idesc(256) & ~(31u << 24) | (uint32_t)(2 * kTileM >> 4) << 24;
        const bool cut = MODE == kWeights;                          // rows of both operands by index
        if ((q.a.gather || encode(&q.ta, q.a, 0, A_K ? kTileM : kChunk, bf16)) &&
            (q.b.gather || encode(&q.tb, q.b, MODE == kWeights ? 0 : q.experts, B_K ? kTileM : kChunk, bf16)) &&
            (!(cut || q.a.gather) || encode(&q.ra, q.a, 0, 1, bf16)) && (!cut || encode(&q.rb, q.b, 0, 1, bf16)))
            return q.a.gather || q.b.gather ? launch_pair<MODE, true>(q, tall_tiles, st) : launch_pair<MODE, false>(q, tall_tiles, st);
    }
    if (tiles(256) >= kTrainSMs) {
        q.idesc = idesc(256);
        return prepare<MODE, 256>(q, tiles(256), bf16, st);
    }
    if (tiles(128) >= kTrainSMs) {
        q.idesc = idesc(128);
        return prepare<MODE, 128>(q, tiles(128), bf16, st);
    }
    q.idesc = idesc(64);
    return prepare<MODE, 64>(q, tiles(64), bf16, st);
}

bool on_16(const void* p, int64_t ld) { return aligned_to(p, 16) && ld % 8 == 0; }

Operand places_of(const void* p, int64_t ld, int64_t rows, int columns, bool gather)
{
    return {(const uint16_t*)p, ld, 0, rows, columns, gather, on_16(p, ld) && ld > 0};
}

Operand weights_of(const void* p, int64_t ld, int64_t stride, int experts, int rows, int columns)
{
    if (experts == 1) stride = rows * ld;
    return {(const uint16_t*)p, ld, stride, rows, columns, 0, on_16(p, ld) && ld > 0 && stride % 8 == 0 && stride > 0};
}

constexpr int64_t kMaxPlaces = INT32_MAX - (1 << 16);            // int arithmetic on places, tiles included, stays far from its end
bool half_type(int32_t type) { return type == GEM_NLR_F16 || type == GEM_NLR_BF16; }
bool halves(const void* p) { return p && aligned_to(p, 2); }
bool sizes_fine(int32_t type, int64_t x_rows, int64_t places, int32_t experts, int32_t d_in, int32_t d_out, int32_t turned, const int32_t* row)
{
    return half_type(type) && x_rows >= 0 && x_rows <= INT32_MAX && places >= 0 && places <= kMaxPlaces && experts >= 1 && experts <= GEM_NLR_MAX_EXPERTS && d_in >= 1 &&
           d_in <= kMaxColumns && d_out >= 1 && d_out <= kMaxColumns && (turned == 0 || turned == 1) && aligned_to(row, 4) && (row || x_rows >= places);
}

}  // namespace
}  // namespace gemnlr

using namespace gemnlr;

extern "C" int gem_nlr_expert_product(const void* x_dev, int32_t type, int64_t ld_x, int64_t x_rows, const void* w_dev, int64_t ld_w, int64_t stride_w,
                                      int32_t w_turned, const int32_t* offset_dev, const int32_t* row_dev, int64_t places, int32_t experts, int32_t d_in,
                                      int32_t d_out, void* y_dev, int64_t ld_y, void* cuda_stream)
{
    if (!sizes_fine(type, x_rows, places, experts, d_in, d_out, w_turned, row_dev) || ld_x < 0 || ld_w < 0 || stride_w < 0) return GEM_NLR_E_INVALID;
    if (places == 0) return GEM_NLR_OK;
    if ((x_rows > 0 && !halves(x_dev)) || !halves(w_dev) || !offset_dev || !aligned_to(offset_dev, 4) || !halves(y_dev) || ld_y < d_out || y_dev == x_dev || y_dev == w_dev)
        return GEM_NLR_E_INVALID;
    Product q = {};
    q.a = places_of(x_dev, ld_x, x_rows, d_in, row_dev != nullptr);
    if (x_rows == 0) q.a.wide = 0;
    q.b = weights_of(w_dev, ld_w, stride_w, experts, w_turned ? d_out : d_in, w_turned ? d_in : d_out);
    q.offset = offset_dev;
    q.row = row_dev;
    q.places = places;
    q.experts = experts;
    q.n = d_out;
    q.k = d_in;
    q.c = (uint16_t*)y_dev;
    q.ldc = ld_y;
    q.c_wide = on_16(y_dev, ld_y);
    q.bf16 = type == GEM_NLR_BF16;
    return w_turned ? run<kRowsTimesTurned>(q, q.bf16, (cudaStream_t)cuda_stream) : run<kRowsTimesPlain>(q, q.bf16, (cudaStream_t)cuda_stream);
}

extern "C" int gem_nlr_expert_product_backward(const void* dy_dev, int64_t ld_dy, const void* x_dev, int32_t type, int64_t ld_x, int64_t x_rows, const void* w_dev,
                                               int64_t ld_w, int64_t stride_w, int32_t w_turned, const int32_t* offset_dev, const int32_t* row_dev,
                                               int64_t places, int32_t experts, int32_t d_in, int32_t d_out, void* dx_dev, int64_t ld_dx, void* dw_dev,
                                               int64_t ld_dw, int64_t stride_dw, void* cuda_stream)
{
    const int64_t wide = w_turned ? d_in : d_out, tall = w_turned ? d_out : d_in;
    if (!sizes_fine(type, x_rows, places, experts, d_in, d_out, w_turned, row_dev) || ld_dy < 0 || (!dx_dev && !dw_dev)) return GEM_NLR_E_INVALID;
    if (places > 0 && (!halves(dy_dev) || !offset_dev || !aligned_to(offset_dev, 4))) return GEM_NLR_E_INVALID;
    if (dx_dev && places > 0 && (!halves(dx_dev) || ld_dx < d_in || !halves(w_dev) || ld_w < 0 || stride_w < 0 || dx_dev == dy_dev || dx_dev == w_dev)) return GEM_NLR_E_INVALID;
    if (dw_dev && (!halves(dw_dev) || ld_dw < wide || (experts > 1 && stride_dw < tall * ld_dw) || (places > 0 && (ld_x < 0 || (x_rows > 0 && !halves(x_dev)))) ||
                   dw_dev == dy_dev || dw_dev == x_dev || dw_dev == dx_dev))
        return GEM_NLR_E_INVALID;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    Product q = {};
    q.offset = offset_dev;
    q.row = row_dev;
    q.places = places;
    q.experts = experts;
    q.bf16 = type == GEM_NLR_BF16;
    const Operand dy = places_of(dy_dev, ld_dy, places, d_out, false);
    if (dx_dev && places > 0) {
        q.a = dy;
        q.b = weights_of(w_dev, ld_w, stride_w, experts, w_turned ? d_out : d_in, w_turned ? d_in : d_out);
        q.n = d_in;
        q.k = d_out;
        q.c = (uint16_t*)dx_dev;
        q.ldc = ld_dx;
        q.c_wide = on_16(dx_dev, ld_dx);
        const int rc = w_turned ? run<kRowsTimesPlain>(q, q.bf16, st) : run<kRowsTimesTurned>(q, q.bf16, st);
        if (rc != GEM_NLR_OK) return rc;
    }
    if (!dw_dev) return GEM_NLR_OK;
    if (places == 0) {
        for (int e = 0; e < experts; ++e)
            if (cudaMemset2DAsync((uint16_t*)dw_dev + e * stride_dw, (size_t)ld_dw * 2, 0, (size_t)wide * 2, tall, st) != cudaSuccess) {
                cudaGetLastError();
                return GEM_NLR_E_CUDA;
            }
        return GEM_NLR_OK;
    }
    const Operand x = [&] {
        Operand o = places_of(x_dev, ld_x, x_rows, d_in, row_dev != nullptr);
        if (x_rows == 0) o.wide = 0;
        return o;
    }();
    q.a = w_turned ? dy : x;
    q.b = w_turned ? x : dy;
    q.m = (int)tall;
    q.n = (int)wide;
    q.k = 0;
    q.c = (uint16_t*)dw_dev;
    q.ldc = ld_dw;
    q.stride_c = stride_dw;
    q.c_wide = on_16(dw_dev, ld_dw) && stride_dw % 8 == 0;
    return run<kWeights>(q, q.bf16, st);
}
