// Runs a translated CUDA kernel on the host, one cluster at a time: a fiber a thread, scheduled at random; copies and
// messages land at random times after they were sent.  What a GPU would fault on, hang on or leave undefined is recorded:
// copies that read outside the given regions, misaligned accesses, an arrival too many at a barrier, a block that ends with
// a copy in flight.  A wait without an end aborts the process (a missing arrival shows as no runnable fiber).
#pragma once
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <functional>
#include <map>
#include <tuple>
#include <type_traits>
#include <vector>

#undef __launch_bounds__
#undef __shared__
#undef __device__
#undef __global__
#undef __host__
#undef __forceinline__
#define __launch_bounds__(...)
#define __device__
#define __global__
#define __host__
#define __forceinline__ inline

namespace emu {

constexpr uint32_t kArena = 1 << 20;             // a block's shared memory, with room between the objects
constexpr size_t   kStack = 96 << 10;

struct Copy {                                    // on its way: 0 a thread's, 1 a bulk copy, 2 a message
    int kind;
    const void* from;                            // nullptr: zeros
    unsigned char* to;
    uint32_t bytes;
    int block;                                   // whose barrier it arrives at
    uint32_t bar, value;
    int fiber, group;
};
struct Barrier { uint32_t count = 0, pending = 0, phase = 0; int64_t bytes = 0; };
struct Meeting { uint32_t turn = 0; int here = 0; };
struct Warp { uint32_t turn = 0; int here = 0; uint64_t slot[2][32]; };
struct Block { std::vector<unsigned char> mem; std::map<uint32_t, Barrier> bars; std::vector<Warp> warps; Meeting named[17]; };
struct Fiber { ucontext_t ctx; dim3 tid; int block, lin, group; bool done; std::function<bool()> ready; };
struct Grid {
    std::vector<Block> blocks;
    std::vector<Fiber> fibers;
    std::vector<Copy> on_their_way;
    std::map<int, uint32_t> places;              // of the shared objects, the same in every block
    uint32_t top = 1024;
    int dynamic = 0, first_block = 0, cluster = 1, threads = 0;
    Meeting meeting;
    dim3 dim;
    ucontext_t main;
};

extern Grid* grid;
extern Fiber* self;
extern int resident;                             // clusters that a launch may have at most
extern int lost, lost_message;                   // number of the bulk copy, the message, that never lands; 0: none
extern uint64_t state;
extern char report[200];
extern std::vector<std::pair<const char*, size_t>> regions;

inline uint32_t random32() { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return (uint32_t)(state >> 11); }
inline void wrong(const char* what)
{
    if (!report[0]) snprintf(report, sizeof(report), "%s (block %d of the cluster, thread %d)", what, self ? self->block : -1, self ? self->lin : -1);
}
inline void pause() { swapcontext(&self->ctx, &grid->main); }
template <typename F> void until(F f) { if (!f()) { self->ready = f; pause(); self->ready = nullptr; } }
inline Block& block() { return grid->blocks[self->block]; }
inline unsigned char* arena(int b) { return grid->blocks[b].mem.data(); }
inline int dynamic_bytes() { return grid->dynamic; }
inline void* shared(int id, size_t bytes)
{
    auto it = grid->places.find(id);
    if (it == grid->places.end()) {
        grid->top = (grid->top + 127) / 128 * 128;
        it = grid->places.emplace(id, grid->top).first;
        grid->top += (uint32_t)bytes + 64;
        if (grid->top > kArena) abort();
    }
    return arena(self->block) + it->second;
}
// addresses in shared memory: a byte's place in the arena; with the top bit, of block (bits 24 on) of the cluster
inline uint32_t place(const void* p) { return (uint32_t)((const unsigned char*)p - arena(self->block)); }
inline unsigned char* at(uint32_t a, int& b)
{
    b = a & 0x80000000u ? (int)(a >> 24 & 15) : self->block;
    if ((a & 0xffffff) >= kArena || b >= (int)grid->blocks.size()) { wrong("an address outside shared memory"); return arena(self->block); }
    return arena(b) + (a & 0xffffff);
}
inline unsigned char* at(uint32_t a) { int b; return at(a, b); }
inline void readable(const void* p, size_t n)
{
    for (auto& r : regions)
        if ((const char*)p >= r.first && (const char*)p + n <= r.first + r.second) return;
    wrong("a copy that reads outside its matrix");
}
inline void settle(Barrier& b)
{
    if (b.pending == 0 && b.bytes == 0) { b.phase ^= 1; b.pending = b.count; }
}
inline void land(size_t i)
{
    const Copy c = grid->on_their_way[i];
    grid->on_their_way[i] = grid->on_their_way.back();
    grid->on_their_way.pop_back();
    if (c.kind == 2) memcpy(c.to, &c.value, 4);
    else if (c.from) memcpy(c.to, c.from, c.bytes);
    else memset(c.to, 0, c.bytes);
    if (c.kind) { Barrier& b = grid->blocks[c.block].bars[c.bar]; b.bytes -= c.bytes; settle(b); }
}
inline void meet(Meeting& m, int count)
{
    const uint32_t turn = m.turn;
    Meeting* p = &m;
    if (++m.here == count) { m.here = 0; ++m.turn; } else until([p, turn] { return p->turn != turn; });
}
inline void sync_threads() { meet(block().named[0], grid->threads); }
template <typename T> T shuffle_xor(T v, int o)
{
    Warp& w = block().warps[self->lin / 32];
    Warp* p = &w;
    const int l = self->lin & 31;
    const uint32_t turn = w.turn;
    memcpy(&w.slot[turn & 1][l], &v, sizeof(T));
    if (++w.here == 32) { w.here = 0; ++w.turn; } else until([p, turn] { return p->turn != turn; });
    T r;
    memcpy(&r, &w.slot[turn & 1][l ^ o], sizeof(T));
    return r;
}

// ---- instructions
inline void op_cluster_rank(uint32_t& r) { r = (uint32_t)self->block; }
inline void op_cluster_barrier() { meet(grid->meeting, grid->cluster * grid->threads); }
inline void op_bar_sync(int id, int n) { meet(block().named[id], n); }
inline void op_fence_mbarrier_init_release_cluster() {}
inline void op_griddepcontrol_launch_dependents() {}
inline void op_griddepcontrol_wait() {}
inline void op_createpolicy_fractional_L2__evict_first_b64(uint64_t& p) { p = 0; }
inline void op_ex2_approx_ftz_f32(float& y, float x) { y = exp2f(x); if (fabsf(y) < 1.17549435e-38f) y = 0.0f; }
inline void op_cp_async_cg_shared_global(uint32_t to, const void* from)
{
    readable(from, 16);
    if (((uintptr_t)from | to) & 15) wrong("a copy of 16 bytes off 16 bytes");
    grid->on_their_way.push_back({0, from, at(to), 16, 0, 0, 0, self->lin + self->block * grid->threads, self->group});
}
inline void op_cp_async_ca_shared_global(uint32_t to, const void* from, int n)
{
    if (n) readable(from, 4);
    grid->on_their_way.push_back({0, n ? from : nullptr, at(to), 4, 0, 0, 0, self->lin + self->block * grid->threads, self->group});
}
inline void op_cp_async_commit_group() { ++self->group; }
inline void op_cp_async_wait_group(int left)
{
    const int me = self->lin + self->block * grid->threads;
    auto& on = grid->on_their_way;
    for (size_t i = 0; i < on.size();)
        if (on[i].kind == 0 && on[i].fiber == me && on[i].group < self->group - left) land(i); else ++i;
}
inline void op_ld_shared_b32(uint32_t& v, uint32_t a) { memcpy(&v, at(a), 4); }
inline void op_ld_shared_v4_b32(uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d, uint32_t from)
{
    if (from & 15) wrong("a load of 16 bytes off 16 bytes");
    uint32_t w[4];
    memcpy(w, at(from), 16);
    a = w[0]; b = w[1]; c = w[2]; d = w[3];
}
inline void op_st_shared_v4_b32(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    if (to & 15) wrong("a store of 16 bytes off 16 bytes");
    const uint32_t w[4] = {a, b, c, d};
    memcpy(at(to), w, 16);
}
inline void op_st_shared_v4_b32(uint32_t to, uint32_t a) { op_st_shared_v4_b32(to, a, a, a, a); }
inline void op_cp_async_bulk_shared__cluster_global_mbarrier__complete_tx__bytes(uint32_t to, const void* from, uint32_t bytes, uint32_t bar)
{
    readable(from, bytes);
    if ((((uintptr_t)from | to | bytes) & 15) || bytes == 0) wrong("a bulk copy off 16 bytes");
    if (lost > 0 && --lost == 0) return;
    grid->on_their_way.push_back({1, from, at(to), bytes, self->block, bar, 0, -1, 0});
}
inline void op_cp_async_bulk_shared__cluster_global_mbarrier__complete_tx__bytes_L2__cache_hint(uint32_t to, const void* from, uint32_t bytes,
                                                                                                uint32_t bar, uint64_t)
{
    op_cp_async_bulk_shared__cluster_global_mbarrier__complete_tx__bytes(to, from, bytes, bar);
}
inline void op_mbarrier_init_shared__cta_b64(uint32_t bar, uint32_t n) { Barrier b; b.count = b.pending = n; block().bars[bar] = b; }
inline void op_mbarrier_arrive_expect_tx_shared__cta_b64(uint32_t bar, uint32_t bytes)
{
    Barrier& b = block().bars[bar];
    if (b.pending == 0) { wrong("an arrival too many at a barrier"); return; }
    b.bytes += bytes;
    --b.pending;
    settle(b);
}
inline void op_try_wait(uint32_t& ok, uint32_t bar, uint32_t parity)
{
    if (parity > 1) wrong("a parity that is none");
    ok = (block().bars[bar].phase & 1) != (parity & 1);
    if (!ok) {
        self->ready = [] { return true; };
        pause();
        self->ready = nullptr;
        ok = (block().bars[bar].phase & 1) != (parity & 1);
    }
}
inline void op_mapa_shared__cluster_u32(uint32_t& d, uint32_t a, int r) { d = 0x80000000u | (uint32_t)r << 24 | (a & 0xffffff); }
inline void op_st_async_shared__cluster_mbarrier__complete_tx__bytes_b32(uint32_t to, uint32_t v, uint32_t bar)
{
    int b;
    unsigned char* p = at(to, b);
    if (lost_message > 0 && --lost_message == 0) return;
    grid->on_their_way.push_back({2, nullptr, p, 4, b, bar & 0xffffff, v, -1, 0});
}
inline void op_ld_shared__cluster_f64(double& v, uint32_t a) { memcpy(&v, at(a), 8); }
inline void op_ld_shared__cluster_f32(float& v, uint32_t a) { memcpy(&v, at(a), 4); }

// ---- launches
extern std::function<void()> body;
inline void enter() { body(); self->done = true; }

inline void run(dim3 dim, int threads, int cluster, int dynamic, std::function<void()> f)
{
    static std::vector<std::vector<char>> stacks;
    const int blocks = (int)(dim.x * dim.y);
    if (blocks % cluster) { wrong("a grid that is no multiple of its clusters"); return; }
    Grid g;
    grid = &g;
    body = f;
    g.dim = dim;
    g.cluster = cluster;
    g.threads = threads;
    g.dynamic = dynamic;
    g.blocks.resize(cluster);
    for (auto& b : g.blocks) b.mem.resize(kArena);
    g.fibers.resize((size_t)cluster * threads);
    while (stacks.size() < g.fibers.size()) stacks.emplace_back(kStack);
    for (g.first_block = 0; g.first_block < blocks; g.first_block += cluster) {
        g.on_their_way.clear();
        g.meeting = Meeting();
        for (auto& b : g.blocks) {
            b.bars.clear();
            b.warps.assign(threads / 32, Warp());
            for (auto& m : b.named) m = Meeting();
            memset(b.mem.data(), random32() & 1 ? 0xff : 0xa5, kArena);           // nothing may hang on what it held
        }
        std::vector<int> live(g.fibers.size());
        for (size_t i = 0; i < g.fibers.size(); ++i) {
            Fiber& t = g.fibers[i];
            t.block = (int)i / threads;
            t.lin = (int)i % threads;
            t.tid = dim3(t.lin, 0, 0);
            t.group = 0;
            t.done = false;
            t.ready = nullptr;
            getcontext(&t.ctx);
            t.ctx.uc_stack.ss_sp = stacks[i].data();
            t.ctx.uc_stack.ss_size = kStack;
            t.ctx.uc_link = &g.main;
            makecontext(&t.ctx, enter, 0);
            live[i] = (int)i;
        }
        const uint32_t style = random32() % 3;                                     // in turn; at random; at random with slow copies
        size_t turn = 0, idle = 0;
        while (!live.empty()) {
            auto& on = g.on_their_way;
            const uint32_t chance = random32() % 64;
            if (!on.empty() && chance < (style == 2 ? 1u : 8u)) {
                const size_t i = random32() % on.size();
                if (on[i].kind || chance == 0) land(i);
            }
            const size_t l = style == 0 ? turn++ % live.size() : random32() % live.size();
            Fiber& t = g.fibers[live[l]];
            if (t.ready && !t.ready()) {
                if (++idle > 200000 + 50 * live.size()) {
                    idle = 0;
                    if (!on.empty()) land(0);
                    else if (std::none_of(live.begin(), live.end(), [&](int k) { return !g.fibers[k].ready || g.fibers[k].ready(); })) {
                        fprintf(stderr, "emulation: no thread can go on\n");
                        abort();
                    }
                }
                continue;
            }
            idle = 0;
            self = &t;
            swapcontext(&g.main, &t.ctx);
            self = nullptr;
            if (t.done) { live[l] = live.back(); live.pop_back(); }
        }
        for (auto& c : g.on_their_way)
            if (c.kind == 1) { wrong("a block that ends with a copy in flight"); break; }
    }
    grid = nullptr;
}
template <typename... P, typename... A>
cudaError_t launch_rows(void (*k)(P...), int blocks, int cluster, int bytes, bool, cudaStream_t, const A&... args)
{
    std::tuple<P...> t((P)args...);
    run(dim3(blocks), 256, cluster, bytes, [&] { std::apply(k, t); });
    return cudaSuccess;
}
template <typename... P, typename... A>
cudaError_t launch_early(void (*k)(P...), dim3 dim, int threads, cudaStream_t, const A&... args)
{
    std::tuple<P...> t((P)args...);
    run(dim, threads, 1, 0, [&] { std::apply(k, t); });
    return cudaSuccess;
}
template <typename... P, typename... A> void launch_plain(void (*k)(P...), dim3 dim, int threads, const A&... args)
{
    launch_early(k, dim, threads, (cudaStream_t)0, args...);
}

}  // namespace emu

// ---- what the kernels call
static inline uint32_t emu_bits(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
static inline float emu_float(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
static inline float2 emu_add2(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
static inline float2 emu_mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
static inline float2 emu_fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
static inline unsigned atomicAdd(unsigned* p, unsigned v) { const unsigned o = *p; *p += v; return o; }
template <typename T2> static inline T2 emu_max2(T2 a, T2 b)          // a NaN is passed over
{
    const float ax = (float)a.x, ay = (float)a.y, bx = (float)b.x, by = (float)b.y;
    T2 r;
    r.x = ax != ax ? b.x : bx != bx ? a.x : ax > bx ? a.x : b.x;
    r.y = ay != ay ? b.y : by != by ? a.y : ay > by ? a.y : b.y;
    return r;
}
using std::max;
using std::min;
#define threadIdx (emu::self->tid)
#define blockIdx (dim3((emu::grid->first_block + emu::self->block) % emu::grid->dim.x, (emu::grid->first_block + emu::self->block) / emu::grid->dim.x))
#define gridDim (emu::grid->dim)
#define __syncthreads() emu::sync_threads()
#define __syncwarp() emu::shuffle_xor(0, 0)
#define __shfl_xor_sync(mask, v, o) emu::shuffle_xor(v, o)
#define __cvta_generic_to_shared(p) emu::place(p)
#define __threadfence()
#define __float_as_uint emu_bits
#define __uint_as_float emu_float
#define __int_as_float emu_float
#define __fadd2_rn emu_add2
#define __fmul2_rn emu_mul2
#define __ffma2_rn emu_fma2
#define __hmax2 emu_max2
#define __fdividef(a, b) ((a) / (b))
#define __stcs(p, v) (*(p) = (v))
#define rsqrtf(x) (1.0f / sqrtf(x))
#define cudaGetLastError() cudaSuccess
