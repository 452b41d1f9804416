// Block tables and slot maps of the 8-bit cache from the units' lengths.
//
// With n tokens and a new ones, unit u needs ceil((n + a) / p) - ceil(n / p)
// pages; page i of the ones it gets is ring[(head + before_u + i) mod pages],
// before_u the sum of the needs of the units before it.  One launch: every
// block sums the needs of all units (8 bytes each, out of L2) for the total,
// which decides whether anything is given, and for its own first unit's
// before, scans its own units, and writes what belongs to them.  That costs
// less than a second launch as long as the units' lengths are a few hundred
// kilobytes, and needs no scratch and no atomics: the ring is handed out in
// the units' order whatever the blocks' timing.  A step of 448 units takes 4.9
// us, 4.2M slots of 16384 units 18 (half of it the slots, the rest the sums and
// the scan, all bound by instructions and latencies); a call costs about as
// much on the host.
#include "bacon.h"
#include "cache.h"
#include "common.cuh"

namespace bacon {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanUnits = 1024;  // own units of a block, at most

__device__ __forceinline__ long long warp_sum(long long x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

struct PlanGeom {
    int layers, hkv, page_log2, pages, max_blocks;
};

// (a unit has fewer than 2^31 - 1024 tokens)
__device__ __forceinline__ int blocks_of(int tokens, int page_log2)
{
    return (tokens + (1 << page_log2) - 1) >> page_log2;
}

// x mod pages for x < 2 pages
__device__ __forceinline__ int wrapped(unsigned x, int pages)
{
    return (int)(x < (unsigned)pages ? x : x - pages);
}

__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(PlanGeom g, PlanArgs a, int own, int* err)
{
    __shared__ int s_n[kPlanUnits], s_a[kPlanUnits], s_page[kPlanUnits], s_row[kPlanUnits];
    __shared__ long long s_sum[32][4];
    __shared__ int s_bad;
    __shared__ unsigned long long s_scan[32];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lh = g.layers * g.hkv;
    const int u0 = blockIdx.x * own, u1 = min(a.units, u0 + own), r0 = u0 / lh;
    const int most = g.max_blocks << g.page_log2;
    const bool alloc = a.ring != nullptr;
    if (tid == 0) s_bad = 0;
    __syncthreads();

    // all units: pages wanted in total and before this block's units, tokens
    // in total and before
    long long sum[4] = {0, 0, 0, 0};
    bool bad = false;
#pragma unroll 8
    for (int u = tid; u < a.units; u += kPlanThreads) {
        const int n = a.lengths ? a.lengths[u] : 0;
        const int m = a.per_unit ? a.added[u] : a.added ? a.added[u / lh] : 1;
        const bool fine = n >= 0 && n <= most && m >= 0 && m <= most - n;
        const int need = fine ? blocks_of(n + m, g.page_log2) - blocks_of(n, g.page_log2) : 0;
        const int tokens = fine && a.per_unit ? m : 0;
        bad |= !fine;
        sum[0] += need;
        sum[1] += u < u0 ? need : 0;
        sum[2] += tokens;
        sum[3] += u < u0 ? tokens : 0;
    }
    if (!a.per_unit)
        for (int r = tid; r < a.requests; r += kPlanThreads) {
            const int m = a.added ? a.added[r] : 1;
            sum[2] += m;
            if (r < r0) sum[3] += m;
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum[i] = warp_sum(sum[i]);
        if (lane == 0) s_sum[warp][i] = sum[i];
    }
    if (bad) s_bad = 1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = warp_sum(s_sum[lane][i]);
    const int head = alloc ? a.state[0] : 0, count = alloc ? a.state[1] : 0;
    bad = s_bad != 0 || sum[2] > a.rows || head < 0 || head >= g.pages || count < 0 ||
          count > g.pages;
    const bool poor = alloc && !bad && sum[0] > count;
    const bool given = !bad && !poor;
    if (!given && blockIdx.x == 0 && tid == 0) atomicCAS(err, 0, poor ? kCacheNoPages : kCacheBadIndex);

    // own units: where their pages and tokens start
    int n = 0, m = 0, need = 0;
    if (u0 + tid < u1) {
        n = a.lengths ? a.lengths[u0 + tid] : 0;
        if (given) {
            m = a.per_unit ? a.added[u0 + tid] : a.added ? a.added[(u0 + tid) / lh] : 1;
            need = blocks_of(n + m, g.page_log2) - blocks_of(n, g.page_log2);
        }
        if (a.lengths_out) a.lengths_out[u0 + tid] = n + m;
    }
    // pages in the upper, tokens in the lower half: neither sum passes 2^31
    const unsigned long long mine = (unsigned long long)(uint32_t)need << 32 | (uint32_t)m;
    unsigned long long x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) s_scan[warp] = x;
    __syncthreads();
    unsigned long long before = lane < warp ? s_scan[lane] : 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
    x += before - mine;
    if (tid < own && u0 + tid < u1) {
        s_n[tid] = n;
        s_a[tid] = m;
        s_page[tid] = wrapped(wrapped((unsigned)head + (unsigned)sum[1], g.pages) + (unsigned)(x >> 32), g.pages);
        int row = (int)sum[3];
        if (a.per_unit) {
            row += (int)(uint32_t)x;
        } else if (given) {
            for (int r = r0; r < (u0 + tid) / lh; ++r) row += a.added ? a.added[r] : 1;
        }
        s_row[tid] = row;
    }
    if (alloc && blockIdx.x == 0 && tid == 0) {
        a.state_out[0] = given ? wrapped((unsigned)head + (unsigned)sum[0], g.pages) : head;
        a.state_out[1] = given ? (int)(count - sum[0]) : count;
    }
    __syncthreads();

    // a warp per unit
    if (given) {
        bool wrong = false;
        for (int i = warp; i < u1 - u0; i += kPlanThreads / 32) {
            const int u = u0 + i, n0 = s_n[i], add = s_a[i], row = s_row[i], first = s_page[i];
            const int have = blocks_of(n0, g.page_log2);
            const int gets = alloc ? blocks_of(n0 + add, g.page_log2) - have : 0;
            int32_t* const entry = a.table + (size_t)u * g.max_blocks;
            for (int b = lane; b < gets; b += 32) entry[have + b] = a.ring[wrapped((unsigned)first + b, g.pages)];
            int32_t* const to = a.per_unit
                                    ? a.slots + row
                                    : a.slots + ((size_t)(u / g.hkv % g.layers) * a.rows + row) * g.hkv + u % g.hkv;
            const int step = a.per_unit ? 1 : g.hkv;
#pragma unroll 4
            for (int j = lane; j < add; j += 32) {
                const int pos = n0 + j, b = pos >> g.page_log2;
                const int page = alloc && b >= have ? a.ring[wrapped((unsigned)first + (b - have), g.pages)]
                                                    : entry[b];
                const bool fine = page >= 0 && page < g.pages;
                wrong |= !fine;
                to[(size_t)j * step] =
                    fine ? (page << g.page_log2) + (pos & ((1 << g.page_log2) - 1)) : -1;
            }
        }
        if (wrong) atomicCAS(err, 0, kCacheBadIndex);
    }
    // entries beyond the last token
    const int used = given ? (int)sum[2] : 0;
    const long long rest = (long long)(a.rows - used) * (a.per_unit ? 1 : lh);
    for (long long i = (long long)blockIdx.x * kPlanThreads + tid; i < rest;
         i += (long long)gridDim.x * kPlanThreads) {
        long long at = used + i;
        if (!a.per_unit) {
            const int h = (int)(i % g.hkv);
            const long long t = i / g.hkv;
            at = (t / (a.rows - used) * a.rows + used + t % (a.rows - used)) * g.hkv + h;
        }
        a.slots[at] = -1;
    }
}

// Pages back to the ring, in the units' order: of the finished requests, or
// (done null) what holds none but the last fewer[r] tokens of request r's units.
// One block, since the lengths that the order is made from change.
__global__ void __launch_bounds__(kPlanThreads)
release_kernel(PlanGeom g, int units, const int32_t* done, const int32_t* fewer, int32_t* lengths,
               int32_t* table, int32_t* ring, int32_t* state, int* err)
{
    __shared__ long long s_sum[32];
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lh = g.layers * g.hkv;
    const long long most = (long long)g.max_blocks << g.page_log2;
    // whether a unit gives something back, and the tokens that it keeps of n
    auto gives = [&](int u) { return done ? done[u / lh] != 0 : fewer[u / lh] != 0; };
    auto kept = [&](int u, int n) { return done ? 0 : n - fewer[u / lh]; };
    if (tid == 0) s_bad = 0;
    __syncthreads();
    long long total = 0;
    bool bad = false;
    for (int u = warp; u < units; u += kPlanThreads / 32) {
        if (!gives(u)) continue;
        const int n = lengths[u];
        if (n < 0 || n > most || (!done && (fewer[u / lh] < 0 || fewer[u / lh] > n))) {
            bad = true;
            continue;
        }
        const int from = blocks_of(kept(u, n), g.page_log2), blocks = blocks_of(n, g.page_log2);
        for (int b = from + lane; b < blocks; b += 32) {
            const int page = table[(size_t)u * g.max_blocks + b];
            bad |= page < 0 || page >= g.pages;
        }
        total += blocks - from;
    }
    if (lane == 0) s_sum[warp] = total;
    if (bad) s_bad = 1;
    __syncthreads();
    total = warp_sum(s_sum[lane]);
    const int head = state[0], count = state[1];
    if (s_bad || head < 0 || head >= g.pages || count < 0 || count + total > g.pages) {
        if (tid == 0) atomicCAS(err, 0, kCacheBadIndex);
        return;
    }
    long long at = (long long)head + count;
    for (int base = 0; base < units; base += kPlanThreads) {
        const int u = base + tid;
        const bool leaves = u < units && gives(u);
        const int keeps = leaves ? kept(u, lengths[u]) : 0;
        const int from = blocks_of(keeps, g.page_log2);
        const int blocks = leaves ? blocks_of(lengths[u], g.page_log2) - from : 0;
        long long x = blocks;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) s_sum[warp] = x;
        __syncthreads();
        const long long all = warp_sum(s_sum[lane]);
        x += warp_sum(lane < warp ? s_sum[lane] : 0) - blocks;
        for (int b = 0; b < blocks; ++b) {
            int32_t* const entry = table + (size_t)u * g.max_blocks + from + b;
            ring[(at + x + b) % g.pages] = *entry;
            *entry = -1;
        }
        if (leaves) lengths[u] = keeps;
        at += all;
    }
    if (tid == 0) state[1] = (int)(count + total);
}

PlanGeom geom_of(const CacheGeom& g)
{
    return PlanGeom{g.layers, g.hkv, g.page_log2, g.pages, g.max_blocks};
}

}  // namespace

cudaError_t launch_cache_plan(const CacheGeom& g, const PlanArgs& a, cudaStream_t st)
{
    // a block per SM; more only when the units of one would not fit
    int grid = a.units < 152 ? a.units : 152;
    if ((a.units + grid - 1) / grid > kPlanUnits) grid = (a.units + kPlanUnits - 1) / kPlanUnits;
    const int own = (a.units + grid - 1) / grid;
    grid = (a.units + own - 1) / own;
    return launch_first(plan_kernel, grid, kPlanThreads, 0, st, geom_of(g), a, own, g.err);
}

cudaError_t launch_cache_release(const CacheGeom& g, int units, const int32_t* done,
                                 const int32_t* fewer, int32_t* lengths, int32_t* table,
                                 int32_t* ring, int32_t* state, cudaStream_t st)
{
    return launch_first(release_kernel, 1, kPlanThreads, 0, st, geom_of(g), units, done, fewer,
                        lengths, table, ring, state, g.err);
}

}  // namespace bacon
