// What the two attention kernels over the 8-bit pages share: the units'
// queries and lengths, page loads, and the exponent that folds V's scale in.
//
// With s_x = scale q . k_x, k_x = sK[page] * code and v_x = sV[page] * code,
//     w_x = 2^(log2e s_x + log2 sV[page] - M),  M the running maximum of that
//                                               exponent,
//     out = sum_x w_x code_x / sum_x (w_x / sV[page]),
//     lse = ln2 (log2 sum_x (w_x / sV[page]) + M):
// one exponential per logit and no multiplication by V's scale.  Sums, maxima
// and the log-sum-exp are fp32.  What is rounded to fewer bits, since operands
// of 16 bits are what the tensor cores take at full rate:
// - Nothing of K and V: codes of either format are exact in fp16.
// - Nothing that counts of the queries: a row is scaled by a power of two
//   (kQueryTop), which leaves its entries exact down to 2^-31 (bf16; fp16:
//   2^-28) of the largest; smaller ones are off by 2^-39 of it at most, less
//   than the fp32 sums lose.
// - The weights beside V, to fp16's 11 bits (the weights that are summed are
//   not).  With the largest at 2^kWeightTop they are fp16's normal values down
//   to 2^-28 of it, less and less exact below, and 0 from 2^-39 on.  The kernel
//   of many queries lets M lag and has its own range.
// Against 64 bits, relative to the output's norm: 0.0016 to 0.0017 for bf16,
// the output's own rounding; 2.1e-4 to 2.4e-4 for fp16, whose own rounding is
// 2.04e-4: the rest are the weights.
#pragma once

#include <cuda.h>

#include "cache.h"
#include "cache_values.cuh"
#include "tc.cuh"

namespace bacon {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kWeightTop = 14.0f;
constexpr int kQueryTop = 14;
constexpr int kBoxRows = 16;  // rows of one TMA load: the least page

// The queries of one request: [start, start + asked) of the call's tokens; none
// when they are the other kernel's.
struct Asked {
    int start, asked;
};

__device__ __forceinline__ Asked asked_of(const CacheGeom& g, const AttendArgs& a, int r)
{
    Asked q;
    if (!a.starts) {
        q.asked = a.tokens / a.requests;
        q.start = r * q.asked;
    } else {
        const int s = a.starts[r], e = a.starts[r + 1];
        if (s < 0 || e < s || e > a.tokens) return Asked{0, 0};
        q = Asked{s, e - s};
    }
    const long long rows = (long long)q.asked * g.group;
    return rows > a.above && rows <= a.upto ? q : Asked{0, 0};
}

// Whether the queries' ranges are what they have to be: one after the other from
// 0 to the call's tokens.  If not, no request is asked anything: ranges that
// overlap could be more items than the blocks' shares are made for, whose parts
// would be counted, and read, beyond the last block.  (A thread's first range is
// fetched when this is made and looked at in bad(), with other loads between:
// four drafts of 8 requests take 37.8 us, 38.8 with the check in one place.)
struct Ranges {
    int from, to;

    __device__ __forceinline__ Ranges(const AttendArgs& a, int tid) : from(0), to(0)
    {
        if (a.starts && tid < a.requests) {
            from = a.starts[tid];
            to = a.starts[tid + 1];
        }
    }
    __device__ __forceinline__ bool bad(const AttendArgs& a, int tid, int threads) const
    {
        if (!a.starts) return false;
        bool wrong = from > to || (tid == 0 && from != 0) || (tid == a.requests - 1 && to != a.tokens);
        for (int r = tid + threads; r < a.requests; r += threads)
            wrong |= a.starts[r] > a.starts[r + 1] || (r == a.requests - 1 && a.starts[r + 1] != a.tokens);
        return wrong;
    }
};

// Tokens of kv-head h of request r; a length that the table cannot hold counts
// as none (`bad` is set).
__device__ __forceinline__ int length_of(const CacheGeom& g, const AttendArgs& a, int r, int h,
                                         bool& bad)
{
    const int n = a.lengths[((size_t)r * g.layers + a.layer) * g.hkv + h];
    if (n >= 0 && n <= (long long)g.max_blocks << g.page_log2) return n;
    bad = true;
    return 0;
}

// How many positions query j of `asked` sees.
__device__ __forceinline__ int seen_by(const AttendArgs& a, int n, int asked, int j)
{
    return a.causal ? max(0, n - asked + j + 1) : n;
}

// TMA load of 16 rows of the pool (swizzled by the row's bytes).
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, int row, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];\n" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(bar)
        : "memory");
}

// Untiled copy of `bytes` bytes (a multiple of 16, both ends 16-byte aligned).
__device__ __forceinline__ void load_bytes(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(dst),
        "l"(src), "r"(bytes), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(bytes)
                 : "memory");
}

// The power of two that brings a query row of largest magnitude amax to
// [2^kQueryTop, 2^(kQueryTop + 1)), and its inverse; 1 for a row of zeros or
// one that is not finite.
__device__ __forceinline__ float query_scale(float amax, float& back)
{
    back = 1.0f;
    if (!(amax > 0.0f && amax < INFINITY)) return 1.0f;
    int e = (int)(__float_as_uint(amax) >> 23) - 127 - kQueryTop;  // a subnormal: at 2^-127
    e = min(max(e, -110), 120);
    back = __uint_as_float((uint32_t)(e + 127) << 23);
    return __uint_as_float((uint32_t)(127 - e) << 23);
}

// Counts a part that the block's threads have written (a block barrier lies
// between their writes and this) and tells whether it is the last of `parts`.
// Release and acquire at once: what the other blocks wrote before their counts
// can be read by the block's threads after the next barrier.
__device__ __forceinline__ bool arrive_last(int* count, int parts)
{
    int before;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;\n" : "=r"(before) : "l"(count) : "memory");
    if (before != parts - 1) return false;
    *count = 0;
    return true;
}

__device__ __forceinline__ uint32_t half2_of(float x, float y)
{
    uint32_t w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(w) : "f"(y), "f"(x));
    return w;
}

__device__ __forceinline__ float2 unpack16(int dtype, uint32_t w)
{
    return dtype == BACON_BF16 ? unpack16<BACON_BF16>(w) : unpack16<BACON_FP16>(w);
}
__device__ __forceinline__ uint32_t pack16(int dtype, float x, float y)
{
    return dtype == BACON_BF16 ? pack16<BACON_BF16>(x, y) : pack16<BACON_FP16>(x, y);
}

__device__ __forceinline__ void ldmatrix4(uint32_t* r, uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t* r, uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
// A word of a transposed V load: token 2t's codes of dims 2g and 2g + 1, then
// token 2t + 1's.  lo: both tokens of dim 2g, hi: of dim 2g + 1.
template <int FORMAT>
__device__ __forceinline__ void pairs_half(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    if (FORMAT == BACON_E4M3) {
        codes_half<FORMAT>(__byte_perm(w, 0, 0x3120), lo, hi);
    } else {
        const uint32_t u = w ^ 0x80808080u;
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4240);
        const uint32_t b = __byte_perm(u, 0x64646464u, 0x4341);
        const uint32_t off = 0x64806480u;
        asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(lo) : "r"(a), "r"(off));
        asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(hi) : "r"(b), "r"(off));
    }
}

// ROWS rows (columns, where the tokens are the rows) of a unit's queries: row c
// is query c / group, head c % group.
struct Item {
    int r, h, block;
    int n, start, asked;
    int seen;   // positions that some row sees
    int tiles;  // at least one, so that an item of no token writes its outputs
};

template <int ROWS>
__device__ __forceinline__ int blocks_of(const CacheGeom& g, int asked)
{
    return (int)(((long long)asked * g.group + ROWS - 1) / ROWS);
}

template <int ROWS, int TILE>
__device__ __forceinline__ void set_block(const CacheGeom& g, const AttendArgs& a, Item& it, int block)
{
    it.block = block;
    const int last = min(it.asked - 1, (block * ROWS + ROWS - 1) / g.group);
    it.seen = seen_by(a, it.n, it.asked, last);
    it.tiles = max(1, (int)(((long long)it.seen + TILE - 1) / TILE));
}

template <int ROWS, int TILE>
__device__ __forceinline__ Item item_of(const CacheGeom& g, const AttendArgs& a, int unit, int block,
                                        bool& bad)
{
    Item it;
    it.r = unit / g.hkv;
    it.h = unit - it.r * g.hkv;
    const Asked q = asked_of(g, a, it.r);
    it.start = q.start;
    it.asked = q.asked;
    it.n = length_of(g, a, it.r, it.h, bad);
    set_block<ROWS, TILE>(g, a, it, block);
    return it;
}

// The length of the unit after `unit`, as it stands there (nothing waits for it).
__device__ __forceinline__ int length_ahead(const CacheGeom& g, const AttendArgs& a, int unit)
{
    if (++unit >= a.requests * g.hkv) return 0;
    const int r = unit / g.hkv;
    return a.lengths[((size_t)r * g.layers + a.layer) * g.hkv + (unit - r * g.hkv)];
}

// The item after `it` that has rows; false at the end of the call's.
template <int ROWS, int TILE>
__device__ __forceinline__ bool next_item(const CacheGeom& g, const AttendArgs& a, int& unit, Item& it)
{
    if (it.block + 1 < blocks_of<ROWS>(g, it.asked)) {
        set_block<ROWS, TILE>(g, a, it, it.block + 1);
        return true;
    }
    bool bad = false;
    while (++unit < a.requests * g.hkv) {
        it = item_of<ROWS, TILE>(g, a, unit, 0, bad);
        if (it.asked > 0) return true;
    }
    return false;
}

// x / y; in 32 bits where that is enough.
__device__ __forceinline__ long long quotient(long long x, long long y)
{
    return (x | y) >> 32 ? x / y : (long long)((unsigned)x / (unsigned)y);
}

// What a block does: tiles [lo, hi), counted so that the first of them lies in
// the item that `Found` has, one of unit `unit` whose first tile is `at`.
//
// Dealt evenly, the tiles of all items stand one after the other and block b
// has the b-th share, wherever items end.  A block whose tiles lie in two items
// forms and joins sums twice, which a few tiles do not pay for: a call with
// few items and few tiles gives each item blocks of its own, `run` tiles each.
struct Place {
    long long total, lo, hi, at;
    long long share;  // tiles of a block; the first `more` blocks have one more
    int blocks, more, unit;
    int run;          // > 0: blocks of their own
    int first, parts; // and then the first of them and their number

    __device__ __forceinline__ long long first_tile(int b) const { return share * b + min(b, more); }
    __device__ __forceinline__ int owner_of(long long tile) const
    {
        const long long long_ones = (share + 1) * more;
        return tile < long_ones ? (int)quotient(tile, share + 1)
                                : more + (int)quotient(tile - long_ones, share);
    }
    // the blocks of a cut item whose first tile is `item_at`
    __device__ __forceinline__ void parts_of(long long item_at, int tiles, int& from, int& count) const
    {
        from = run ? first : owner_of(item_at);
        count = run ? parts : owner_of(item_at + tiles - 1) - from + 1;
    }
};
struct Found {
    Item it;
    long long at;
    int unit;
};

// Finds the block's place by a scan of all items; false when it has none.
//
// An entry is an item when all requests have the same number of queries, else
// a unit with all its items.  Each warp takes a run of entries, a lane an
// entry at a time: their sums give the total and the warps' places, and the
// warp that has the block's first tile walks its entries again to find it.
template <int ROWS, int TILE, int THREADS, int LEAST>
__device__ __forceinline__ bool find_place(const CacheGeom& g, const AttendArgs& a, long long* scan,
                                           Found& found, Place& p)
{
    constexpr int kWarps = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool same = a.starts == nullptr;
    Asked q = {0, 0};
    if (same) q = asked_of(g, a, 0);
    const unsigned each = same ? blocks_of<ROWS>(g, q.asked) : 1;
    const unsigned entries = (unsigned)a.requests * g.hkv * each;
    const unsigned run = (entries + THREADS - 1) / THREADS * 32;
    const unsigned e0 = warp * run + lane, e1 = min(entries, (warp + 1) * run);
    const Ranges ranges(a, threadIdx.x);
    bool bad = false, refused = false;

    // one item a unit, which sees all its tokens: only lengths are needed, on
    // their way together and kept
    const bool short_run = same && each == 1 && run <= 256;
    int n[8];
    if (short_run) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned e = e0 + i * 32, r = e / (unsigned)g.hkv;
            n[i] = -1;
            if (e < e1) n[i] = a.lengths[((size_t)r * g.layers + a.layer) * g.hkv + (e - r * g.hkv)];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (e0 + i * 32 < e1 && (n[i] < 0 || n[i] > (long long)g.max_blocks << g.page_log2)) {
                bad = true;
                n[i] = 0;
            }
    }
    auto tiles_of_unit = [](int x) { return max(1, (int)(((unsigned)x + TILE - 1) / TILE)); };

    // entry e as its first item, the number of its items in `items`
    auto entry = [&](unsigned e, int& unit, int& items) {
        Item it;
        int block = 0;
        unit = (int)e;
        if (each > 1) {
            unit = (int)(e / each);
            block = (int)(e - unit * each);
        }
        it.r = (unsigned)unit / (unsigned)g.hkv;
        it.h = unit - it.r * g.hkv;
        it.n = length_of(g, a, it.r, it.h, bad);
        if (!same) q = asked_of(g, a, it.r);
        it.asked = q.asked;
        it.start = same ? it.r * q.asked : q.start;
        items = same ? 1 : blocks_of<ROWS>(g, q.asked);
        set_block<ROWS, TILE>(g, a, it, block);
        return it;
    };
    // runs of `by` tiles of all of an entry's items
    auto runs_of = [&](Item it, int items, int by) {
        long long sum = 0;
        for (int i = 0; i < items; ++i) {
            if (i) set_block<ROWS, TILE>(g, a, it, i);
            sum += by == 1 ? it.tiles : (unsigned)(it.tiles + by - 1) / (unsigned)by;
        }
        return sum;
    };
    // the sum of them over all entries, that of the warps before in `before`
    long long mine, before = 0;
    auto sum_of = [&](int by) {
        mine = 0;
        if (short_run) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (n[i] >= 0) {
                    const int tiles = tiles_of_unit(n[i]);
                    mine += by == 1 ? tiles : (unsigned)(tiles + by - 1) / (unsigned)by;
                }
        } else {
            for (unsigned e = e0; e < e1; e += 32) {
                int unit, items;
                const Item it = entry(e, unit, items);
                mine += runs_of(it, items, by);
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
        if (by == 1) refused = ranges.bad(a, threadIdx.x, THREADS);
        if (__any_sync(0xFFFFFFFFu, refused)) mine = -(1ll << 56);  // all of it then
        if (lane == 0) scan[warp] = mine;
        __syncthreads();
        long long all = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) before = all;
            all += scan[w];
        }
        return all;
    };
    p.total = sum_of(1);
    if (bad || (refused && blockIdx.x == 0)) atomicCAS(g.err, 0, kCacheBadIndex);
    if (p.total < 0) return false;
    // requests with other numbers of queries: no more items than this
    const long long items = same ? (long long)entries
                                 : ((long long)a.tokens * g.group / ROWS + a.requests) * g.hkv;
    const int grid = gridDim.x, b = blockIdx.x;
    p.run = 0;
    if (items * 4 <= grid && p.total <= 16LL * grid) {
        // at most total / run + items blocks
        p.run = max(LEAST, (int)((unsigned)(p.total + grid - items - 1) / (unsigned)(grid - items)));
        p.blocks = (int)p.total;
        if (p.run > 1) {
            __syncthreads();
            p.blocks = (int)sum_of(p.run);
        }
    } else {
        p.blocks = p.total < grid ? (int)p.total : grid;
        p.share = p.blocks ? quotient(p.total, p.blocks) : 0;
        p.more = (int)(p.total - p.share * p.blocks);
    }
    if (b >= p.blocks) return false;
    if (!p.run) {
        p.lo = p.first_tile(b);
        p.hi = p.first_tile(b + 1);
    }
    const int by = max(p.run, 1);
    const long long target = p.run ? b : p.lo;
    const bool has = target >= before && target < before + mine;
    if (has && short_run) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int tiles = n[i] < 0 ? 0 : tiles_of_unit(n[i]);
            const int own = by == 1 ? tiles : (unsigned)(tiles + by - 1) / (unsigned)by;
            int x = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
                if (lane >= o) x += y;
            }
            const int all = __shfl_sync(0xFFFFFFFFu, x, 31);
            if (target < before + all) {
                if (before + x - own <= target && target < before + x) {
                    Item it;
                    const int unit = (int)(e0 + i * 32);
                    it.r = (unsigned)unit / (unsigned)g.hkv;
                    it.h = unit - it.r * g.hkv;
                    it.block = 0;
                    it.n = it.seen = n[i];
                    it.asked = q.asked;
                    it.start = it.r * q.asked;
                    it.tiles = tiles;
                    found = Found{it, before + x - own, unit};
                }
                break;
            }
            before += all;
        }
    } else if (has) {
        for (unsigned e = e0;; e += 32) {
            int unit = 0, count_of = 0;
            Item it;
            long long own = 0;
            if (e < e1) {
                it = entry(e, unit, count_of);
                own = runs_of(it, count_of, by);
            }
            long long x = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
                if (lane >= o) x += y;
            }
            const long long all = __shfl_sync(0xFFFFFFFFu, x, 31);
            if (target < before + all) {
                long long at = before + x - own;
                if (at <= target && target < at + own) {
                    for (int i = 1; target >= at + (it.tiles + by - 1) / by; ++i) {
                        at += (it.tiles + by - 1) / by;
                        set_block<ROWS, TILE>(g, a, it, i);
                    }
                    found = Found{it, at, unit};
                }
                break;
            }
            before += all;
        }
    }
    __syncthreads();
    p.at = found.at;
    p.unit = found.unit;
    if (p.run) {
        const int k = b - (int)found.at, tiles = found.it.tiles;
        p.first = (int)found.at;
        p.parts = (tiles + by - 1) / by;
        p.at = 0;
        p.lo = (long long)k * by;
        p.hi = min((long long)tiles, p.lo + by);
    }
    return true;
}

}  // namespace bacon
