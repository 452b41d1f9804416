// Attention of few queries per unit over the 8-bit pages: a decoding step, or
// a few drafted tokens.
//
// Bound by the pages' bytes: a token of a unit is 2 d bytes for 4 d flops a
// query head, so with up to 32 columns (query heads of the kv-head x queries)
// the work is a stream through HBM with two small matrix products beside it.
// A token of 32 requests over 16384 rows (28 / 4 heads of 128) takes 96 us, 86 %
// of the measured copy bandwidth; of four requests over 1024, 12 us, which are
// the launch, the scan, one tile and the joining of 17 parts one after the
// other.  (At head_dim 128 the computing warps' registers do not suffice: 12 to
// 84 bytes a thread are spilled.)
// The products are warp-level (m16n8k16, fp16 in, fp32 sums) with the tokens
// as rows and the columns as n, so that no more than the next 8 columns are
// padded: S^T = K Q^T, then O^T = V^T P^T.  K and V codes go from shared
// memory to fragments by 8x8 matrix loads whose 16-bit elements are two codes
// (V's transposed ones bring two tokens' codes of two dims into a register),
// and become fp16 there; what order the dims take inside a product is the
// same for Q's fragments.  S^T turns into P^T's operand by 8x8 transposes.
//
// The call's tiles are dealt out to the blocks evenly, an item (8 NT CG columns
// of a unit) after the other, whatever the units' lengths.  Every block finds
// its place by a scan of the lengths, so no host synchronisation and no second
// launch come before; a warp of it loads (16 rows a TMA load, only rows that
// the item sees, pages and scales on their way ahead), the others compute, each
// with its own running maximum, and join at the item's end.  An item cut by a
// block's edge leaves partial sums; the last of its blocks to arrive adds them
// up in the blocks' order, so the result does not depend on timing.
#include <cmath>

#include "cache_attend.cuh"

namespace bacon {
namespace {

using namespace tc;

constexpr int kGroups = 4;  // warps beside one another on a stage's tokens

struct Meta {  // of 16 tokens of a stage
    float k_scale, v_log2, v_inv;
};

// Sizes for CG groups of 8 NT columns.  A warp takes 16 MT tokens of a stage and
// a group's columns; with two groups the codes are converted by two warps each,
// which costs less than 32 columns' sums in one warp's registers do: 9 warps
// have 168 registers a thread, 128 of them would be sums.  MT = 2 gives a stage
// the bytes that its barriers and its maximum are worth, and two independent
// chains: at head_dim 64 and for two groups (us, MT = 1 and 2: a token of 32
// requests over 8192 rows of 64 69 and 56; four tokens of 8 over 16384 of 128
// 75 and 72), but with one group at 128 it leaves two blocks on an SM instead
// of three (a token of 24 multi-head requests over 256 rows 25.7 and 27.7).
template <int D, int NT, int CG>
struct Sizes {
    static constexpr int kMT = D == 64 || CG == 2 ? 2 : 1;
    static constexpr int kTile = 16 * kMT * kGroups;  // tokens of a stage
    static constexpr int kWarps = kGroups * CG;       // that compute
    static constexpr int kThreads = 32 * (kWarps + 1);
    static constexpr int kColumns = 8 * NT * CG;
    static constexpr int kPerSm = CG == 2 ? 1 : NT == 2 ? 2 : 3;
    static constexpr int kStages = D == 128 && CG == 2 ? 3 : CG == 2 ? 6 : NT == 2 ? 4 : 3;
    static constexpr int kRows = kTile * D;        // bytes of K, or V, of a stage
    static constexpr int kStage = 2 * kRows;
    static constexpr int kJoin = kStages * kStage; // the warps' outputs
    static constexpr int kPitch = D * 2 + 32;      // of a query row: 8 rows on distinct banks
    static constexpr int kQueries = kColumns * kPitch;
    static constexpr int kRaw = kJoin + kWarps * NT * D * 8 * 4;  // two items' query rows
    static constexpr int kShared = kRaw + 2 * kQueries;
    static constexpr int kBytes = kShared + 3072;
};
static_assert(Sizes<128, 1, 1>::kPerSm * (Sizes<128, 1, 1>::kBytes + 1024) <= 228 * 1024, "blocks on an SM");
static_assert(Sizes<64, 1, 1>::kPerSm * (Sizes<64, 1, 1>::kBytes + 1024) <= 228 * 1024, "blocks on an SM");
static_assert(2 * (Sizes<128, 2, 1>::kBytes + 1024) <= 228 * 1024, "two blocks on an SM");
static_assert(Sizes<128, 2, 2>::kBytes <= 227 * 1024, "one block on an SM");

struct Segment {  // tiles [begin, end) of an item, whose first tile is tile `at` of the call
    Item it;
    int begin, end;
    long long at;
};

template <int STAGES, int MT>
struct Shared {
    Meta meta[STAGES][kGroups * MT];
    float top[kGroups][32], sum[kGroups][32];
    uint64_t full[STAGES], empty[STAGES], q_full[2], q_empty[2];
    Segment seg[2];
    long long scan[9];
    Found found;
    int abort, last, quit;
    int nan_at[128];  // per dim: first position of a NaN of V that not every column sees
    int nan_any;
};
static_assert(sizeof(Shared<6, 2>) <= 3072, "shared record");

__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int FORMAT, int D, int NT, int CG>
__global__ void __launch_bounds__(Sizes<D, NT, CG>::kThreads, Sizes<D, NT, CG>::kPerSm)
few_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
           CacheGeom g, AttendArgs a, SplitScratch sc)
{
    using S = Sizes<D, NT, CG>;
    constexpr int kChunks = D / 16, kWarps = S::kWarps, kStages = S::kStages;
    constexpr int kThreads = S::kThreads, kColumns = S::kColumns, kTile = S::kTile, kMT = S::kMT;
    extern __shared__ __align__(1024) uint8_t smem[];
    auto& sh = *reinterpret_cast<Shared<kStages, kMT>*>(smem + S::kShared);
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 1);
            mbar_init(smem_u32(&sh.empty[s]), kWarps);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&sh.q_full[s]), 1);
            mbar_init(smem_u32(&sh.q_empty[s]), kWarps);
        }
        fence_barrier_init();
        sh.abort = sh.nan_any = 0;
    }
    for (int i = tid; i < 128; i += kThreads) sh.nan_at[i] = 0x7FFFFFFF;

    Place place;
    if (!find_place<kColumns, kTile, kThreads, 1>(g, a, sh.scan, sh.found, place)) return;
    const int b = blockIdx.x;
    const long long lo = place.lo, hi = place.hi;
    const uint32_t abort_flag = smem_u32(&sh.abort);

    if (warp == kWarps) {
        // ------------------------------------------------------ loads
        int unit = place.unit;
        Item it = sh.found.it;
        long long at = place.at;  // the item's first tile
        // tiles, counted so that the one whose load a test withholds is tile 0
        const int from = a.fault ? 1 - a.fault : 0;
        int stage = 0, issued = from, items = 0;
        uint32_t phase = 0;
        bool stop = false;
        // Nothing is asked for once the block has given up: warps that did go on
        // freeing stages, also one whose load never came and whose barrier is
        // still open.  (The flag is set before the stage is freed; to have those
        // warps keep such a stage instead costs a register where there is none:
        // 26.4 us for 25.5.)  One answer for the warp, whose lanes vote below.
        auto gone = [&](uint32_t bar, uint32_t parity) {
            const bool there = mbar_wait(bar, parity, abort_flag) && !ld_shared_volatile(abort_flag);
            return !__all_sync(0xFFFFFFFFu, there);
        };
        long long t = lo;
        while (t < hi && !stop) {
            const int begin = (int)(t - at), end = (int)min((long long)it.tiles, hi - at);
            {
                // the item and its query rows, a lane a column
                const int slot = items & 1;
                const uint32_t full = smem_u32(&sh.q_full[slot]);
                if (gone(smem_u32(&sh.q_empty[slot]), (items >> 1 & 1) ^ 1)) {
                    stop = true;
                    break;
                }
                if (lane == 0) sh.seg[slot] = Segment{it, begin, end, at};
                const int c = it.block * kColumns + lane, j = c / g.group;
                const bool live = lane < kColumns && j < it.asked;
                const int rows = __popc(__ballot_sync(0xFFFFFFFFu, live));
                if (lane == 0) mbar_expect_tx(full, rows * D * 2);
                __syncwarp();
                const int row = S::kRaw + slot * S::kQueries + lane * S::kPitch;
                if (live) {
                    load_bytes(base + row,
                               a.q + (long long)(it.start + j) * a.q_token_stride +
                                   (it.h * g.group + c % g.group) * a.q_head_stride,
                               D * 2, full);
                } else if (lane < kColumns) {
#pragma unroll 1
                    for (int i = 0; i < D * 2; i += 16)
                        *reinterpret_cast<uint4*>(smem + row + i) = make_uint4(0, 0, 0, 0);
                    // a later item's copy writes the same bytes
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(full);
                ++items;
            }
            // on their way ahead of their use: the next unit's length, pages
            // by two tiles, scales by one
            const bool last_of_unit = it.block + 1 >= blocks_of<kColumns>(g, it.asked);
            const int ahead = last_of_unit ? length_ahead(g, a, unit) : 0;
            // a lane a 16-row group of a tile: K's first, then V's
            constexpr int kBoxes = kGroups * kMT;
            const int group = lane % kBoxes;
            const bool of_v = lane >= kBoxes;
            const float* const scales = of_v ? g.v_scale : g.k_scale;
            const int32_t* const table =
                a.table + (((size_t)it.r * g.layers + a.layer) * g.hkv + it.h) * g.max_blocks;
            const int upto = lane < 2 * kBoxes ? (int)min((long long)it.seen, (long long)end * kTile) : 0;
            auto page_of = [&](int i) {
                const int pos = i * kTile + group * 16;
                return pos < upto ? table[pos >> g.page_log2] : 0;
            };
            auto checked = [&](int page) {
                if (page >= 0 && page < g.pages) return page;
                atomicCAS(g.err, 0, kCacheBadIndex);
                return 0;
            };
            int page = page_of(begin), page1 = page_of(begin + 1);
            page = checked(page);
            float s = scales[page];
            for (int i = begin; i < end; ++i, ++t) {
                const int pos = i * kTile + group * 16;
                const bool live = pos < upto;
                const int page2 = page_of(i + 2);
                page1 = checked(page1);
                const float s1 = scales[page1];
                const uint32_t full = smem_u32(&sh.full[stage]);
                if (gone(smem_u32(&sh.empty[stage]), phase ^ 1)) {
                    stop = true;
                    break;
                }
                const int boxes = __popc(__ballot_sync(0xFFFFFFFFu, live));
                if (lane == 0 && boxes) mbar_expect_tx(full, boxes * kBoxRows * D);
                __syncwarp();
                if (live && !(a.fault && b == 0 && issued == 0 && lane == 0))
                    load_rows(base + stage * S::kStage + (of_v ? S::kRows : 0) + group * 16 * D,
                              of_v ? &vmap : &kmap, (page << g.page_log2) + (pos & (g.page - 1)), full);
                if (!live) s = 1.0f;
                if (lane < kBoxes) {
                    sh.meta[stage][group].k_scale = s;
                } else if (lane < 2 * kBoxes) {
                    sh.meta[stage][group].v_log2 = log2f(s);
                    sh.meta[stage][group].v_inv = 1.0f / s;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(full);
                ++issued;
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1;
                }
                page = page1;
                page1 = page2;
                s = s1;
            }
            at += it.tiles;
            if (at >= hi || stop) break;
            if (last_of_unit) {
                ++unit;
                it.n = ahead >= 0 && ahead <= (long long)g.max_blocks << g.page_log2 ? ahead : 0;
                it.r = unit / g.hkv;
                it.h = unit - it.r * g.hkv;
                const Asked q = asked_of(g, a, it.r);
                it.start = q.start;
                it.asked = q.asked;
                set_block<kColumns, kTile>(g, a, it, 0);
                if (it.asked == 0 && !next_item<kColumns, kTile>(g, a, unit, it)) break;
            } else {
                set_block<kColumns, kTile>(g, a, it, it.block + 1);
            }
        }
        if (stop && lane == 0) {
            st_shared_volatile(abort_flag, 1);
            atomicCAS(g.err, 0, kCacheTimeout);
        }
        // The block's copies end before it does, also when those who waited for
        // them have given up after the last was asked for: the last phase of
        // each barrier (there, as a rule, by the time the warp gets here).
        issued -= from;
        for (int i = max(0, issued - kStages); i < issued; ++i)
            mbar_wait(smem_u32(&sh.full[i % kStages]), i / kStages & 1, 0);
        for (int i = max(0, items - 2); i < items; ++i)
            mbar_wait(smem_u32(&sh.q_full[i & 1]), i >> 1 & 1, 0);
        return;
    }

    // ---------------------------------------------------------- products
    const int gr = lane >> 2, tq = lane & 3;
    const int group = warp % kGroups, first_col = warp / kGroups * 8 * NT;
    int stage = 0;
    uint32_t phase = 0;
    float acc[kChunks][NT][4];
    float top[NT][2], sum[NT][2], factor[NT][2];
    int sees[NT][2];
    uint32_t qf[kChunks][NT][2];
    // matrix loads: lane l gives row l & 7 of matrix l >> 3; matrices are rows
    // 0-7, rows 8-15, of 16-byte chunk c, then of c + 1
    const int mrow = group * 16 * kMT + (lane & 7) + (lane >> 3 & 1) * 8, mchunk = lane >> 4;
    const uint32_t swizzle = D == 128 ? mrow & 7 : mrow >> 1 & 3;

    int items = 0;
    for (long long t = lo; t < hi; ++items) {
        const int slot = items & 1;
        const bool there = mbar_wait(smem_u32(&sh.q_full[slot]), items >> 1 & 1, abort_flag);
        if (!there && lane == 0) {
            st_shared_volatile(abort_flag, 1);
            atomicCAS(g.err, 0, kCacheTimeout);
        }
        if (tid == 0) sh.quit = !there;
        named_barrier_sync(1, 32 * kWarps);
        if (sh.quit) return;  // the same for all that compute
        const Segment seg = sh.seg[slot];
        const Item& it = seg.it;
        // the item's queries as fragments: column g of an n-tile, dims 16 c +
        // 4 tq ... + 3 of every chunk c
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float amax = 0.0f;
            uint2 raw[kChunks];
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
                raw[k] = *reinterpret_cast<const uint2*>(smem + S::kRaw + slot * S::kQueries +
                                                         (first_col + nt * 8 + gr) * S::kPitch + k * 32 + tq * 8);
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                const float2 u = unpack16(g.dtype, raw[k].x), v = unpack16(g.dtype, raw[k].y);
                amax = fmaxf(fmaxf(amax, fmaxf(fabsf(u.x), fabsf(u.y))), fmaxf(fabsf(v.x), fabsf(v.y)));
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
            float back;
            const float up = query_scale(amax, back);
            back *= a.scale * kLog2e;
            factor[nt][0] = __shfl_sync(0xFFFFFFFFu, back, tq * 8);
            factor[nt][1] = __shfl_sync(0xFFFFFFFFu, back, tq * 8 + 4);
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                const float2 u = unpack16(g.dtype, raw[k].x), v = unpack16(g.dtype, raw[k].y);
                qf[k][nt][0] = half2_of(u.x * up, u.y * up);
                qf[k][nt][1] = half2_of(v.x * up, v.y * up);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int col = it.block * kColumns + first_col + nt * 8 + tq * 2 + i;
                sees[nt][i] = col / g.group < it.asked ? seen_by(a, it.n, it.asked, col / g.group) : 0;
                top[nt][i] = -INFINITY;
                sum[nt][i] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[k][nt][i] = 0.0f;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.q_empty[slot]));
        // positions that every column sees
        const int all = seen_by(a, it.n, it.asked, it.block * kColumns / g.group);
        const int begin = seg.begin, end = seg.end;
        for (int i = begin; i < end; ++i) {
            if (!mbar_wait(smem_u32(&sh.full[stage]), phase, abort_flag) && lane == 0) {
                st_shared_volatile(abort_flag, 1);
                atomicCAS(g.err, 0, kCacheTimeout);
            }
            __syncwarp();
            const int pos = i * kTile + group * 16 * kMT;
            if (pos < it.seen) {
                const uint32_t krow = base + stage * S::kStage + mrow * D;
                float y[kMT][NT][4];
#pragma unroll
                for (int t = 0; t < kMT; ++t) {
                    float s[NT][2][4];  // two chains of products
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[nt][0][e] = s[nt][1][e] = 0.0f;
#pragma unroll
                    for (int c = 0; c < kChunks; c += 2) {
                        uint32_t w[4], f[8];
                        ldmatrix4(w, krow + t * 16 * D + (((c + mchunk) ^ swizzle) << 4));
                        // rows gr and gr + 8, first pairs of dims then second ones
                        codes_half<FORMAT>(w[0], f[0], f[2]);
                        codes_half<FORMAT>(w[1], f[1], f[3]);
                        codes_half<FORMAT>(w[2], f[4], f[6]);
                        codes_half<FORMAT>(w[3], f[5], f[7]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma(s[nt][0], f, qf[c][nt][0], qf[c][nt][1]);
                            mma(s[nt][1], f + 4, qf[c + 1][nt][0], qf[c + 1][nt][1]);
                        }
                    }
                    const float ks = sh.meta[stage][group * kMT + t].k_scale;
                    const float vl = sh.meta[stage][group * kMT + t].v_log2;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            y[t][nt][e] = (s[nt][0][e] + s[nt][1][e]) * (factor[nt][e & 1] * ks) + vl;
                }
                // exponents, the running maximum, weights
                const bool cut = pos + 16 * kMT > all;
                uint32_t p[kMT][NT][2];
                bool grew = false;
                float keep[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (cut) {
#pragma unroll
                        for (int t = 0; t < kMT; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (pos + t * 16 + gr + (e >> 1) * 8 >= sees[nt][e & 1]) y[t][nt][e] = -INFINITY;
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float high = fmaxf(y[0][nt][k], y[0][nt][k + 2]);
#pragma unroll
                        for (int t = 1; t < kMT; ++t) high = fmaxf(high, fmaxf(y[t][nt][k], y[t][nt][k + 2]));
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) high = fmaxf(high, __shfl_xor_sync(0xFFFFFFFFu, high, o));
                        keep[nt][k] = 1.0f;
                        if (high > top[nt][k]) {
                            keep[nt][k] = fast_exp2(top[nt][k] - high);
                            top[nt][k] = high;
                            grew = true;
                        }
                        const float m = top[nt][k] == -INFINITY ? 0.0f : top[nt][k] - kWeightTop;
                        sum[nt][k] *= keep[nt][k];
#pragma unroll
                        for (int t = 0; t < kMT; ++t) {
                            y[t][nt][k] = fast_exp2(y[t][nt][k] - m);
                            y[t][nt][k + 2] = fast_exp2(y[t][nt][k + 2] - m);
                            sum[nt][k] = fmaf(y[t][nt][k] + y[t][nt][k + 2],
                                              sh.meta[stage][group * kMT + t].v_inv, sum[nt][k]);
                        }
                    }
#pragma unroll
                    for (int t = 0; t < kMT; ++t) {
                        p[t][nt][0] = transpose8(half2_of(y[t][nt][0], y[t][nt][1]));
                        p[t][nt][1] = transpose8(half2_of(y[t][nt][2], y[t][nt][3]));
                    }
                }
                if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[c][nt][e] *= keep[nt][e & 1];
                }
#pragma unroll
                for (int t = 0; t < kMT; ++t) {
                    const uint32_t vrow = krow + S::kRows + t * 16 * D;
#pragma unroll
                    for (int c = 0; c < kChunks; c += 2) {
                        uint32_t w[4], f[8];
                        ldmatrix4_trans(w, vrow + (((c + mchunk) ^ swizzle) << 4));
                        if (cut) {
                            // rows that no column sees are whatever the page
                            // holds; a NaN that some column does not see is
                            // taken out and put back at the item's end
#pragma unroll
                            for (int m = 0; m < 4; ++m) {
                                const int x0 = pos + t * 16 + (m & 1) * 8 + 2 * tq;
                                if (x0 >= it.seen) w[m] &= 0xFFFF0000u;
                                if (x0 + 1 >= it.seen) w[m] &= 0x0000FFFFu;
                                if (FORMAT == BACON_E4M3 &&
                                    (((w[m] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u)) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        if ((w[m] >> (8 * e) & 0x7Fu) == 0x7Fu) {
                                            w[m] &= ~(0xFFu << (8 * e));
                                            atomicMin(&sh.nan_at[(c + (m >> 1)) * 16 + 2 * gr + (e & 1)],
                                                      x0 + (e >> 1));
                                            sh.nan_any = 1;
                                        }
                                }
                            }
                        }
                        // rows gr: dim 2 gr, rows gr + 8: dim 2 gr + 1 of a chunk
                        pairs_half<FORMAT>(w[0], f[0], f[1]);
                        pairs_half<FORMAT>(w[1], f[2], f[3]);
                        pairs_half<FORMAT>(w[2], f[4], f[5]);
                        pairs_half<FORMAT>(w[3], f[6], f[7]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma(acc[c][nt], f, p[t][nt][0], p[t][nt][1]);
                            mma(acc[c + 1][nt], f + 4, p[t][nt][0], p[t][nt][1]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.empty[stage]));
            if (++stage == kStages) {
                stage = 0;
                phase ^= 1;
            }
        }

        // ------------------------------------------- the warps' sums joined
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) sum[nt][k] += __shfl_xor_sync(0xFFFFFFFFu, sum[nt][k], o);
                if (gr == 0) {
                    sh.top[group][first_col + nt * 8 + tq * 2 + k] = top[nt][k];
                    sh.sum[group][first_col + nt * 8 + tq * 2 + k] = sum[nt][k];
                }
            }
        named_barrier_sync(1, 32 * kWarps);
        const bool nan = sh.nan_any != 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int col = first_col + nt * 8 + tq * 2 + k;
                float m = sh.top[0][col];
#pragma unroll
                for (int w = 1; w < kGroups; ++w) m = fmaxf(m, sh.top[w][col]);
                const float f = top[nt][k] == -INFINITY ? 0.0f : fast_exp2(top[nt][k] - m);
                float l = 0.0f;
#pragma unroll
                for (int w = 0; w < kGroups; ++w)  // (a sum of NaN has no maximum)
                    l += sh.sum[w][col] * (sh.top[w][col] == -INFINITY ? 0.0f : fast_exp2(sh.top[w][col] - m));
                top[nt][k] = m;
                sum[nt][k] = l;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    acc[c][nt][k] *= f;
                    acc[c][nt][k + 2] *= f;
                }
            }
        // every warp adds up its chunks of all groups' outputs
        constexpr int kOwn = kChunks / kGroups;
        const int c0 = group * kOwn;
        float4* const join =
            reinterpret_cast<float4*>(smem + S::kJoin) + warp / kGroups * kGroups * kChunks * NT * 32;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                join[(group * kChunks * NT + c * NT + nt) * 32 + lane] = *reinterpret_cast<float4*>(acc[c][nt]);
        named_barrier_sync(1, 32 * kWarps);
        float o[kOwn][NT][4];
#pragma unroll
        for (int c = 0; c < kOwn; ++c)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float4 x = join[((c0 + c) * NT + nt) * 32 + lane];
#pragma unroll
                for (int w = 1; w < kGroups; ++w) {
                    const float4 y = join[(w * kChunks * NT + (c0 + c) * NT + nt) * 32 + lane];
                    x.x += y.x;
                    x.y += y.y;
                    x.z += y.z;
                    x.w += y.w;
                }
                *reinterpret_cast<float4*>(o[c][nt]) = x;
                if (nan) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (sh.nan_at[(c0 + c) * 16 + 2 * gr + (e >> 1)] < sees[nt][e & 1]) o[c][nt][e] = NAN;
                }
            }

        const bool whole = begin == 0 && end == it.tiles;
        // the columns' outputs of this warp's chunks
        auto write = [&] {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int col = it.block * kColumns + first_col + nt * 8 + tq * 2 + k, j = col / g.group;
                    if (j >= it.asked) continue;
                    const size_t row = (size_t)(it.start + j) * g.hq + it.h * g.group + col % g.group;
                    const bool none = sees[nt][k] == 0;
                    const float inv = none ? 0.0f : 1.0f / sum[nt][k];
                    uint32_t* const to = reinterpret_cast<uint32_t*>(a.out + row * D) + c0 * 8 + gr;
#pragma unroll
                    for (int c = 0; c < kOwn; ++c)
                        to[c * 8] = none ? 0u : pack16(g.dtype, o[c][nt][k] * inv, o[c][nt][k + 2] * inv);
                    if (a.lse && gr == 0 && group == 0)
                        a.lse[row] = none ? -INFINITY
                                          : (log2f(sum[nt][k]) + (top[nt][k] - kWeightTop)) * kLn2;
                }
        };
        if (whole) {
            write();
        } else {
            int first, parts;
            place.parts_of(seg.at, it.tiles, first, parts);
            // of a part: a column group's outputs as its warp holds them, then
            // the columns' maxima and sums
            const int mine = warp / kGroups * kChunks * NT * 32 + lane;
            // slot 2 b + 1: the item's first part, 2 b: a later one
            const size_t part = 2 * (size_t)b + (begin == 0 ? 1 : 0);
            float4* const po = reinterpret_cast<float4*>(sc.out + part * 32 * 128) + mine;
            float2* const pm = reinterpret_cast<float2*>(sc.sums + part * 64) + first_col;
#pragma unroll
            for (int c = 0; c < kOwn; ++c)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    po[((c0 + c) * NT + nt) * 32] = *reinterpret_cast<float4*>(o[c][nt]);
            if (gr == 0 && group == 0)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        pm[nt * 8 + tq * 2 + k] = make_float2(top[nt][k], sum[nt][k]);
            named_barrier_sync(1, 32 * kWarps);
            if (tid == 0) sh.last = arrive_last(&sc.arrived[first], parts);
            named_barrier_sync(1, 32 * kWarps);
            if (sh.last) {
                // the parts in the blocks' order, some at a time
                constexpr int kBatch = NT == 1 ? 8 : 4;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    top[nt][0] = top[nt][1] = -INFINITY;
                    sum[nt][0] = sum[nt][1] = 0.0f;
#pragma unroll
                    for (int c = 0; c < kOwn; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[c][nt][e] = 0.0f;
                }
#pragma unroll 1
                for (int q0 = 0; q0 < parts; q0 += kBatch) {
                    float2 z[kBatch][NT][2];
                    float4 x[kBatch][kOwn][NT];
#pragma unroll
                    for (int q = 0; q < kBatch; ++q) {
                        const bool there = q0 + q < parts;
                        const size_t part = 2 * (size_t)(first + q0 + q) + (q0 + q == 0 ? 1 : 0);
                        const float2* const pm = reinterpret_cast<const float2*>(sc.sums + part * 64) + first_col;
                        const float4* const po = reinterpret_cast<const float4*>(sc.out + part * 32 * 128) + mine;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                z[q][nt][k] = there ? __ldcg(&pm[nt * 8 + tq * 2 + k])
                                                    : make_float2(-INFINITY, 0.0f);
#pragma unroll
                            for (int c = 0; c < kOwn; ++c)
                                x[q][c][nt] = there ? __ldcg(&po[((c0 + c) * NT + nt) * 32])
                                                    : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float m = top[nt][k];
#pragma unroll
                            for (int q = 0; q < kBatch; ++q) m = fmaxf(m, z[q][nt][k].x);
                            const float keep = top[nt][k] == -INFINITY ? 0.0f : fast_exp2(top[nt][k] - m);
                            top[nt][k] = m;
                            sum[nt][k] *= keep;
#pragma unroll
                            for (int c = 0; c < kOwn; ++c) {
                                o[c][nt][k] *= keep;
                                o[c][nt][k + 2] *= keep;
                            }
#pragma unroll
                            for (int q = 0; q < kBatch; ++q) {
                                const float2 y = z[q][nt][k];
                                const float f = y.x == -INFINITY ? 0.0f : fast_exp2(y.x - m);
                                sum[nt][k] = fmaf(y.y, f, sum[nt][k]);
#pragma unroll
                                for (int c = 0; c < kOwn; ++c) {
                                    const float4 w = x[q][c][nt];
                                    o[c][nt][k] = fmaf(k ? w.y : w.x, f, o[c][nt][k]);
                                    o[c][nt][k + 2] = fmaf(k ? w.w : w.z, f, o[c][nt][k + 2]);
                                }
                            }
                        }
                }
                write();
            }
        }
        named_barrier_sync(1, 32 * kWarps);
        if (nan) {  // the item's, not the next one's
            for (int i = tid; i < 128; i += 32 * kWarps) sh.nan_at[i] = 0x7FFFFFFF;
            if (tid == 0) sh.nan_any = 0;
            named_barrier_sync(1, 32 * kWarps);
        }
        t = seg.at + end;
    }
}

template <int FORMAT, int D, int NT, int CG>
cudaError_t go(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc, cudaStream_t st)
{
    using S = Sizes<D, NT, CG>;
    // (at every call: it belongs to the device)
    const cudaError_t e = cudaFuncSetAttribute(
        few_kernel<FORMAT, D, NT, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
    if (e != cudaSuccess) return e;
    static_assert(S::kPerSm <= kBlocksPerSm, "room for partial sums");
    return launch_first(few_kernel<FORMAT, D, NT, CG>, sc.sms * S::kPerSm, S::kThreads, S::kBytes, st,
                        sc.kmap, sc.vmap, g, a, sc);
}

template <int FORMAT, int D>
cudaError_t by_columns(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc, int columns,
                       cudaStream_t st)
{
    if (columns <= 8) return go<FORMAT, D, 1, 1>(g, a, sc, st);
    if (columns <= 16) return go<FORMAT, D, 2, 1>(g, a, sc, st);
    return go<FORMAT, D, 2, 2>(g, a, sc, st);
}

}  // namespace

cudaError_t launch_cache_few(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                             int typical, cudaStream_t st)
{
    if (g.format == BACON_E4M3)
        return g.d == 128 ? by_columns<BACON_E4M3, 128>(g, a, sc, typical, st)
                          : by_columns<BACON_E4M3, 64>(g, a, sc, typical, st);
    return g.d == 128 ? by_columns<BACON_INT8, 128>(g, a, sc, typical, st)
                      : by_columns<BACON_INT8, 64>(g, a, sc, typical, st);
}

// Which kernel has which requests, by their rows (queries x query heads of a
// kv-head).  Both on calls of 28 / 4 and 32 / 8 heads of 128, in us, few and
// many:
//   21 rows, 8 x  4096 tokens  27   32        24 rows, 8 x 4096  44   49
//   21 rows, 8 x 32768        111  111        24 rows, 1 x 1024  17   23
//   56 rows, 8 x  4096         74   51        56 rows, 1 x 1024  17   23
// so up to 32 rows, a block of columns, are few.  When the requests ask
// differently, which ones do is known on the device only; each kernel then
// takes its own, and one that has none still costs a launch, one that has some
// the time of its own split and joining.  So a call that has few rows a
// request on average leaves up to 64 with the others (32 requests of 7 to 49
// rows over 1024 tokens: 52, 70 with the cut at 32), and one that has many
// lets only what is close to a single token be few (8 requests of 21 to 49
// rows over 4096: 40, 63 with the cut at 32; 39 now).  Where the rule changes it
// jumps: ragged requests are all few with an average of 32 rows (4 to 60 each;
// 32 of them over 1024 tokens 69 us, 8 over 4096 67) and mostly many with one of
// 36 (4 to 68 each; 109 and 74).
cudaError_t launch_cache_attend(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                                cudaStream_t st)
{
    constexpr int kFew = 32;
    const long long rows = (long long)a.tokens * g.group, each = rows / a.requests;
    AttendArgs few = a, many = a;
    few.above = 0;
    many.upto = 1ll << 62;
    int typical = (int)(each < kFew ? each : kFew);
    if (!a.starts) {
        few.upto = many.above = each <= kFew ? many.upto : 0;
    } else if (each <= kFew) {
        few.upto = many.above = 2 * kFew;
    } else {
        few.upto = many.above = kFew / 2;
        typical = g.group;
    }
    cudaError_t e = cudaSuccess;
    if (few.upto > 0) e = launch_cache_few(g, few, sc, typical, st);
    if (e == cudaSuccess && many.above < rows) e = launch_cache_many(g, many, sc, st);
    return e;
}

}  // namespace bacon
