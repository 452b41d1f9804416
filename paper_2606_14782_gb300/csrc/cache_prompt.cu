// Attention of many queries per unit over the 8-bit pages: a follow-up turn,
// or a prompt over a cache.
//
// Bound by the tensor cores: 4 d flops for every query head and token it sees.
// 4096 queries over 16384 tokens (28 / 4 heads of 128) take 566 us, 1487 TFLOP/s,
// 77 % of the measured burst rate of a library product; 100 queries each of
// three requests over 2000 tokens 31 us, most of it filling, draining and
// joining.
// An item is 256 rows (query x head of the kv-head) of a unit, two 128-row
// tiles of S = Q K^T and O = P V on tcgen05 (fp16 in, fp32 in tensor memory),
// against tiles of 128 tokens.  Codes cannot be operands beside 16-bit
// queries, so four warps turn each page tile into fp16 once for all 256 rows:
// K as it lies, V transposed to [dim][token] by 8x8 matrix loads and stores.
// Two row tiles are what makes that pay: 1024 cycles of products a row tile
// and token tile against some 900 issue slots of softmax and conversion for
// one row tile, 1400 in 2048 for two.
//
// Roles: warps 0-3 and 4-7 take a row tile each, a thread a row: it reads its
// logits from tensor memory, forms the weights w (cache_attend.cuh) and writes
// them over the logits as the second product's operand; warps 8-11 convert;
// one thread issues products, in the order P0 V, Q0 K', P1 V, Q1 K' (K' the
// next tile), so that one row tile's softmax runs beside the other's products;
// one warp loads.  A row's reference M follows its maximum only when that has
// grown by more than 2^8 (published as conditional, or lazy, rescaling of a
// running softmax); only then O is scaled, in tensor memory, which is idle for
// this row tile while its softmax runs.  The largest weight therefore lies
// between 2^7 and 2^15, and a weight is fp16's normal value down to 2^-21 of it
// at least, less and less exact below, and may be 0 from 2^-32 on: of n tokens
// that small, n 2^-32 of the largest weight's share can be lost.  The roles'
// code runs at the same time and shares the instruction cache: what runs once an
// item or on its last tiles only is rolled (555 us for 647 with straight-line
// code there).
//
// Tiles are dealt out and cut items joined as in cache_attend.cu.
#include <cmath>

#include "cache_attend.cuh"

namespace bacon {
namespace {

using namespace tc;

constexpr int kRows = 256;   // of an item
constexpr int kHalf = 128;   // rows of a row tile
constexpr int kTile = 128;   // tokens
constexpr int kGroups = kTile / 16;
constexpr int kValueWarp = 8, kKeyWarp = 12, kIssueWarp = 14;  // first of each role; the loads are last
constexpr int kThreads = 16 * 32;
// Registers of the softmax's threads and of the others, out of 128 a thread at
// launch: 256 x 184 + 256 x 72 = 512 x 128.
constexpr int kSoftmaxRegs = 184, kOtherRegs = 72;
static_assert(256 * (kSoftmaxRegs + kOtherRegs) <= kThreads * 128, "register split");
// A row's reference follows its maximum when that has grown by 2^kSlack, with
// the largest weight at 2^kTop then: below fp16's 2^16 in between.
constexpr float kSlack = 8.0f, kTop = 7.0f;

template <int D>
struct Smem {
    static constexpr int kPanel = 128 * 128;         // 64 fp16 columns of 128 rows
    static constexpr int kQHalf = kHalf * D * 2;
    static constexpr int kKeys = 2 * kQHalf;         // two tiles of K in fp16
    static constexpr int kKeysTile = kTile * D * 2;
    static constexpr int kValues = kKeys + 2 * kKeysTile;  // two of V, [dim][token]
    static constexpr int kValuesTile = D * kTile * 2;
    static constexpr int kRawK = kValues + 2 * kValuesTile;
    static constexpr int kRawV = kRawK + kTile * D;
    static constexpr int kShared = kRawV + kTile * D;
    static constexpr int kBytes = kShared + 3072;
};

// Tiles [begin, end) of an item, whose first tile is tile `at` of the call.
struct Segment {
    Item it;
    int begin, end;
    long long at;
};
// The loads are at most this many items ahead of the outputs.
constexpr int kItems = 2;

template <int D>
struct Shared {
    float k_scale[4][kGroups], v_log2[4][kGroups], v_inv[4][kGroups];
    uint64_t rawk_full, rawk_empty, rawv_full, rawv_empty;
    uint64_t key_full[2], key_empty[2], value_full[2], value_empty[2];
    uint64_t s_full[2], p_full[2][2], o_full[2], q_full[2];
    uint64_t meta_full[4], item_full[kItems], item_done[kItems], drain;
    Segment seg[kItems];
    long long scan[kThreads / 32];
    Found found;
    Place place;
    uint32_t tmem;
    int abort, last[2], quit[2];
    int nan_any[kItems];
    int nan_at[kItems][D];  // of an item, per dim: first position of a NaN of V that not every row sees
};
static_assert(sizeof(Shared<128>) <= 3072, "shared record");

__device__ __forceinline__ uint32_t bar(uint64_t& b) { return smem_u32(&b); }

// 8x8 matrices of 16-bit elements to shared memory, a row address a lane.
__device__ __forceinline__ void stmatrix4(uint32_t addr, const uint32_t* r)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};\n" ::"r"(addr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
                 : "memory");
}

__host__ __device__ constexpr uint32_t idesc_f16(int M, int N)
{
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// D[tmem] (+)= A[tmem] * B[smem]^T
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi,
                                        uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 db;\n setp.ne.b32 p, %5, 0;\n mov.b64 db, {%2, %3};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}\n" ::"r"(d),
        "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}

template <int D>
__device__ __forceinline__ void give_up(Shared<D>& sh, int* err)
{
    st_shared_volatile(smem_u32(&sh.abort), 1);
    atomicCAS(err, 0, kCacheTimeout);
}

// Bounded wait of a role's thread: one that runs out raises the abort flag, at
// which every other wait that is not over yet ends at once.  The roles then run
// through the item that they have (a warpgroup's named barriers need all its
// warps) and leave before the next.
template <int D>
__device__ __forceinline__ bool wait(Shared<D>& sh, uint32_t b, uint32_t parity, int* err)
{
    if (mbar_wait(b, parity, smem_u32(&sh.abort))) return true;
    give_up(sh, err);
    return false;
}
// The same with one answer for a whole warp, whose lanes need not run out of
// time at once, where they go on together: those left would wait at the next
// warp barrier for good.  (The long turn takes 563 us with it, 558 without.)
template <int D>
__device__ __forceinline__ bool wait_all(Shared<D>& sh, uint32_t b, uint32_t parity, int* err)
{
    return __all_sync(0xFFFFFFFFu, wait(sh, b, parity, err));
}

// ------------------------------------------------------------------ loads

template <int D>
__device__ __forceinline__ void load(const CUtensorMap* kmap, const CUtensorMap* vmap,
                                     const CacheGeom& g, const AttendArgs& a, const Place& p,
                                     Shared<D>& sh, uint32_t base)
{
    using S = Smem<D>;
    const int lane = threadIdx.x & 31, group = lane & 7;
    const bool of_v = lane >= 8;
    int unit = p.unit, k = 0;
    bool ok = true;
    Item it = sh.found.it;
    long long at = p.at, t = p.lo;
    uint32_t seq = 0, more = 0;  // tiles asked for; one more whose K alone is
    while (t < p.hi && ok) {
        // (after giving up the softmax frees items that are not done)
        ok = wait_all(sh, bar(sh.item_done[k % kItems]), (k / kItems & 1) ^ 1, g.err) &&
             __all_sync(0xFFFFFFFFu, !ld_shared_volatile(smem_u32(&sh.abort)));
        if (!ok) break;
        for (int i = lane; i < D; i += 32) sh.nan_at[k % kItems][i] = 0x7FFFFFFF;
        const int end = (int)min((long long)it.tiles, p.hi - at);
        if (lane == 0) {
            sh.nan_any[k % kItems] = 0;
            sh.seg[k % kItems] = Segment{it, (int)(t - at), end, at};
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(sh.item_full[k % kItems]));
        const int32_t* const table =
            a.table + (((size_t)it.r * g.layers + a.layer) * g.hkv + it.h) * g.max_blocks;
        for (int i = (int)(t - at); i < end && ok; ++i, ++t, ++seq) {
            const int pos = i * kTile + group * 16;
            const bool live = lane < 16 && pos < it.seen;
            int page = 0;
            if (live) {
                page = table[pos >> g.page_log2];
                if (page < 0 || page >= g.pages) {
                    atomicCAS(g.err, 0, kCacheBadIndex);
                    page = 0;
                }
            }
            const int row = (page << g.page_log2) + (pos & (g.page - 1));
            const int boxes = __popc(__ballot_sync(0xFFFFFFFFu, live && !of_v));
            const uint32_t parity = (seq & 1) ^ 1;
            ok = wait_all(sh, bar(sh.rawk_empty), parity, g.err);
            if (!ok) break;
            if (lane == 0 && boxes) mbar_expect_tx(bar(sh.rawk_full), boxes * kBoxRows * D);
            __syncwarp();
            if (live && !of_v && !(a.fault && blockIdx.x == 0 && (int)seq == a.fault - 1 && lane == 0))
                load_rows(base + S::kRawK + group * 16 * D, kmap, row, bar(sh.rawk_full));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.rawk_full));
            const int slot = seq & 3;
            if (lane < 16) {
                const float s = live ? (of_v ? g.v_scale : g.k_scale)[page] : 1.0f;
                if (of_v) {
                    sh.v_log2[slot][group] = log2f(s);
                    sh.v_inv[slot][group] = 1.0f / s;
                } else {
                    sh.k_scale[slot][group] = s;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.meta_full[slot]));
            ok = wait_all(sh, bar(sh.rawv_empty), parity, g.err);
            if (!ok) {
                more = 1;
                break;
            }
            if (lane == 0 && boxes) mbar_expect_tx(bar(sh.rawv_full), boxes * kBoxRows * D);
            __syncwarp();
            if (live && of_v) load_rows(base + S::kRawV + group * 16 * D, vmap, row, bar(sh.rawv_full));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.rawv_full));
        }
        at += it.tiles;
        ++k;
        if (t < p.hi && ok && !next_item<kRows, kTile>(g, a, unit, it)) break;
    }
    // The block's copies end before it does, also when those who waited for them
    // have given up after the last was asked for.
    if (seq + more) mbar_wait(bar(sh.rawk_full), (seq + more - 1) & 1, 0);
    if (seq) mbar_wait(bar(sh.rawv_full), (seq - 1) & 1, 0);
}

// -------------------------------------------------------------- conversion

// K: a row of the tile a lane, 16 codes at a time.
template <int FORMAT, int D>
__device__ __forceinline__ void convert_keys(const CacheGeom& g, const Place& p, Shared<D>& sh,
                                             uint8_t* smem)
{
    using S = Smem<D>;
    constexpr int kChunks = D / 16;
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - kKeyWarp;
    const uint32_t tiles = (uint32_t)(p.hi - p.lo);
    for (uint32_t seq = 0; seq < tiles; ++seq) {
        const int buf = seq & 1;
        if (!wait_all(sh, bar(sh.rawk_full), seq & 1, g.err) ||
            !wait_all(sh, bar(sh.key_empty[buf]), (seq >> 1 & 1) ^ 1, g.err))
            return;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = warp * 64 + half * 32 + lane;
            const uint32_t swizzle = D == 128 ? row & 7 : row >> 1 & 3;
            const uint8_t* const src = smem + S::kRawK + row * D;
            uint8_t* const dst = smem + S::kKeys + buf * S::kKeysTile + row * 128;
#pragma unroll
            for (int c0 = 0; c0 < kChunks; c0 += 4) {
                uint4 w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    w[c] = *reinterpret_cast<const uint4*>(src + (((c0 + c) ^ swizzle) << 4));
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint4 x, y;
                    codes_half<FORMAT>(w[c].x, x.x, x.y);
                    codes_half<FORMAT>(w[c].y, x.z, x.w);
                    codes_half<FORMAT>(w[c].z, y.x, y.y);
                    codes_half<FORMAT>(w[c].w, y.z, y.w);
                    uint8_t* const panel = dst + (c0 >> 2) * S::kPanel;
                    *reinterpret_cast<uint4*>(panel + (((2 * c) ^ (row & 7)) << 4)) = x;
                    *reinterpret_cast<uint4*>(panel + (((2 * c + 1) ^ (row & 7)) << 4)) = y;
                }
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(bar(sh.key_full[buf]));
            mbar_arrive(bar(sh.rawk_empty));
        }
    }
}

// V: 16 tokens x 32 dims at a time; row n of a chunk's 16 in the transposed
// tile is dim 2 n for n < 8, 2 (n - 8) + 1 above.  CUT: some row of the item
// does not see some token of the tile, so rows that no one sees are cleared (a
// page holds anything there) and so is a NaN, which is put back at the item's
// end in the rows that see it.
template <int FORMAT, int D, bool CUT>
__device__ __forceinline__ void convert_value_tile(Shared<D>& sh, uint32_t base, int buf, int pos,
                                                   int seen, int item)
{
    using S = Smem<D>;
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - kValueWarp;
    const int gr = lane >> 2, tq = lane & 3;
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
        const int group = warp * 2 + half;
        const int mrow = group * 16 + (lane & 7) + (lane >> 3 & 1) * 8;
        const uint32_t swizzle = D == 128 ? mrow & 7 : mrow >> 1 & 3;
        const uint32_t src = base + S::kRawV + mrow * D;
        // row n0 and chunk of tokens of the transposed tile's panel of 64 tokens
        const int n0 = (lane >> 3 & 1) * 8 + (lane & 7);
        const int chunk = (group & 3) * 2 + (lane >> 4);
        const uint32_t dst = base + S::kValues + buf * S::kValuesTile + (group >> 2) * (D * 128) +
                             n0 * 128 + ((chunk ^ (n0 & 7)) << 4);
        // (loads together where nothing is cut; cut tiles are few, and their
        // loop is rolled to be fetched at once)
        constexpr int kTogether = CUT ? 1 : D / 32;
#pragma unroll 1
        for (int c0 = 0; c0 < D / 32; c0 += kTogether) {
            uint32_t w[kTogether][4];
#pragma unroll
            for (int z = 0; z < kTogether; ++z)
                ldmatrix4_trans(w[z], src + (((2 * (c0 + z) + (lane >> 4)) ^ swizzle) << 4));
#pragma unroll
            for (int z = 0; z < kTogether; ++z) {
                const int c = c0 + z;
                uint32_t f[8];
                if (CUT) {
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const int x0 = pos + group * 16 + (m & 1) * 8 + 2 * tq;
                        if (x0 >= seen) w[z][m] &= 0xFFFF0000u;
                        if (x0 + 1 >= seen) w[z][m] &= 0x0000FFFFu;
                        if (FORMAT == BACON_E4M3 && (((w[z][m] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u)) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if ((w[z][m] >> (8 * e) & 0x7Fu) == 0x7Fu) {
                                    w[z][m] &= ~(0xFFu << (8 * e));
                                    atomicMin(&sh.nan_at[item % kItems][(2 * c + (m >> 1)) * 16 + 2 * gr + (e & 1)],
                                              x0 + (e >> 1));
                                    sh.nan_any[item % kItems] = 1;
                                }
                        }
                    }
                }
                pairs_half<FORMAT>(w[z][0], f[0], f[1]);
                pairs_half<FORMAT>(w[z][1], f[2], f[3]);
                pairs_half<FORMAT>(w[z][2], f[4], f[5]);
                pairs_half<FORMAT>(w[z][3], f[6], f[7]);
                stmatrix4(dst + c * 32 * 128, f);
                stmatrix4(dst + (c * 32 + 16) * 128, f + 4);
            }
        }
    }
}

template <int FORMAT, int D>
__device__ __forceinline__ void convert_values(const CacheGeom& g, const AttendArgs& a, const Place& p,
                                               Shared<D>& sh, uint32_t base)
{
    const int lane = threadIdx.x & 31;
    const uint32_t tiles = (uint32_t)(p.hi - p.lo);
    uint32_t seq = 0;
    for (int k = 0; seq < tiles; ++k) {
        if (!wait_all(sh, bar(sh.item_full[k % kItems]), k / kItems & 1, g.err)) return;
        const Segment& seg = sh.seg[k % kItems];
        const int all = seen_by(a, seg.it.n, seg.it.asked, seg.it.block * kRows / g.group);
        const int end = seg.end, seen = seg.it.seen;
        for (int i = seg.begin; i < end; ++i, ++seq) {
            const int buf = seq & 1;
            if (!wait_all(sh, bar(sh.rawv_full), seq & 1, g.err) ||
                !wait_all(sh, bar(sh.value_empty[buf]), (seq >> 1 & 1) ^ 1, g.err))
                return;
            if ((i + 1) * kTile > all)
                convert_value_tile<FORMAT, D, true>(sh, base, buf, i * kTile, seen, k);
            else
                convert_value_tile<FORMAT, D, false>(sh, base, buf, i * kTile, seen, k);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar(sh.value_full[buf]));
                mbar_arrive(bar(sh.rawv_empty));
            }
        }
    }
}

// ---------------------------------------------------------------- products

// Row tiles of an item.
__device__ __forceinline__ int halves_of(const CacheGeom& g, const Item& it)
{
    return (long long)it.asked * g.group - (long long)it.block * kRows > kHalf ? 2 : 1;
}

template <int D>
__device__ __forceinline__ void issue(const CacheGeom& g, const Place& p, Shared<D>& sh, uint32_t base)
{
    using S = Smem<D>;
    const bool leader = elect_one();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, ld_shared(smem_u32(&sh.tmem)), 0);
    constexpr uint32_t hi = sdesc_hi(1024u);
    const uint32_t q_lo = sdesc_lo(base), k_lo = sdesc_lo(base + S::kKeys), v_lo = sdesc_lo(base + S::kValues);
    bool ok = true;
    const uint32_t every = (uint32_t)(p.hi - p.lo);
    uint32_t seq = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};

    auto scores = [&](int m, uint32_t s) {
        if (leader) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t step = (kk / 4) * (S::kPanel >> 4) + (kk % 4) * 2u;
                umma_bf16(tmem + m * 128, q_lo + m * (S::kQHalf >> 4) + step, hi,
                          k_lo + (s & 1) * (S::kKeysTile >> 4) + step, hi, idesc_f16(kHalf, kTile), kk > 0);
            }
            umma_commit(bar(sh.s_full[m]));
        }
    };
    for (int k = 0; seq < every && ok; ++k) {
        ok = wait(sh, bar(sh.item_full[k % kItems]), k / kItems & 1, g.err);
        if (!ok) break;
        const Segment& seg = sh.seg[k % kItems];
        const int halves = halves_of(g, seg.it), tiles = seg.end - seg.begin;
        for (int m = 0; m < halves && ok; ++m) {
            ok = wait(sh, bar(sh.q_full[m]), q_phase[m], g.err);
            q_phase[m] ^= 1;
        }
        ok = ok && wait(sh, bar(sh.key_full[seq & 1]), seq >> 1 & 1, g.err);
        if (!ok) break;
        fence_after_sync();
        for (int m = 0; m < halves; ++m) scores(m, seq);
        if (leader) umma_commit(bar(sh.key_empty[seq & 1]));
        for (int i = 0; i < tiles && ok; ++i, ++seq) {
            for (int m = 0; m < halves && ok; ++m) {
                // what is there long before the weights is waited for first
                if (m == 0) ok = wait(sh, bar(sh.value_full[seq & 1]), seq >> 1 & 1, g.err);
                if (m == 0 && i + 1 < tiles)
                    ok = ok && wait(sh, bar(sh.key_full[(seq + 1) & 1]), (seq + 1) >> 1 & 1, g.err);
                // the weights of the first and of the second 64 tokens
                for (int h = 0; h < 2 && ok; ++h) {
                    ok = wait(sh, bar(sh.p_full[m][h]), p_phase[m], g.err);
                    if (!ok) break;
                    fence_after_sync();
                    if (leader) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            umma_ts(tmem + 256 + m * 128, tmem + m * 128 + h * 32 + kk * 8,
                                    v_lo + (seq & 1) * (S::kValuesTile >> 4) + h * (D * 128 >> 4) + kk * 2u,
                                    hi, idesc_f16(kHalf, D), i > 0 || h > 0 || kk > 0);
                    }
                }
                p_phase[m] ^= 1;
                if (!ok) break;
                if (leader) {
                    if (m == halves - 1) umma_commit(bar(sh.value_empty[seq & 1]));
                    if (i == tiles - 1) umma_commit(bar(sh.o_full[m]));
                }
                if (i + 1 < tiles) {
                    scores(m, seq + 1);
                    if (leader && m == halves - 1) umma_commit(bar(sh.key_empty[(seq + 1) & 1]));
                }
            }
        }
    }
    // every product issued ends before tensor memory is given back
    if (leader) {
        umma_commit(bar(sh.drain));
        mbar_wait(bar(sh.drain), 0, 0);
    }
    __syncwarp();
}

// ----------------------------------------------------------------- softmax

// Largest of 16 values.
__device__ __forceinline__ float max16(const float* v)
{
    const float a = max3(v[0], v[1], v[2]), b = max3(v[3], v[4], v[5]), c = max3(v[6], v[7], v[8]);
    const float d = max3(v[9], v[10], v[11]), e = max3(v[12], v[13], v[14]);
    return max3(max3(a, b, c), max3(d, e, v[15]), v[15]);
}

// The row's reference follows its maximum `high` when that has grown; `scaled`:
// O holds sums that follow it too.
template <int D>
__device__ __forceinline__ void follow(float high, bool scaled, uint32_t out, float& top, float& sum)
{
    const bool grew = high > top + kSlack;
    if (!__any_sync(0xFFFFFFFFu, grew)) return;
    const float keep = grew ? fast_exp2(top - high) : 1.0f;
    if (grew) top = high;
    sum *= keep;
    if (scaled) {
#pragma unroll
        for (int q = 0; q < D / 16; ++q) {
            float o[16];
            tmem_ld16(out + q * 16, o);
            tmem_ld_wait_regs16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= keep;
            tmem_st8(out + q * 16, o);
            tmem_st8(out + q * 16 + 8, o + 8);
        }
    }
}

// One tile of a row's logits, all of which it sees, into weights.
template <int D>
__device__ __forceinline__ void softmax_tile(Shared<D>& sh, int m, uint32_t slot, uint32_t logits,
                                             uint32_t out, bool scaled, float factor, float& top, float& sum)
{
    const int lane = threadIdx.x & 31;
    float v[128], high = -INFINITY;
#pragma unroll
    for (int q = 0; q < 4; ++q) tmem_ld32(logits + q * 32, v + q * 32);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        tmem_ld_wait_regs32(v + q * 32);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int grp = q * 2 + h;
            const float x = max16(v + grp * 16);
            high = fmaxf(high, fmaf(x, factor * sh.k_scale[slot][grp], sh.v_log2[slot][grp]));
        }
    }
    follow<D>(high, scaled, out, top, sum);
    const float ref = top == -INFINITY ? 0.0f : top - kTop;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int grp = half * 4 + h;
            float w[8];
            const float f = factor * sh.k_scale[slot][grp], b = sh.v_log2[slot][grp] - ref;
            const unsigned long long f2 = pack2(f, f), b2 = pack2(b, b);
            unsigned long long part = pack2(0.0f, 0.0f);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float* const x = v + grp * 16 + e;
                float2 y = unpack2(fma2(pack2(x[0], x[1]), f2, b2));
                y.x = fast_exp2(y.x);
                y.y = fast_exp2(y.y);
                part = add2(part, pack2(y.x, y.y));
                w[e / 2] = __uint_as_float(half2_of(y.x, y.y));
            }
            const float2 y = unpack2(part);
            sum = fmaf(y.x + y.y, sh.v_inv[slot][grp], sum);
            // over the logits: 16 tokens' weights in 8 columns
            tmem_st8(logits + grp * 8, w);
        }
        tmem_st_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(sh.p_full[m][half]));
    }
}

// The same for a tile of which the row sees the first `left` tokens (all, with
// left >= 128).  An item has two or three such tiles, so the loops are rolled:
// fetching straight-line code once would cost more than running it.
template <int D>
__device__ __forceinline__ void softmax_cut_tile(Shared<D>& sh, int m, uint32_t slot, uint32_t logits,
                                                 uint32_t out, bool scaled, int left, float factor,
                                                 float& top, float& sum)
{
    const int lane = threadIdx.x & 31;
    float high = -INFINITY;
#pragma unroll 1
    for (int grp = 0; grp < kGroups; ++grp) {
        float v[16];
        tmem_ld16(logits + grp * 16, v);
        tmem_ld_wait_regs16(v);
        const int some = left - grp * 16;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (e >= some) v[e] = -INFINITY;
        const float x = max16(v);
        // (a factor that underflows would make -inf a NaN)
        if (x != -INFINITY) high = fmaxf(high, fmaf(x, factor * sh.k_scale[slot][grp], sh.v_log2[slot][grp]));
    }
    follow<D>(high, scaled, out, top, sum);
    const float ref = top == -INFINITY ? 0.0f : top - kTop;
#pragma unroll 1
    for (int grp = 0; grp < kGroups; ++grp) {
        float v[16], w[8], part = 0.0f;
        tmem_ld16(logits + grp * 16, v);
        tmem_ld_wait_regs16(v);
        const int some = left - grp * 16;
        const float f = factor * sh.k_scale[slot][grp], b = sh.v_log2[slot][grp] - ref;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            v[e] = e < some ? fast_exp2(fmaf(v[e], f, b)) : 0.0f;
            part += v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __uint_as_float(half2_of(v[2 * e], v[2 * e + 1]));
        sum = fmaf(part, sh.v_inv[slot][grp], sum);
        tmem_st8(logits + grp * 8, w);
        if ((grp & 3) == 3) {
            tmem_st_wait();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.p_full[m][grp >> 2]));
        }
    }
}

// Four dims of a row of a part, rows side by side.
__device__ __forceinline__ float4& part_of(const SplitScratch& sc, size_t slot, int quad, int row)
{
    return reinterpret_cast<float4*>(sc.many_out)[slot * 32 + quad * kHalf + row];
}

// 32 columns of a row of O, column 16 c + 8 o + n being dim 16 c + 2 n + o, as
// the output's values.
__device__ __forceinline__ void store_row(uint16_t* dst, const float* v, float scale, bool some, int dtype)
{
    uint32_t w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int z = (e & 8) * 2 + (e & 7);
        w[e] = some ? pack16(dtype, v[z] * scale, v[z + 8] * scale) : 0u;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        *reinterpret_cast<uint4*>(dst + e * 8) =
            make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
}

template <int FORMAT, int D>
__device__ __forceinline__ void softmax(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                                        const Place& p, Shared<D>& sh, uint8_t* smem)
{
    using S = Smem<D>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, m = warp >> 2;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lanes = ld_shared(smem_u32(&sh.tmem)) + ((uint32_t)(warp & 3) << 21);
    const uint32_t logits = lanes + m * 128, out = lanes + 256 + m * 128;
    const uint32_t tiles = (uint32_t)(p.hi - p.lo);
    uint32_t seq = 0, s_phase = 0, o_phase = 0;

    for (int k = 0; seq < tiles; ++k) {
        const bool there = wait(sh, bar(sh.item_full[k % kItems]), k / kItems & 1, g.err);
        if (row == 0) sh.quit[m] = !there || ld_shared_volatile(smem_u32(&sh.abort));
        named_barrier_sync(1 + m, kHalf);
        if (sh.quit[m]) return;  // the same for the warpgroup's threads
        const Segment& seg = sh.seg[k % kItems];
        const Item& it = seg.it;
        const int begin = seg.begin, end = seg.end;
        const long long c = (long long)it.block * kRows + m * kHalf + row;
        if (m < halves_of(g, it)) {
            const int j = (int)(c / g.group), head = it.h * g.group + (int)(c % g.group);
            const bool mine = j < it.asked;
            const int sees = mine ? seen_by(a, it.n, it.asked, j) : 0;
            const bool live = __any_sync(0xFFFFFFFFu, mine);  // else the warp only keeps time
            const int all = seen_by(a, it.n, it.asked, (it.block * kRows + m * kHalf) / g.group);
            // the rows' queries as fp16, each scaled into its range: D / 8
            // lanes a row
            float factor = 1.0f;
            {
                constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
                const long long offset = mine ? (long long)(it.start + j) * a.q_token_stride +
                                                    head * a.q_head_stride
                                              : -1;
                const int piece = lane % kLanes;
                // (a rolled loop: straight-line code that runs once an item
                // costs more in instruction fetches than it does)
#pragma unroll 1
                for (int i0 = 0; i0 < kLanes; i0 += 8) {
                    uint4 raw[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const long long from =
                            __shfl_sync(0xFFFFFFFFu, offset, (i0 + i) * kAtOnce + lane / kLanes);
                        raw[i] = make_uint4(0, 0, 0, 0);
                        if (from >= 0) raw[i] = *reinterpret_cast<const uint4*>(a.q + from + piece * 8);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                        float2 v[4];
                        float amax = 0.0f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[e] = unpack16(g.dtype, w[e]);
                            amax = max3(amax, fabsf(v[e].x), fabsf(v[e].y));
                        }
#pragma unroll
                        for (int o = 1; o < kLanes; o <<= 1)
                            amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
                        float back;
                        const float up = query_scale(amax, back);
                        const int r = (i0 + i) * kAtOnce;
#pragma unroll
                        for (int z = 0; z < kAtOnce; ++z) {
                            const float f = __shfl_sync(0xFFFFFFFFu, back, z * kLanes);
                            if (lane == r + z) factor = f;
                        }
                        const int to = (warp & 3) * 32 + r + lane / kLanes;
                        *reinterpret_cast<uint4*>(smem + m * S::kQHalf + (piece >> 3) * S::kPanel +
                                                  to * 128 + (((piece & 7) ^ (to & 7)) << 4)) =
                            make_uint4(half2_of(v[0].x * up, v[0].y * up),
                                       half2_of(v[1].x * up, v[1].y * up),
                                       half2_of(v[2].x * up, v[2].y * up),
                                       half2_of(v[3].x * up, v[3].y * up));
                    }
                }
                factor *= a.scale * kLog2e;
            }
            fence_proxy_async_smem();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.q_full[m]));

            float top = -INFINITY, sum = 0.0f;
            // the tile's logits are there
            auto arrived = [&](int i) {
                const uint32_t s = seq + (i - begin);
                wait(sh, bar(sh.meta_full[s & 3]), s >> 2 & 1, g.err);
                wait(sh, bar(sh.s_full[m]), s_phase, g.err);
                s_phase ^= 1;
                fence_after_sync();
                return s & 3;
            };
            int i = begin;
            if (!live) {
                for (; i < end; ++i) {
                    arrived(i);
                    if (lane < 2) mbar_arrive(bar(sh.p_full[m][lane]));
                }
            }
            for (const int full = min(end, all / kTile); i < full; ++i)
                softmax_tile<D>(sh, m, arrived(i), logits, out, i > begin, factor, top, sum);
            for (; i < end; ++i)
                softmax_cut_tile<D>(sh, m, arrived(i), logits, out, i > begin, sees - i * kTile, factor, top, sum);

            // ------------------------------------------------- outputs
            wait(sh, bar(sh.o_full[m]), o_phase, g.err);
            o_phase ^= 1;
            fence_after_sync();
            const bool whole = begin == 0 && end == it.tiles;
            const bool nan = sh.nan_any[k % kItems] != 0;
            const size_t orow = (size_t)(it.start + j) * g.hq + head;
            uint16_t* const dst = a.out + orow * D;
            const int b = blockIdx.x;
            const size_t slot = ((2 * (size_t)b + (begin == 0 ? 1 : 0)) * 2 + m) * kHalf;
            const float inv = sees > 0 ? 1.0f / sum : 0.0f;
#pragma unroll 1
            for (int q = 0; live && q < D / 32; ++q) {
                float v[32];
                tmem_ld32(out + q * 32, v);
                tmem_ld_wait_regs32(v);
                if (nan) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)  // column 16 c + 8 o + n is dim 16 c + 2 n + o
                        if (sh.nan_at[k % kItems][q * 32 + (e & 16) + (e & 7) * 2 + (e >> 3 & 1)] < sees) v[e] = NAN;
                }
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        part_of(sc, slot, q * 8 + e / 4, row) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                } else if (mine) {
                    store_row(dst + q * 32, v, inv, sees > 0, g.dtype);
                }
            }
            if (whole) {
                if (mine && a.lse)
                    a.lse[orow] = sees > 0 ? (log2f(sum) + (top - kTop)) * kLn2 : -INFINITY;
            } else {
                sc.many_sums[slot + row] = make_float2(top, sum);
                int first, parts;
                p.parts_of(seg.at, it.tiles, first, parts);
                named_barrier_sync(1 + m, kHalf);
                if (row == 0) sh.last[m] = arrive_last(&sc.many_arrived[first * 2 + m], parts);
                named_barrier_sync(1 + m, kHalf);
                if (sh.last[m]) {
                    auto part = [&](int q) { return ((2 * (size_t)(first + q) + (q == 0 ? 1 : 0)) * 2 + m) * kHalf; };
                    float high = -INFINITY, total = 0.0f;
#pragma unroll 8
                    for (int q = 0; q < parts; ++q) high = fmaxf(high, __ldcg(&sc.many_sums[part(q) + row]).x);
#pragma unroll 8
                    for (int q = 0; q < parts; ++q) {
                        const float2 z = __ldcg(&sc.many_sums[part(q) + row]);
                        total += z.y * (z.x == -INFINITY ? 0.0f : fast_exp2(z.x - high));
                    }
                    const float scale = sees > 0 ? 1.0f / total : 0.0f;
                    // 32 dims at a time, out of two parts at a time
#pragma unroll 1
                    for (int d = 0; live && d < D / 32; ++d) {
                        float v[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0.0f;
#pragma unroll 1
                        for (int q0 = 0; q0 < parts; q0 += 2) {
                            float f[2];
                            float4 x[2][8];
#pragma unroll
                            for (int z = 0; z < 2; ++z) {
                                const bool there = q0 + z < parts;
                                f[z] = there ? __ldcg(&sc.many_sums[part(q0 + z) + row]).x : -INFINITY;
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    x[z][e] = there ? __ldcg(&part_of(sc, part(q0 + z), d * 8 + e, row))
                                                    : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                            }
#pragma unroll
                            for (int z = 0; z < 2; ++z) {
                                const float w = f[z] == -INFINITY ? 0.0f : fast_exp2(f[z] - high);
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    v[4 * e] = fmaf(x[z][e].x, w, v[4 * e]);
                                    v[4 * e + 1] = fmaf(x[z][e].y, w, v[4 * e + 1]);
                                    v[4 * e + 2] = fmaf(x[z][e].z, w, v[4 * e + 2]);
                                    v[4 * e + 3] = fmaf(x[z][e].w, w, v[4 * e + 3]);
                                }
                            }
                        }
                        if (mine) store_row(dst + d * 32, v, scale, sees > 0, g.dtype);
                    }
                    if (mine && a.lse)
                        a.lse[orow] = sees > 0 ? (log2f(total) + (high - kTop)) * kLn2 : -INFINITY;
                }
            }
        }
        seq += end - begin;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(sh.item_done[k % kItems]));
    }
}

template <int FORMAT, int D>
__global__ void __launch_bounds__(kThreads, 1)
many_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
            CacheGeom g, AttendArgs a, SplitScratch sc)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared<D>& sh = *reinterpret_cast<Shared<D>*>(smem + Smem<D>::kShared);
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (uint64_t* b : {&sh.rawk_full, &sh.rawv_full, &sh.drain}) mbar_init(smem_u32(b), 1);
        mbar_init(bar(sh.rawk_empty), kIssueWarp - kKeyWarp);
        mbar_init(bar(sh.rawv_empty), kKeyWarp - kValueWarp);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(sh.key_full[i]), kIssueWarp - kKeyWarp);
            mbar_init(bar(sh.value_full[i]), kKeyWarp - kValueWarp);
            mbar_init(bar(sh.key_empty[i]), 1);
            mbar_init(bar(sh.value_empty[i]), 1);
            mbar_init(bar(sh.s_full[i]), 1);
            mbar_init(bar(sh.o_full[i]), 1);
            mbar_init(bar(sh.p_full[i][0]), 4);
            mbar_init(bar(sh.p_full[i][1]), 4);
            mbar_init(bar(sh.q_full[i]), 4);
        }
        for (int i = 0; i < 4; ++i) mbar_init(bar(sh.meta_full[i]), 1);
        for (int i = 0; i < kItems; ++i) {
            mbar_init(bar(sh.item_full[i]), 1);
            mbar_init(bar(sh.item_done[i]), kValueWarp);
        }
        fence_barrier_init();
        sh.abort = 0;
    }
    {
        Place p;
        if (!find_place<kRows, kTile, kThreads, 2>(g, a, sh.scan, sh.found, p)) return;
        if (threadIdx.x == 0) sh.place = p;
    }
    const Place& p = sh.place;
    if (warp == kIssueWarp) {
        tmem_alloc(smem_u32(&sh.tmem), 512);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t base = smem_u32(smem);
    if (warp < kValueWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kSoftmaxRegs));
        softmax<FORMAT, D>(g, a, sc, p, sh, smem);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kOtherRegs));
        if (warp < kKeyWarp)
            convert_values<FORMAT, D>(g, a, p, sh, base);
        else if (warp < kIssueWarp)
            convert_keys<FORMAT, D>(g, p, sh, smem);
        else if (warp == kIssueWarp)
            issue<D>(g, p, sh, base);
        else
            load<D>(&kmap, &vmap, g, a, p, sh, base);
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == kIssueWarp) tmem_dealloc(ld_shared(smem_u32(&sh.tmem)), 512);
}

template <int FORMAT, int D>
cudaError_t go(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc, cudaStream_t st)
{
    constexpr int bytes = Smem<D>::kBytes;
    // (at every call: it belongs to the device)
    const cudaError_t e = cudaFuncSetAttribute(
        many_kernel<FORMAT, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    return launch_first(many_kernel<FORMAT, D>, sc.sms, kThreads, bytes, st, sc.kmap, sc.vmap, g, a, sc);
}

}  // namespace

cudaError_t launch_cache_many(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                              cudaStream_t st)
{
    if (g.format == BACON_E4M3)
        return g.d == 128 ? go<BACON_E4M3, 128>(g, a, sc, st) : go<BACON_E4M3, 64>(g, a, sc, st);
    return g.d == 128 ? go<BACON_INT8, 128>(g, a, sc, st) : go<BACON_INT8, 64>(g, a, sc, st);
}

}  // namespace bacon
