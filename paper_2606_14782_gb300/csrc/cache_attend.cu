// Attention of few queries per unit over the 8-bit pages: a decoding step, or
// a few drafted tokens.
//
// Bound by the pages' bytes: a token of a unit is 2 d bytes for 4 d flops a
// query head, so with up to 32 columns (query heads of the kv-head x queries)
// the work is a stream through HBM with two small matrix products beside it.
// The products are warp-level (m16n8k16, fp16 in, fp32 sums) with the tokens
// as rows and the columns as n, so that no more than the next 8 columns are
// padded: S^T = K Q^T, then O^T = V^T P^T.  K and V codes go from shared
// memory to fragments by 8x8 matrix loads whose 16-bit elements are two codes
// (V's transposed ones bring two tokens' codes of two dims into a register),
// and become fp16 there; what order the dims take inside a product is the
// same for Q's fragments.  S^T turns into P^T's operand by 8x8 transposes.
//
// The call's tiles of 64 tokens are dealt out evenly: block b of E takes tiles
// [T b / E, T (b + 1) / E) of the items one after the other, an item being 8 NT
// columns of a unit, whatever the units' lengths.  Every block finds its place
// by a scan of the lengths, so no host synchronisation and no second launch
// come before; a warp of it loads (16 rows a TMA load, only rows that the item
// sees), four compute, each 16 tokens of a tile with its own running maximum,
// and join at the item's end.  An item cut by a block's edge leaves partial
// sums; the last of its blocks to arrive adds them up in the blocks' order, so
// the result does not depend on timing.
#include <cmath>

#include "cache_attend.cuh"

namespace bacon {
namespace {

using namespace tc;

constexpr int kTile = 64;     // tokens
constexpr int kWarps = 4;     // that compute
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kStages = 4;

struct Meta {  // of 16 tokens of a stage
    float k_scale, v_log2, v_inv;
};

template <int D, int NT>
struct Smem {
    static constexpr int kRows = kTile * D;        // bytes of K, or V, of a stage
    static constexpr int kStage = 2 * kRows;
    static constexpr int kJoin = kStages * kStage; // two warps' outputs
    static constexpr int kQ = kJoin + 2 * NT * D * 8 * 4;
    // queries as fp16 fragments, where they do not stay in registers
    static constexpr int kMeta = kQ + (NT > 2 ? NT * D * 8 * 2 : 0);
    static constexpr int kBytes = kMeta + 2048;
};

struct Shared {
    Meta meta[kStages][kWarps];
    float top[kWarps][32], sum[kWarps][32];
    uint64_t full[kStages], empty[kStages];
    long long scan[kWarps + 1];
    Found found;
    int abort;
    int nan_at[128];        // per dim: first position of a NaN of V that not every column sees
    int nan_any;
};
static_assert(sizeof(Shared) <= 2048, "shared record");

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

template <int FORMAT, int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 3 : NT == 2 ? 2 : 1)
few_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
           CacheGeom g, AttendArgs a, SplitScratch sc)
{
    using S = Smem<D, NT>;
    constexpr int kChunks = D / 16;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared& sh = *reinterpret_cast<Shared*>(smem + S::kMeta);
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 1);
            mbar_init(smem_u32(&sh.empty[s]), kWarps);
        }
        fence_barrier_init();
        sh.abort = sh.nan_any = 0;
    }
    for (int i = tid; i < 128; i += kThreads) sh.nan_at[i] = 0x7FFFFFFF;

    Place place;
    if (!find_place<8 * NT, kTile, kThreads>(g, a, sh.scan, sh.found, place)) return;
    const int b = blockIdx.x, blocks = place.blocks;
    const long long total = place.total, lo = place.lo, hi = place.hi;
    bool bad = false;

    int unit = place.unit;
    Item it = item_of<8 * NT, kTile>(g, a, unit, place.block, bad);
    long long at = place.at;  // the item's first tile
    const uint32_t abort_flag = smem_u32(&sh.abort);

    if (warp == kWarps) {
        // ------------------------------------------------------ loads
        // lanes 0-3: K's 16-row groups of a tile, lanes 4-7: V's
        const int group = lane & 3;
        const CUtensorMap* const map = lane < 4 ? &kmap : &vmap;
        const float* const scales = lane < 4 ? g.k_scale : g.v_scale;
        int stage = 0, issued = 0;
        uint32_t phase = 0;
        bool stop = false;
        long long t = lo;
        while (t < hi && !stop) {
            const int32_t* const table =
                a.table + (((size_t)it.r * g.layers + a.layer) * g.hkv + it.h) * g.max_blocks;
            const int end = (int)min((long long)it.tiles, hi - at);
            for (int i = (int)(t - at); i < end; ++i, ++t) {
                const int pos = i * kTile + group * 16;
                const bool live = lane < 8 && pos < it.seen;
                int page = 0;
                if (live) {
                    page = table[pos >> g.page_log2];
                    if (page < 0 || page >= g.pages) {
                        atomicCAS(g.err, 0, kCacheBadIndex);
                        page = 0;
                    }
                }
                const uint32_t full = smem_u32(&sh.full[stage]);
                if (!mbar_wait(smem_u32(&sh.empty[stage]), phase ^ 1, abort_flag)) {
                    stop = true;
                    break;
                }
                const int boxes = __popc(__ballot_sync(0xFFFFFFFFu, live));
                if (lane == 0 && boxes) mbar_expect_tx(full, boxes * kBoxRows * D);
                __syncwarp();
                float s = 1.0f;
                if (live) {
                    load_rows(base + stage * S::kStage + (lane >> 2) * S::kRows + group * 16 * D, map,
                              (page << g.page_log2) + (pos & (g.page - 1)), full);
                    s = scales[page];
                }
                if (lane < 4) {
                    sh.meta[stage][group].k_scale = s;
                } else if (lane < 8) {
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
            }
            at += it.tiles;
            if (t < hi && !stop && !next_item<8 * NT, kTile>(g, a, unit, it)) break;
        }
        if (stop) {
            // the block's copies end before it does
            if (lane == 0) {
                st_shared_volatile(abort_flag, 1);
                atomicCAS(g.err, 0, kCacheTimeout);
            }
            for (int i = max(0, issued - kStages); i < issued; ++i)
                mbar_wait(smem_u32(&sh.full[i % kStages]), i / kStages & 1, 0);
        }
        return;
    }

    // ---------------------------------------------------------- products
    const int gr = lane >> 2, tq = lane & 3;
    int stage = 0;
    uint32_t phase = 0;
    float acc[kChunks][NT][4];
    float top[NT][2], sum[NT][2], factor[NT][2];
    int sees[NT][2];
    uint32_t qf[NT > 2 ? 1 : kChunks][NT > 2 ? 1 : NT][2];
    // matrix loads: lane l gives row l & 7 of matrix l >> 3; matrices are rows
    // 0-7, rows 8-15, of 16-byte chunk c, then of c + 1
    const int mrow = warp * 16 + (lane & 7) + (lane >> 3 & 1) * 8, mchunk = lane >> 4;
    const uint32_t swizzle = D == 128 ? mrow & 7 : mrow >> 1 & 3;

    for (long long t = lo; t < hi;) {
        // the item's queries as fragments: column g of an n-tile, dims 16 c +
        // 4 tq ... + 3 of every chunk c
        const uint16_t* qrow[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int c = it.block * 8 * NT + nt * 8 + gr, j = c / g.group;
            qrow[nt] = j < it.asked ? a.q + (long long)(it.start + j) * a.q_token_stride +
                                          (it.h * g.group + c % g.group) * a.q_head_stride
                                    : nullptr;
            float amax = 0.0f;
            uint2 raw[kChunks];
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                raw[k] = make_uint2(0, 0);
                if (qrow[nt]) raw[k] = *reinterpret_cast<const uint2*>(qrow[nt] + k * 16 + tq * 4);
            }
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
                const uint2 f = make_uint2(half2_of(u.x * up, u.y * up), half2_of(v.x * up, v.y * up));
                if (NT > 2) {
                    if (warp == nt % kWarps)
                        *reinterpret_cast<uint2*>(smem + S::kQ + ((k * NT + nt) * 32 + lane) * 8) = f;
                } else {
                    qf[NT > 2 ? 0 : k][NT > 2 ? 0 : nt][0] = f.x;
                    qf[NT > 2 ? 0 : k][NT > 2 ? 0 : nt][1] = f.y;
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int col = it.block * 8 * NT + nt * 8 + tq * 2 + i;
                sees[nt][i] = col / g.group < it.asked ? seen_by(a, it.n, it.asked, col / g.group) : 0;
                top[nt][i] = -INFINITY;
                sum[nt][i] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[k][nt][i] = 0.0f;
        }
        if (NT > 2) named_barrier_sync(1, 32 * kWarps);
        // positions that every column sees
        const int all = seen_by(a, it.n, it.asked, it.block * 8 * NT / g.group);

        const int begin = (int)(t - at), end = (int)min((long long)it.tiles, hi - at);
        for (int i = begin; i < end; ++i) {
            if (!mbar_wait(smem_u32(&sh.full[stage]), phase, abort_flag) && lane == 0) {
                st_shared_volatile(abort_flag, 1);
                atomicCAS(g.err, 0, kCacheTimeout);
            }
            __syncwarp();
            const int pos = i * kTile + warp * 16;
            if (pos < it.seen) {
                const uint32_t krow = base + stage * S::kStage + mrow * D;
                const Meta meta = sh.meta[stage][warp];
                float s[NT][2][4];  // two chains of products
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[nt][0][e] = s[nt][1][e] = 0.0f;
#pragma unroll
                for (int c = 0; c < kChunks; c += 2) {
                    uint32_t w[4], f[8];
                    ldmatrix4(w, krow + (((c + mchunk) ^ swizzle) << 4));
                    // rows gr and gr + 8, first pairs of dims then second ones
                    codes_half<FORMAT>(w[0], f[0], f[2]);
                    codes_half<FORMAT>(w[1], f[1], f[3]);
                    codes_half<FORMAT>(w[2], f[4], f[6]);
                    codes_half<FORMAT>(w[3], f[5], f[7]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        uint2 q0, q1;
                        if (NT > 2) {
                            q0 = *reinterpret_cast<const uint2*>(smem + S::kQ + ((c * NT + nt) * 32 + lane) * 8);
                            q1 = *reinterpret_cast<const uint2*>(smem + S::kQ +
                                                                 (((c + 1) * NT + nt) * 32 + lane) * 8);
                        } else {
                            constexpr int z = NT > 2 ? 0 : 1;
                            q0 = make_uint2(qf[c * z][nt * z][0], qf[c * z][nt * z][1]);
                            q1 = make_uint2(qf[(c + 1) * z][nt * z][0], qf[(c + 1) * z][nt * z][1]);
                        }
                        mma(s[nt][0], f, q0.x, q0.y);
                        mma(s[nt][1], f + 4, q1.x, q1.y);
                    }
                }
                // exponents, the running maximum, weights
                const bool cut = pos + 16 > all;
                uint32_t p[NT][2];
                bool grew = false;
                float keep[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float y[4], high[2];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[e] = (s[nt][0][e] + s[nt][1][e]) * (factor[nt][e & 1] * meta.k_scale) + meta.v_log2;
                        if (cut && pos + gr + (e >> 1) * 8 >= sees[nt][e & 1]) y[e] = -INFINITY;
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        high[k] = fmaxf(y[k], y[k + 2]);
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1)
                            high[k] = fmaxf(high[k], __shfl_xor_sync(0xFFFFFFFFu, high[k], o));
                        keep[nt][k] = 1.0f;
                        if (high[k] > top[nt][k]) {
                            keep[nt][k] = fast_exp2(top[nt][k] - high[k]);
                            top[nt][k] = high[k];
                            grew = true;
                        }
                        const float m = top[nt][k] == -INFINITY ? 0.0f : top[nt][k] - kWeightTop;
                        y[k] = fast_exp2(y[k] - m);
                        y[k + 2] = fast_exp2(y[k + 2] - m);
                        sum[nt][k] = sum[nt][k] * keep[nt][k] + (y[k] + y[k + 2]) * meta.v_inv;
                    }
                    p[nt][0] = transpose8(half2_of(y[0], y[1]));
                    p[nt][1] = transpose8(half2_of(y[2], y[3]));
                }
                if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[c][nt][e] *= keep[nt][e & 1];
                }
                const uint32_t vrow = krow + S::kRows;
#pragma unroll
                for (int c = 0; c < kChunks; c += 2) {
                    uint32_t w[4], f[8];
                    ldmatrix4_trans(w, vrow + (((c + mchunk) ^ swizzle) << 4));
                    if (cut) {
                        // rows that no column sees are whatever the page holds;
                        // a NaN that some column does not see is taken out
                        // and put back at the item's end
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            const int x0 = pos + (m & 1) * 8 + 2 * tq;
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
                        mma(acc[c][nt], f, p[nt][0], p[nt][1]);
                        mma(acc[c + 1][nt], f + 4, p[nt][0], p[nt][1]);
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
                    sh.top[warp][nt * 8 + tq * 2 + k] = top[nt][k];
                    sh.sum[warp][nt * 8 + tq * 2 + k] = sum[nt][k];
                }
            }
        named_barrier_sync(1, 32 * kWarps);
        const bool nan = sh.nan_any != 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int col = nt * 8 + tq * 2 + k;
                float m = sh.top[0][col];
#pragma unroll
                for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sh.top[w][col]);
                const float f = top[nt][k] == -INFINITY ? 0.0f : fast_exp2(top[nt][k] - m);
                float l = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w)  // (a sum of NaN has no maximum)
                    l += sh.sum[w][col] * (sh.top[w][col] == -INFINITY ? 0.0f : fast_exp2(sh.top[w][col] - m));
                top[nt][k] = m;
                sum[nt][k] = l;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    acc[c][nt][k] *= f;
                    acc[c][nt][k + 2] *= f;
                }
            }
        float4* const join = reinterpret_cast<float4*>(smem + S::kJoin);
        if (warp >= 2) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    join[((warp - 2) * kChunks * NT + c * NT + nt) * 32 + lane] =
                        *reinterpret_cast<float4*>(acc[c][nt]);
        }
        named_barrier_sync(1, 32 * kWarps);
        if (warp < 2) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float4* const z = &join[(warp * kChunks * NT + c * NT + nt) * 32 + lane];
                    const float4 o = *z;
                    acc[c][nt][0] += o.x;
                    acc[c][nt][1] += o.y;
                    acc[c][nt][2] += o.z;
                    acc[c][nt][3] += o.w;
                    if (warp == 1) *z = *reinterpret_cast<float4*>(acc[c][nt]);
                }
        }
        named_barrier_sync(1, 32 * kWarps);

        const bool whole = begin == 0 && end == it.tiles;
        const long long item_at = at;
        bool write = warp == 0;
        if (warp == 0) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float4 o = join[(kChunks * NT + c * NT + nt) * 32 + lane];
                    acc[c][nt][0] += o.x;
                    acc[c][nt][1] += o.y;
                    acc[c][nt][2] += o.z;
                    acc[c][nt][3] += o.w;
                }
            if (nan) {
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (sh.nan_at[c * 16 + 2 * gr + (e >> 1)] < sees[nt][e & 1])
                                acc[c][nt][e] = NAN;
            }
            if (!whole) {
                // slot 2 b + 1: the item's first part, 2 b: a later one
                const size_t slot = 2 * (size_t)b + (begin == 0 ? 1 : 0);
                float4* const po = reinterpret_cast<float4*>(sc.out + slot * 32 * 128);
                float2* const pm = reinterpret_cast<float2*>(sc.sums + slot * 64);
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        po[(c * NT + nt) * 32 + lane] = *reinterpret_cast<float4*>(acc[c][nt]);
                if (gr == 0)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            pm[nt * 8 + tq * 2 + k] = make_float2(top[nt][k], sum[nt][k]);
                __threadfence();
                __syncwarp();
                const int first = owner_of(total, item_at, blocks);
                const int parts = owner_of(total, item_at + it.tiles - 1, blocks) - first + 1;
                int last = 0;
                if (lane == 0) {
                    last = atomicAdd(&sc.arrived[first], 1) == parts - 1;
                    if (last) sc.arrived[first] = 0;
                }
                write = __shfl_sync(0xFFFFFFFFu, last, 0) != 0;
                if (write) {
                    __threadfence();
                    float m[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            m[nt][k] = -INFINITY;
                            for (int q = 0; q < parts; ++q) {
                                const float2* const pq = reinterpret_cast<const float2*>(
                                    sc.sums + (2 * (size_t)(first + q) + (q == 0)) * 64);
                                m[nt][k] = fmaxf(m[nt][k], __ldcg(&pq[nt * 8 + tq * 2 + k]).x);
                            }
                            top[nt][k] = m[nt][k];
                            sum[nt][k] = 0.0f;
                        }
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[c][nt][e] = 0.0f;
                    for (int q = 0; q < parts; ++q) {
                        const size_t part = 2 * (size_t)(first + q) + (q == 0);
                        const float2* const pq = reinterpret_cast<const float2*>(sc.sums + part * 64);
                        const float4* const oq = reinterpret_cast<const float4*>(sc.out + part * 32 * 128);
                        float f[NT][2];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const float2 z = __ldcg(&pq[nt * 8 + tq * 2 + k]);
                                f[nt][k] = z.x == -INFINITY ? 0.0f : fast_exp2(z.x - m[nt][k]);
                                sum[nt][k] += z.y * f[nt][k];
                            }
#pragma unroll
                        for (int c = 0; c < kChunks; ++c)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const float4 o = __ldcg(&oq[(c * NT + nt) * 32 + lane]);
                                acc[c][nt][0] = fmaf(o.x, f[nt][0], acc[c][nt][0]);
                                acc[c][nt][1] = fmaf(o.y, f[nt][1], acc[c][nt][1]);
                                acc[c][nt][2] = fmaf(o.z, f[nt][0], acc[c][nt][2]);
                                acc[c][nt][3] = fmaf(o.w, f[nt][1], acc[c][nt][3]);
                            }
                    }
                }
            }
        }
        if (write) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int col = it.block * 8 * NT + nt * 8 + tq * 2 + k, j = col / g.group;
                    if (j >= it.asked) continue;
                    const size_t row = (size_t)(it.start + j) * g.hq + it.h * g.group + col % g.group;
                    const bool none = sees[nt][k] == 0;
                    const float inv = none ? 0.0f : 1.0f / sum[nt][k];
                    uint32_t* const o = reinterpret_cast<uint32_t*>(a.out + row * D);
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
                        o[c * 8 + gr] = none ? 0u : pack16(g.dtype, acc[c][nt][k] * inv, acc[c][nt][k + 2] * inv);
                    if (a.lse && gr == 0)
                        a.lse[row] = none ? -INFINITY
                                          : (log2f(sum[nt][k]) + (top[nt][k] - kWeightTop)) * kLn2;
                }
        }
        named_barrier_sync(1, 32 * kWarps);
        if (nan) {  // the item's, not the next one's
            for (int i = tid; i < 128; i += 32 * kWarps) sh.nan_at[i] = 0x7FFFFFFF;
            if (tid == 0) sh.nan_any = 0;
            named_barrier_sync(1, 32 * kWarps);
        }
        t = at + end;
        at += it.tiles;
        if (t < hi && !next_item<8 * NT, kTile>(g, a, unit, it)) break;
    }
}

template <int FORMAT, int D, int NT>
cudaError_t go(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc, cudaStream_t st)
{
    constexpr int bytes = Smem<D, NT>::kBytes;
    static const cudaError_t ready = cudaFuncSetAttribute(
        few_kernel<FORMAT, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (ready != cudaSuccess) return ready;
    constexpr int per_sm = NT == 1 ? 3 : NT == 2 ? 2 : 1;
    static_assert(per_sm <= kBlocksPerSm, "room for partial sums");
    return launch_first(few_kernel<FORMAT, D, NT>, sc.sms * per_sm, kThreads, bytes, st, sc.kmap, sc.vmap, g, a, sc);
}

template <int FORMAT, int D>
cudaError_t by_columns(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc, cudaStream_t st)
{
    const long long columns = (long long)g.group * ((a.tokens + a.requests - 1) / a.requests);
    if (columns <= 8) return go<FORMAT, D, 1>(g, a, sc, st);
    if (columns <= 16) return go<FORMAT, D, 2>(g, a, sc, st);
    return go<FORMAT, D, 4>(g, a, sc, st);
}

}  // namespace

cudaError_t launch_cache_few(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                             cudaStream_t st)
{
    if (g.format == BACON_E4M3)
        return g.d == 128 ? by_columns<BACON_E4M3, 128>(g, a, sc, st) : by_columns<BACON_E4M3, 64>(g, a, sc, st);
    return g.d == 128 ? by_columns<BACON_INT8, 128>(g, a, sc, st) : by_columns<BACON_INT8, 64>(g, a, sc, st);
}

}  // namespace bacon
