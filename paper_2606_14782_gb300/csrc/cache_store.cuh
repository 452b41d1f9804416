// The kernel that quantises rows into pages (cache_store.cu says how); with
// positions put into the rows of K first, and into Q's, for
// bacon_cache_store_rotated.
#pragma once

#include "cache.h"
#include "cache_values.cuh"
#include "common.cuh"
#include "rotary.cuh"

namespace bacon {
namespace {

constexpr int kChunks = 4;  // 16-byte pieces of rows per thread

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    uint32_t m;
    asm("max.u16x2 %0, %1, %2;\n" : "=r"(m) : "r"(a), "r"(b));
    return m;
}

// The larger of both halves, over the block, for K's and for V's.
__device__ __forceinline__ void block_max(uint32_t (&m)[2], uint32_t (*s_max)[2])
{
    const int lane = threadIdx.x & 31, warps = blockDim.x / 32;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        m[z] = max(m[z] & 0xFFFFu, m[z] >> 16);
        m[z] = __reduce_max_sync(0xFFFFFFFFu, m[z]);
        if (warps > 1 && lane == 0) s_max[threadIdx.x >> 5][z] = m[z];
    }
    if (warps == 1) return;
    __syncthreads();
#pragma unroll
    for (int z = 0; z < 2; ++z) m[z] = __reduce_max_sync(0xFFFFFFFFu, lane < warps ? s_max[lane][z] : 0);
}

// Positions into the rows of K that a run's threads have: 16 bytes of the rows
// t + r, r < len.  The same steps as rotate_eights, rounded to DTYPE as there.
template <int DTYPE, int D, int PAIR>
__device__ __forceinline__ void turn_rows(const RotaryArgs& a, const uint16_t* rows,
                                          long long token_stride, long long t, int len,
                                          uint4 (&raw)[kChunks])
{
    const RotaryTable& tab = a.table;
    const void* const weight = a.rows[1].weight;
    const int q = threadIdx.x % (D / 8), e0 = 8 * q;
    // the rows' places on their way together, and the lane's part of the table once
    RotaryPlace at[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int r = (threadIdx.x + i * blockDim.x) / (D / 8);
        at[i] = RotaryPlace{{0, 0, 0}};
        if (r < len) at[i] = place_of(tab, t + r);
    }
    const RotaryLane<PAIR> lane = lane_of<PAIR>(tab, e0);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        if (i * (int)blockDim.x / (D / 8) >= len) break;  // nobody has a row
        const int r = (threadIdx.x + i * blockDim.x) / (D / 8);
        const bool mine = r < len;
        Eight<DTYPE> w{{raw[i].x, raw[i].y, raw[i].z, raw[i].w}};
        Piece x, other, c, s, y;
        open_piece(w, x);
        pairs_of<DTYPE, PAIR>(tab, w, x, rows + (t + r) * token_stride, mine, q, other);
        factors_of<PAIR>(tab, lane, at[i], e0, c, s);
        if (weight) weigh<DTYPE, PAIR>(tab, weight, q, c, s);
        const float inv = row_inverse(tab, D == 128 ? 4 : 3, weight != nullptr, x, other);
        turn_piece(x, other, c, s, y);
        scale_piece(y, inv);
        close_piece(w, y);
        if (mine) raw[i] = make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]);
    }
}

// The same with eight pairs a lane, into `stage` ([page][D]): half as many lanes have
// a row, so that a run's rows are turned in two steps at most, and each lane works
// out half as many angles.
template <int DTYPE, int D, bool SIXTEEN>
__device__ __forceinline__ void stage_rows(const RotaryArgs& a, const uint16_t* rows,
                                           long long token_stride, long long t, int len, uint16_t* stage)
{
    constexpr int kLanes = D / 16, kSteps = kChunks / 2;
    const RotaryTable& tab = a.table;
    const int q = threadIdx.x % kLanes, group = threadIdx.x / kLanes, groups = blockDim.x / kLanes;
    const RotarySpan span = span_of<SIXTEEN>(tab, q);
    Eight<DTYPE> one[kSteps], two[kSteps];
    RotaryPlace at[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int r = group + i * groups;
#pragma unroll
        for (int j = 0; j < 4; ++j) one[i].w[j] = two[i].w[j] = 0;
        at[i] = RotaryPlace{{0, 0, 0}};
        if (r >= len) continue;
        load_eight(one[i], rows + (t + r) * token_stride + span.e0);
        load_eight(two[i], rows + (t + r) * token_stride + span.e1);
        at[i] = place_of(tab, t + r);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int r = group + i * groups;
        if (i * groups >= len) break;  // nobody has a row
        PairFactors f;
        pair_factors<DTYPE, SIXTEEN, true>(tab, at[i], a.rows[1].weight, q, span, f);
        turn_pairs<DTYPE, SIXTEEN, true>(tab, D == 128 ? 3 : 2, q, a.rows[1].weight != nullptr, span, f, one[i], two[i]);
        if (r >= len) continue;
        store_eight(stage + r * D + span.e0, one[i]);
        store_eight(stage + r * D + span.e1, two[i]);
    }
}

struct NoRotary {};
struct StoreRotary {
    RotaryArgs args;  // rows[0]: Q; rows[1]: K's weight
    RotaryDeal deal;  // of Q's heads
};
constexpr int kNoPair = -1;

// PAIR: kNoPair, or how the rotation of K gets its pairs (rotary.cuh).  ROTARY:
// NoRotary, or StoreRotary with which blocks beyond the heads of K turn Q.
template <int DTYPE, int FORMAT, int D, int PAIR, typename ROTARY>
__global__ void __launch_bounds__(512)
store_kernel(CacheGeom g, StoreArgs a, int window, const __grid_constant__ ROTARY rotary)
{
    extern __shared__ __align__(16) uint16_t s_stage[];  // turned rows of K
    constexpr bool kStaged = PAIR == kPairHalves || PAIR == kPairSixteen;
    if constexpr (PAIR != kNoPair) {
        if (blockIdx.y >= a.heads) {
            const unsigned groups = blockDim.x >> rotary.deal.log_lanes;
            unsigned item = ((blockIdx.y - a.heads) * gridDim.x + blockIdx.x) * groups;
            item += threadIdx.x >> rotary.deal.log_lanes;
            rotate_piece<DTYPE, PAIR, true>(rotary.args, rotary.deal, item);
            return;
        }
    }
    constexpr uint32_t kInfinite = DTYPE == BACON_BF16 ? 0x7F80 : 0x7C00;
    __shared__ uint32_t s_start[4];   // bit i: a run starts at the window's token i
    __shared__ uint32_t s_break[9];   // bit i: no run goes on from token i - 1 to i
    __shared__ uint32_t s_max[2][16][2];
    const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
    const int h = blockIdx.y;
    const int p = g.page;
    const long long t0 = (long long)blockIdx.x * window;
    const long long limit = (long long)g.pages << g.page_log2;
    const uint16_t* const rows[2] = {a.rows[0] + h * a.head_stride[0], a.rows[1] + h * a.head_stride[1]};
    const int32_t* const slots = a.slots + h;

    for (int base = 0; base < window + p; base += threads) {
        const int i = base + tid;
        const long long t = t0 + i;
        bool start = false, stop = true;
        if (i < window + p && t < a.tokens) {
            const int s = slots[t * a.heads], prev = t ? slots[(t - 1) * a.heads] : -1;
            const bool on = (s & (p - 1)) != 0 && prev == s - 1;
            if (s >= 0 && s < limit) {
                stop = !on;
                start = !on && i < window;
                // a page's rows out of order, or with a gap: two blocks could
                // have them, so the later ones are left out (prev in s's page)
                if (start && (unsigned)(prev ^ s) < (unsigned)p) {
                    start = false;
                    atomicCAS(g.err, 0, kCacheBadIndex);
                }
            } else if (s != -1 && i < window) {
                atomicCAS(g.err, 0, kCacheBadIndex);
            }
        }
        const uint32_t starts = __ballot_sync(0xFFFFFFFFu, start);
        const uint32_t stops = __ballot_sync(0xFFFFFFFFu, stop);
        if (lane == 0) {
            const int w = i >> 5;
            if (w < 4) s_start[w] = starts;
            if (w < 9) s_break[w] = stops;
        }
    }
    __syncthreads();

    int parity = 0;
    for (int word = 0; word * 32 < window; ++word) {
        for (uint32_t left = s_start[word]; left; left &= left - 1) {
            const int i = word * 32 + __ffs(left) - 1;
            const long long t = t0 + i;
            const int slot = slots[t * a.heads];
            const int page = slot >> g.page_log2, off = slot & (p - 1);
            // to the next break: within a page's tokens there is one, or the page ends
            int len = p - off;
            for (int w = i >> 5; w * 32 < i + len; ++w) {
                uint32_t x = s_break[w];
                if (w == i >> 5) x &= ~(2u << (i & 31)) + 1u;  // bits above i
                if (x) {
                    len = min(len, w * 32 + __ffs(x) - 1 - i);
                    break;
                }
            }
            const float old[2] = {off ? g.k_scale[page] : 0.0f, off ? g.v_scale[page] : 0.0f};

            uint4 raw[2][kChunks];
            uint32_t most[2] = {0, 0};
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const int e = tid + c * threads, r = e / (D / 8), q = e % (D / 8);
                    raw[z][c] = make_uint4(0, 0, 0, 0);
                    if (r < len && !(kStaged && z == 0))
                        raw[z][c] = *reinterpret_cast<const uint4*>(rows[z] + (t + r) * a.token_stride[z] + q * 8);
                }
            if constexpr (kStaged) {
                __syncthreads();  // the run before has been taken from there
                stage_rows<DTYPE, D, PAIR == kPairSixteen>(rotary.args, rows[0], a.token_stride[0], t, len, s_stage);
                __syncthreads();
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const int e = tid + c * threads;
                    if (e / (D / 8) < len) raw[0][c] = reinterpret_cast<const uint4*>(s_stage)[e];
                }
            } else if constexpr (PAIR != kNoPair) {
                turn_rows<DTYPE, D, PAIR>(rotary.args, rows[0], a.token_stride[0], t, len, raw[0]);
            }
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const uint4 w = raw[z][c];
                    const uint32_t x = max_u16x2(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu);
                    const uint32_t y = max_u16x2(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu);
                    most[z] = max_u16x2(most[z], max_u16x2(x, y));
                }
            block_max(most, s_max[parity]);
            parity ^= 1;
            if (most[0] >= kInfinite || most[1] >= kInfinite) {
                most[0] = most[1] = 0;
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) {
                        const uint32_t w[4] = {raw[z][c].x, raw[z][c].y, raw[z][c].z, raw[z][c].w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t lo = w[j] & 0x7FFFu, hi = w[j] >> 16 & 0x7FFFu;
                            if (lo < kInfinite) most[z] = max(most[z], lo);
                            if (hi < kInfinite) most[z] = max(most[z], hi);
                        }
                    }
                block_max(most, s_max[parity]);
                parity ^= 1;
            }
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const float scale = fmaxf(old[z], scale_of<FORMAT>(unpack16<DTYPE>(most[z]).x));
                const float inv = __fdiv_rn(1.0f, scale);
                uint8_t* const dst = (z ? g.v : g.k) + ((size_t)page << g.page_log2) * D;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const int e = tid + c * threads, r = e / (D / 8), q = e % (D / 8);
                    if (r >= len) continue;
                    const uint4 w = raw[z][c];
                    const float2 v0 = unpack16<DTYPE>(w.x), v1 = unpack16<DTYPE>(w.y);
                    const float2 v2 = unpack16<DTYPE>(w.z), v3 = unpack16<DTYPE>(w.w);
                    uint2 code;
                    code.x = encode4<FORMAT>(make_float4(v0.x, v0.y, v1.x, v1.y), scale, inv);
                    code.y = encode4<FORMAT>(make_float4(v2.x, v2.y, v3.x, v3.y), scale, inv);
                    *reinterpret_cast<uint2*>(dst + (size_t)(off + r) * D + q * 8) = code;
                }
                if (off && scale > old[z])  // older rows of the page
                    for (int e = tid; e < off * D / 4; e += threads) {
                        uint32_t* const w = reinterpret_cast<uint32_t*>(dst) + e;
                        float4 x = codes_float<FORMAT>(*w);
                        x.x *= old[z];
                        x.y *= old[z];
                        x.z *= old[z];
                        x.w *= old[z];
                        *w = encode4<FORMAT>(x, scale, inv);
                    }
                if (tid == 0) (z ? g.v_scale : g.k_scale)[page] = scale;
            }
        }
    }
}

// f(dtype, format, head_dim) with all three as constants
template <template <int, int, int> class F, typename... A>
cudaError_t by_type(const CacheGeom& g, A&&... a)
{
    const int key = (g.dtype == BACON_FP16) << 2 | (g.format == BACON_INT8) << 1 | (g.d == 128);
    switch (key) {
        case 0: return F<BACON_BF16, BACON_E4M3, 64>::go(g, a...);
        case 1: return F<BACON_BF16, BACON_E4M3, 128>::go(g, a...);
        case 2: return F<BACON_BF16, BACON_INT8, 64>::go(g, a...);
        case 3: return F<BACON_BF16, BACON_INT8, 128>::go(g, a...);
        case 4: return F<BACON_FP16, BACON_E4M3, 64>::go(g, a...);
        case 5: return F<BACON_FP16, BACON_E4M3, 128>::go(g, a...);
        case 6: return F<BACON_FP16, BACON_INT8, 64>::go(g, a...);
        default: return F<BACON_FP16, BACON_INT8, 128>::go(g, a...);
    }
}

// Tokens whose runs a block takes: a page's when there are rows for `blocks`
// blocks per SM; fewer when there are few, so that short runs do not queue in
// one block.
int store_window(const CacheGeom& g, const StoreArgs& a, int blocks)
{
    const long long per_block = (long long)a.tokens * a.heads / (152 * blocks);
    return per_block < 1 ? 1 : per_block > g.page ? g.page : (int)per_block;
}

}  // namespace
}  // namespace bacon
