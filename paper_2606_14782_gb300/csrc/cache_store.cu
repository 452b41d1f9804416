// Rows into the pages of the 8-bit cache and back: bound by their bytes, three
// of every element of a row one way or the other.  459k rows of K and V of 128
// are stored in 62 us and loaded in 54 (84 and 96 % of the measured copy
// bandwidth); a row of 256 units in 3.0 and 2.1.
//
// A run is the rows of one call that lie in one page one after the other.  A
// block takes a run of K and V: its rows are read once, into registers (2 x 4 x
// 16 bytes a thread at most), their largest finite magnitude gives the page's
// scale, and the codes leave as 8 bytes a thread.  A page that is appended to
// (the run starts above row 0) keeps its scale unless the new rows need a
// larger one; then its older rows are quantised again.  Blocks find their runs
// themselves: a run belongs to the block whose window of tokens it starts in,
// and one pass over the window's slots and a page's beyond marks where runs
// break.  The magnitudes are compared as 16-bit integers, two at a time; only
// when the largest is an infinity or NaN are they gone through again without
// such values.
#include "cache.h"
#include "cache_values.cuh"
#include "common.cuh"

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

template <int DTYPE, int FORMAT, int D>
__global__ void __launch_bounds__(512)
store_kernel(CacheGeom g, StoreArgs a, int window)
{
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
                    if (r < len)
                        raw[z][c] = *reinterpret_cast<const uint4*>(rows[z] + (t + r) * a.token_stride[z] + q * 8);
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

// Eight codes as values.
template <int DTYPE, int FORMAT>
__device__ __forceinline__ uint4 values_of(uint2 c, float s)
{
    const float4 x = codes_float<FORMAT>(c.x), y = codes_float<FORMAT>(c.y);
    return make_uint4(pack16<DTYPE>(x.x * s, x.y * s), pack16<DTYPE>(x.z * s, x.w * s),
                      pack16<DTYPE>(y.x * s, y.y * s), pack16<DTYPE>(y.z * s, y.w * s));
}

// A thread takes 8 values of K and the same of V (one slot's latency for both)
// of two rows, so that a warp's stores are whole lines.
template <int DTYPE, int FORMAT, int D>
__global__ void __launch_bounds__(256)
load_kernel(CacheGeom g, int rows, const int32_t* slots, uint16_t* k_out, uint16_t* v_out)
{
    constexpr int kLanes = D / 8, kRows = 256 / kLanes;
    const int q = threadIdx.x % kLanes;
    const long long i0 = (long long)blockIdx.x * (2 * kRows) + threadIdx.x / kLanes;
    int slot[2];
    uint2 k[2], v[2];
    float ks[2], vs[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) slot[z] = i0 + z * kRows < rows ? slots[i0 + z * kRows] : -1;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        k[z] = v[z] = make_uint2(0, 0);
        ks[z] = vs[z] = 0.0f;
        if (slot[z] >= 0 && slot[z] < (long long)g.pages << g.page_log2) {
            k[z] = *reinterpret_cast<const uint2*>(g.k + (size_t)slot[z] * D + q * 8);
            v[z] = *reinterpret_cast<const uint2*>(g.v + (size_t)slot[z] * D + q * 8);
            ks[z] = g.k_scale[slot[z] >> g.page_log2];
            vs[z] = g.v_scale[slot[z] >> g.page_log2];
        } else if (slot[z] != -1) {
            atomicCAS(g.err, 0, kCacheBadIndex);
        }
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const long long i = i0 + z * kRows;
        if (i >= rows) break;
        *reinterpret_cast<uint4*>(k_out + i * D + q * 8) = values_of<DTYPE, FORMAT>(k[z], ks[z]);
        *reinterpret_cast<uint4*>(v_out + i * D + q * 8) = values_of<DTYPE, FORMAT>(v[z], vs[z]);
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

template <int DTYPE, int FORMAT, int D>
struct Store {
    static cudaError_t go(const CacheGeom& g, const StoreArgs& a, dim3 grid, int window,
                          cudaStream_t st)
    {
        return launch_first(store_kernel<DTYPE, FORMAT, D>, grid, g.page * D / 8 / kChunks, 0, st, g,
                            a, window);
    }
};
template <int DTYPE, int FORMAT, int D>
struct Load {
    static cudaError_t go(const CacheGeom& g, int rows, const int32_t* slots, void* k_out,
                          void* v_out, cudaStream_t st)
    {
        const int own = 2 * 256 / (D / 8);  // rows of a block
        return launch_first(load_kernel<DTYPE, FORMAT, D>, (unsigned)((rows + own - 1LL) / own),
                            256, 0, st, g, rows, slots, static_cast<uint16_t*>(k_out),
                            static_cast<uint16_t*>(v_out));
    }
};

}  // namespace

cudaError_t launch_cache_store(const CacheGeom& g, const StoreArgs& a, cudaStream_t st)
{
    // windows of a page when there are rows for several blocks per SM; smaller
    // ones when there are few, so that short runs do not queue in one block
    const long long per_block = (long long)a.tokens * a.heads / (152 * 8);
    int window = per_block < 1 ? 1 : per_block > g.page ? g.page : (int)per_block;
    const dim3 grid((unsigned)((a.tokens + window - 1) / window), a.heads);
    return by_type<Store>(g, a, grid, window, st);
}

cudaError_t launch_cache_load(const CacheGeom& g, int rows, const int32_t* slots, void* k_out,
                              void* v_out, cudaStream_t st)
{
    return by_type<Load>(g, rows, slots, k_out, v_out, st);
}

}  // namespace bacon
