// Rows into the pages of the 8-bit cache and back: bound by their bytes, three
// of every element of a row one way or the other.
//
// A run is the rows of one call that lie in one page one after the other.  A
// block takes a run of K or of V: its rows are read once, into registers (4 x
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

// The larger of both halves, over the block.
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* s_max)
{
    m = max(m & 0xFFFFu, m >> 16);
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    const int warps = blockDim.x / 32;
    if (warps == 1) return m;
    if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return __reduce_max_sync(0xFFFFFFFFu, lane < warps ? s_max[lane] : 0);
}

template <int DTYPE, int FORMAT, int D>
__global__ void __launch_bounds__(512)
store_kernel(CacheGeom g, StoreArgs a, int window)
{
    constexpr uint32_t kInfinite = DTYPE == BACON_BF16 ? 0x7F80 : 0x7C00;
    __shared__ uint32_t s_start[4];   // bit i: a run starts at the window's token i
    __shared__ uint32_t s_break[9];   // bit i: no run goes on from token i - 1 to i
    __shared__ uint32_t s_max[2][16];
    const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
    const int h = blockIdx.y, which = blockIdx.z;
    const int p = g.page;
    const long long t0 = (long long)blockIdx.x * window;
    const long long limit = (long long)g.pages << g.page_log2;
    const uint16_t* const rows = a.rows[which] + h * a.head_stride[which];
    const long long stride = a.token_stride[which];
    uint8_t* const pool = which ? g.v : g.k;
    float* const scales = which ? g.v_scale : g.k_scale;
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
            const float old = off ? scales[page] : 0.0f;

            uint4 raw[kChunks];
            uint32_t most = 0;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int e = tid + c * threads, r = e / (D / 8), q = e % (D / 8);
                raw[c] = make_uint4(0, 0, 0, 0);
                if (r < len) raw[c] = *reinterpret_cast<const uint4*>(rows + (t + r) * stride + q * 8);
            }
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const uint32_t x = max_u16x2(raw[c].x & 0x7FFF7FFFu, raw[c].y & 0x7FFF7FFFu);
                const uint32_t y = max_u16x2(raw[c].z & 0x7FFF7FFFu, raw[c].w & 0x7FFF7FFFu);
                most = max_u16x2(most, max_u16x2(x, y));
            }
            most = block_max(most, s_max[parity]);
            parity ^= 1;
            if (most >= kInfinite) {
                most = 0;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const uint32_t w[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t lo = w[j] & 0x7FFFu, hi = w[j] >> 16 & 0x7FFFu;
                        if (lo < kInfinite) most = max(most, lo);
                        if (hi < kInfinite) most = max(most, hi);
                    }
                }
                most = block_max(most, s_max[parity]);
                parity ^= 1;
            }
            const float scale = fmaxf(old, scale_of<FORMAT>(unpack16<DTYPE>(most).x));
            const float inv = __fdiv_rn(1.0f, scale);
            uint8_t* const dst = pool + ((size_t)page << g.page_log2) * D;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int e = tid + c * threads, r = e / (D / 8), q = e % (D / 8);
                if (r >= len) continue;
                const float2 v0 = unpack16<DTYPE>(raw[c].x), v1 = unpack16<DTYPE>(raw[c].y);
                const float2 v2 = unpack16<DTYPE>(raw[c].z), v3 = unpack16<DTYPE>(raw[c].w);
                uint2 code;
                code.x = encode4<FORMAT>(make_float4(v0.x, v0.y, v1.x, v1.y), scale, inv);
                code.y = encode4<FORMAT>(make_float4(v2.x, v2.y, v3.x, v3.y), scale, inv);
                *reinterpret_cast<uint2*>(dst + (size_t)(off + r) * D + q * 8) = code;
            }
            if (off && scale > old)  // older rows of the page
                for (int e = tid; e < off * D / 4; e += threads) {
                    uint32_t* const w = reinterpret_cast<uint32_t*>(dst) + e;
                    float4 x = codes_float<FORMAT>(*w);
                    x.x *= old;
                    x.y *= old;
                    x.z *= old;
                    x.w *= old;
                    *w = encode4<FORMAT>(x, scale, inv);
                }
            if (tid == 0) scales[page] = scale;
        }
    }
}

template <int DTYPE, int FORMAT, int D>
__global__ void __launch_bounds__(256)
load_kernel(CacheGeom g, int rows, const int32_t* slots, uint16_t* k_out, uint16_t* v_out)
{
    const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long i = e / (D / 16);
    const int q = (int)(e % (D / 16));
    if (i >= rows) return;
    const int slot = slots[i];
    uint4* const out = reinterpret_cast<uint4*>((blockIdx.y ? v_out : k_out) + i * D + q * 16);
    if (slot < 0 || slot >= (long long)g.pages << g.page_log2) {
        if (slot != -1) atomicCAS(g.err, 0, kCacheBadIndex);
        out[0] = out[1] = make_uint4(0, 0, 0, 0);
        return;
    }
    const float s = (blockIdx.y ? g.v_scale : g.k_scale)[slot >> g.page_log2];
    const uint4 c = *reinterpret_cast<const uint4*>((blockIdx.y ? g.v : g.k) + (size_t)slot * D + q * 16);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 x = codes_float<FORMAT>(w[j]);
        o[2 * j] = pack16<DTYPE>(x.x * s, x.y * s);
        o[2 * j + 1] = pack16<DTYPE>(x.z * s, x.w * s);
    }
    out[0] = make_uint4(o[0], o[1], o[2], o[3]);
    out[1] = make_uint4(o[4], o[5], o[6], o[7]);
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
        const long long pieces = (long long)rows * (D / 16);
        return launch_first(load_kernel<DTYPE, FORMAT, D>, dim3((unsigned)((pieces + 255) / 256), 2),
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
    const dim3 grid((unsigned)((a.tokens + window - 1) / window), a.heads, 2);
    return by_type<Store>(g, a, grid, window, st);
}

cudaError_t launch_cache_load(const CacheGeom& g, int rows, const int32_t* slots, void* k_out,
                              void* v_out, cudaStream_t st)
{
    return by_type<Load>(g, rows, slots, k_out, v_out, st);
}

}  // namespace bacon
