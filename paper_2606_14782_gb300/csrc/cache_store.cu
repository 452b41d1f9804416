// Rows into the pages of the 8-bit cache and back.
//
// A run is the rows of one call that lie in one page one after the other.  A
// block takes a run: its rows are read once into registers (4 x 16 bytes a
// thread at most), their largest finite magnitude gives the page's scale, and
// the codes leave as 8 bytes a thread.  A page that is appended to (the run
// starts above row 0) keeps its scale unless the new rows need a larger one;
// then its older rows are quantised again.  Blocks find their runs themselves:
// a run belongs to the block whose window of tokens it starts in.
#include <cfloat>

#include "cache.h"
#include "cache_values.cuh"
#include "common.cuh"

namespace bacon {
namespace {

constexpr int kChunks = 4;  // 16-byte pieces of rows per thread

template <int DTYPE, int FORMAT, int D>
__global__ void __launch_bounds__(512)
store_kernel(CacheGeom g, StoreArgs a, int window)
{
    __shared__ uint32_t s_start[4];  // bit i: a run starts at the window's token i
    __shared__ int s_len;
    __shared__ float s_max[16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
    const int h = blockIdx.y, which = blockIdx.z;
    const int p = g.page;
    const long long t0 = (long long)blockIdx.x * window;
    const long long limit = (long long)g.pages << g.page_log2;
    const uint16_t* const rows = a.rows[which] + h * a.head_stride[which];
    const long long stride = a.token_stride[which];
    uint8_t* const pool = which ? g.v : g.k;
    float* const scales = which ? g.v_scale : g.k_scale;

    for (int base = 0; base < window; base += threads) {
        const int i = base + tid;
        const long long t = t0 + i;
        bool start = false;
        if (i < window && t < a.tokens) {
            const int s = a.slots[t * a.heads + h];
            if (s < -1 || s >= limit) {
                atomicCAS(g.err, 0, kCacheBadIndex);
            } else if (s >= 0) {
                const int prev = t ? a.slots[(t - 1) * a.heads + h] : -1;
                start = (s & (p - 1)) == 0 || prev != s - 1;
            }
        }
        const uint32_t bits = __ballot_sync(0xFFFFFFFFu, start);
        if (lane == 0 && base + warp * 32 < window) s_start[(base >> 5) + warp] = bits;
    }
    __syncthreads();

    for (int i = 0; i < window; ++i) {
        if (!(s_start[i >> 5] >> (i & 31) & 1)) continue;
        const long long t = t0 + i;
        const int slot = a.slots[t * a.heads + h];
        const int page = slot >> g.page_log2, off = slot & (p - 1);
        __syncthreads();
        if (tid == 0) s_len = p - off;
        __syncthreads();
        for (int j = tid; j < p - off; j += threads)
            if (t + j >= a.tokens || a.slots[(t + j) * a.heads + h] != slot + j) atomicMin(&s_len, j);
        __syncthreads();
        const int len = s_len;
        const float old = off ? scales[page] : 0.0f;

        uint4 raw[kChunks];
        float amax = 0.0f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int e = tid + c * threads, r = e / (D / 8), q = e % (D / 8);
            raw[c] = make_uint4(0, 0, 0, 0);
            if (r < len) raw[c] = *reinterpret_cast<const uint4*>(rows + (t + r) * stride + q * 8);
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint32_t w[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 v = unpack16<DTYPE>(w[j]);
                const float x = fabsf(v.x), y = fabsf(v.y);
                if (x <= FLT_MAX) amax = fmaxf(amax, x);
                if (y <= FLT_MAX) amax = fmaxf(amax, y);
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
        if (lane == 0) s_max[warp] = amax;
        __syncthreads();
        for (int w = 0; w < threads / 32; ++w) amax = fmaxf(amax, s_max[w]);
        const float scale = fmaxf(old, scale_of<FORMAT>(amax));
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
