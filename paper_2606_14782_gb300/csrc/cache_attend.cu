// Attention over the 8-bit pages: one block per query row.
//
// s_x = scale q . k_x with k_x = k_scale[page] * code; the block's four warps
// take every fourth position each and keep a running maximum, sum and output
// in fp32; they are joined at the end.
#include <cmath>

#include "cache.h"
#include "cache_values.cuh"
#include "common.cuh"

namespace bacon {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int DTYPE, int FORMAT, int D>
__global__ void __launch_bounds__(128)
attend_kernel(CacheGeom g, AttendArgs a)
{
    constexpr int E = D / 32;  // values per lane
    __shared__ float s_o[4][D], s_m[4], s_l[4];
    const int t = blockIdx.x, head = blockIdx.y, h = head / g.group;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int r = 0, j = 0, asked = 0;
    if (a.starts) {
        if (t == 0 && head == 0) {
            bool bad = a.starts[0] != 0 || a.starts[a.requests] != a.tokens;
            for (int i = threadIdx.x; i < a.requests; i += 128) bad |= a.starts[i] > a.starts[i + 1];
            if (bad) atomicCAS(g.err, 0, kCacheBadIndex);
        }
        while (r < a.requests - 1 && a.starts[r + 1] <= t) ++r;
        j = t - a.starts[r];
        asked = a.starts[r + 1] - a.starts[r];
        if (j < 0 || j >= asked) {
            if (threadIdx.x == 0) atomicCAS(g.err, 0, kCacheBadIndex);
            return;
        }
    } else {
        asked = a.tokens / a.requests;
        r = t / asked;
        j = t % asked;
    }
    const int u = (r * g.layers + a.layer) * g.hkv + h;
    int n = a.lengths[u];
    if (n < 0 || n > (long long)g.max_blocks << g.page_log2) {
        if (threadIdx.x == 0) atomicCAS(g.err, 0, kCacheBadIndex);
        n = 0;
    }
    const int seen = a.causal ? max(0, n - asked + j + 1) : n;
    const int32_t* const table = a.table + (size_t)u * g.max_blocks;
    float q[E], o[E], m = -INFINITY, l = 0.0f;
    const uint16_t* const qrow = a.q + t * a.q_token_stride + head * a.q_head_stride + lane * E;
#pragma unroll
    for (int i = 0; i < E; i += 2) {
        const float2 x = unpack16<DTYPE>(*reinterpret_cast<const uint32_t*>(qrow + i));
        q[i] = x.x * (a.scale * kLog2e);
        q[i + 1] = x.y * (a.scale * kLog2e);
        o[i] = o[i + 1] = 0.0f;
    }
    for (int x = warp; x < seen; x += 4) {
        const int page = table[x >> g.page_log2];
        if (page < 0 || page >= g.pages) {
            if (lane == 0) atomicCAS(g.err, 0, kCacheBadIndex);
            break;
        }
        const size_t at = (((size_t)page << g.page_log2) + (x & (g.page - 1))) * D + lane * E;
        const uint32_t kw = E == 4 ? *reinterpret_cast<const uint32_t*>(g.k + at)
                                   : *reinterpret_cast<const uint16_t*>(g.k + at);
        const uint32_t vw = E == 4 ? *reinterpret_cast<const uint32_t*>(g.v + at)
                                   : *reinterpret_cast<const uint16_t*>(g.v + at);
        const float4 kc = codes_float<FORMAT>(kw), vc = codes_float<FORMAT>(vw);
        const float k4[4] = {kc.x, kc.y, kc.z, kc.w}, v4[4] = {vc.x, vc.y, vc.z, vc.w};
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) s = fmaf(q[i], k4[i], s);
#pragma unroll
        for (int b = 16; b; b >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, b);
        s *= g.k_scale[page];
        const float top = fmaxf(m, s), keep = m == -INFINITY ? 0.0f : exp2f(m - top);
        const float p = exp2f(s - top), w = p * g.v_scale[page];
        l = l * keep + p;
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = o[i] * keep + w * v4[i];
        m = top;
    }
    if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) s_o[warp][lane * E + i] = o[i];
    __syncthreads();
    const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    float sum = 0.0f, f[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f[w] = s_m[w] == -INFINITY ? 0.0f : exp2f(s_m[w] - top);
        sum += s_l[w] * f[w];
    }
    const size_t row = (size_t)t * g.hq + head;
    if ((int)threadIdx.x < D / 2) {
        float y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = threadIdx.x * 2 + i;
            y[i] = seen > 0 ? (s_o[0][c] * f[0] + s_o[1][c] * f[1] + s_o[2][c] * f[2] +
                               s_o[3][c] * f[3]) / sum
                            : 0.0f;
        }
        reinterpret_cast<uint32_t*>(a.out + row * D)[threadIdx.x] = pack16<DTYPE>(y[0], y[1]);
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = seen > 0 ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

}  // namespace

cudaError_t launch_cache_attend(const CacheGeom& g, const AttendArgs& a, cudaStream_t st)
{
    const dim3 grid(a.tokens, g.hq);
    const int key = (g.dtype == BACON_FP16) << 2 | (g.format == BACON_INT8) << 1 | (g.d == 128);
    switch (key) {
        case 0: return launch_first(attend_kernel<BACON_BF16, BACON_E4M3, 64>, grid, 128, 0, st, g, a);
        case 1: return launch_first(attend_kernel<BACON_BF16, BACON_E4M3, 128>, grid, 128, 0, st, g, a);
        case 2: return launch_first(attend_kernel<BACON_BF16, BACON_INT8, 64>, grid, 128, 0, st, g, a);
        case 3: return launch_first(attend_kernel<BACON_BF16, BACON_INT8, 128>, grid, 128, 0, st, g, a);
        case 4: return launch_first(attend_kernel<BACON_FP16, BACON_E4M3, 64>, grid, 128, 0, st, g, a);
        case 5: return launch_first(attend_kernel<BACON_FP16, BACON_E4M3, 128>, grid, 128, 0, st, g, a);
        case 6: return launch_first(attend_kernel<BACON_FP16, BACON_INT8, 64>, grid, 128, 0, st, g, a);
        default: return launch_first(attend_kernel<BACON_FP16, BACON_INT8, 128>, grid, 128, 0, st, g, a);
    }
}

}  // namespace bacon
