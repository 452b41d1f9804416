// What the two attention kernels over the 8-bit pages share: the units'
// queries and lengths, page loads, and the exponent that folds V's scale in.
//
// With s_x = scale q . k_x, k_x = sK[page] * code and v_x = sV[page] * code,
//     w_x = 2^(log2e s_x + log2 sV[page] - M),  M the running maximum of that
//                                               exponent,
//     out = sum_x w_x code_x / sum_x (w_x / sV[page]),
//     lse = ln2 (log2 sum_x (w_x / sV[page]) + M):
// one exponential per logit and no multiplication by V's scale.  Codes of
// either format are exact in fp16, and so is a query row scaled by a power of
// two (kQueryTop), so the products are exact and only w is rounded, to fp16's
// 11 bits, the largest at 2^kWeightTop so that it may lie 2^38 below.  Sums
// are fp32.
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

// The queries of one request: [start, start + asked) of the call's tokens.
struct Asked {
    int start, asked;
};

__device__ __forceinline__ Asked asked_of(const AttendArgs& a, int r)
{
    if (!a.starts) {
        const int each = a.tokens / a.requests;
        return Asked{r * each, each};
    }
    const int s = a.starts[r], e = a.starts[r + 1];
    if (s < 0 || e < s || e > a.tokens) return Asked{0, 0};
    return Asked{s, e - s};
}

// Whether the queries' ranges are what they have to be.
__device__ __forceinline__ bool starts_are_bad(const AttendArgs& a, int tid, int threads)
{
    if (!a.starts) return false;
    bool bad = tid == 0 && (a.starts[0] != 0 || a.starts[a.requests] != a.tokens);
    for (int r = tid; r < a.requests; r += threads) bad |= a.starts[r] > a.starts[r + 1];
    return bad;
}

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
    if (!(amax > 0.0f && amax <= 3.0e38f)) return 1.0f;
    int e = (int)(__float_as_uint(amax) >> 23) - 127 - kQueryTop;  // a subnormal: at 2^-127
    e = min(max(e, -110), 120);
    back = __uint_as_float((uint32_t)(e + 127) << 23);
    return __uint_as_float((uint32_t)(127 - e) << 23);
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

}  // namespace bacon
