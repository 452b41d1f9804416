// 8-bit codes of the cache and 16-bit values of its callers.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "bacon.h"
#include "common.cuh"

namespace bacon {

constexpr float kLeastScale = 0x1p-60f;

// Two 16-bit values (bf16 or fp16) as floats.
template <int DTYPE>
__device__ __forceinline__ float2 unpack16(uint32_t w)
{
    if (DTYPE == BACON_BF16)
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    return __half22float2(*reinterpret_cast<__half2*>(&w));
}
template <int DTYPE>
__device__ __forceinline__ uint32_t pack16(float x, float y)
{
    uint32_t w;
    if (DTYPE == BACON_BF16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(w) : "f"(y), "f"(x));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(w) : "f"(y), "f"(x));
    return w;
}

// Two e4m3 codes as fp16 (exact; the NaN code becomes NaN).
__device__ __forceinline__ uint32_t e4m3x2_half2(uint16_t c)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"(c));
    return h;
}
// Four codes of a word as two pairs of fp16 (exact).  int8, by the published
// method of placing an integer in a float's mantissa: the byte with its sign bit
// flipped is u = code + 128; beside the byte 0x64 it is the fp16 1024 + u, and
// 1152 is taken off again.
template <int FORMAT>
__device__ __forceinline__ void codes_half(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    if (FORMAT == BACON_E4M3) {
        lo = e4m3x2_half2(static_cast<uint16_t>(w));
        hi = e4m3x2_half2(static_cast<uint16_t>(w >> 16));
    } else {
        const uint32_t u = w ^ 0x80808080u;
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140);
        const uint32_t b = __byte_perm(u, 0x64646464u, 0x4342);
        const uint32_t off = 0x64806480u;  // 1152
        asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(lo) : "r"(a), "r"(off));
        asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(hi) : "r"(b), "r"(off));
    }
}
template <int FORMAT>
__device__ __forceinline__ float4 codes_float(uint32_t w)
{
    uint32_t lo, hi;
    codes_half<FORMAT>(w, lo, hi);
    const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo));
    const float2 b = __half22float2(*reinterpret_cast<__half2*>(&hi));
    return make_float4(a.x, a.y, b.x, b.y);
}

// The scale of a page whose largest finite magnitude is amax.
template <int FORMAT>
__device__ __forceinline__ float scale_of(float amax)
{
    float s;
    const uint32_t b = __float_as_uint(amax);
    if (FORMAT == BACON_E4M3) {
        // amax = m 2^E with 1 <= m < 2; 448 = 1.75 * 2^8
        const int e = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
        s = e > 0 ? __uint_as_float((uint32_t)e << 23) : 0.0f;
    } else {
        s = __uint_as_float((__float_as_uint(__fdiv_rn(amax, 127.0f)) + 0xFFFFu) & 0xFFFF0000u);
    }
    return fmaxf(s, kLeastScale);
}

// Four values as codes.  `inv` is 1 / scale (exact for e4m3, whose scale is a
// power of two); int8 divides: with 8 significant bits in the scale and at
// most 11 in the value, the rounded quotient is a tie or on a side of one
// exactly when the true quotient is.
template <int FORMAT>
__device__ __forceinline__ uint32_t encode4(float4 x, float scale, float inv)
{
    if (FORMAT == BACON_E4M3) {
        uint16_t a, b;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(a) : "f"(x.y * inv), "f"(x.x * inv));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(b) : "f"(x.w * inv), "f"(x.z * inv));
        return (uint32_t)a | (uint32_t)b << 16;
    }
    const float v[4] = {x.x, x.y, x.z, x.w};
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int c = __float2int_rn(__fdiv_rn(v[i], scale));  // NaN: 0
        c = min(max(c, -127), 127);
        w |= (uint32_t)(c & 0xFF) << (8 * i);
    }
    return w;
}

}  // namespace bacon
