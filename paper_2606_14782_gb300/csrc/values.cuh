// Eight neighbouring values of a row in any of the three types, as floats.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "bacon.h"
#include "cache_values.cuh"

namespace bacon {

// What eight values take: four words of pairs, or eight of fp32.
template <int DTYPE>
struct Eight {
    static constexpr int kWords = DTYPE == BACON_FP32 ? 8 : 4;
    static constexpr int kBytes = DTYPE == BACON_FP32 ? 4 : 2;  // of a value
    uint32_t w[kWords];
};

// 16-byte aligned.
template <int DTYPE>
__device__ __forceinline__ void load_eight(Eight<DTYPE>& x, const void* p)
{
    const uint4* const q = static_cast<const uint4*>(p);
#pragma unroll
    for (int i = 0; i < Eight<DTYPE>::kWords / 4; ++i) {
        const uint4 v = q[i];
        x.w[4 * i] = v.x;
        x.w[4 * i + 1] = v.y;
        x.w[4 * i + 2] = v.z;
        x.w[4 * i + 3] = v.w;
    }
}
template <int DTYPE>
__device__ __forceinline__ void store_eight(void* p, const Eight<DTYPE>& x)
{
    uint4* const q = static_cast<uint4*>(p);
#pragma unroll
    for (int i = 0; i < Eight<DTYPE>::kWords / 4; ++i)
        q[i] = make_uint4(x.w[4 * i], x.w[4 * i + 1], x.w[4 * i + 2], x.w[4 * i + 3]);
}
template <int DTYPE>
__device__ __forceinline__ void unpack_eight(const Eight<DTYPE>& x, float (&v)[8])
{
    if constexpr (DTYPE == BACON_FP32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(x.w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = unpack16<DTYPE>(x.w[j]);
            v[2 * j] = f.x;
            v[2 * j + 1] = f.y;
        }
    }
}
template <int DTYPE>
__device__ __forceinline__ void pack_eight(Eight<DTYPE>& x, const float (&v)[8])
{
    if constexpr (DTYPE == BACON_FP32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.w[j] = __float_as_uint(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x.w[j] = pack16<DTYPE>(v[2 * j], v[2 * j + 1]);
    }
}

// One value at any address that its type allows.
template <int DTYPE>
__device__ __forceinline__ float load_one(const void* p, long long i)
{
    if constexpr (DTYPE == BACON_FP32) return static_cast<const float*>(p)[i];
    if constexpr (DTYPE == BACON_BF16)
        return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
    return __half2float(static_cast<const __half*>(p)[i]);
}
template <int DTYPE>
__device__ __forceinline__ void store_one(void* p, long long i, float v)
{
    if constexpr (DTYPE == BACON_FP32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<uint16_t*>(p)[i] = static_cast<uint16_t>(pack16<DTYPE>(v, 0.0f));
}
__device__ __forceinline__ float load_any(const void* p, long long i, int dtype)
{
    return dtype == BACON_FP32   ? load_one<BACON_FP32>(p, i)
           : dtype == BACON_BF16 ? load_one<BACON_BF16>(p, i)
                                 : load_one<BACON_FP16>(p, i);
}

// Two floats and what the two-float instructions do with them.
typedef unsigned long long Pair;

__device__ __forceinline__ Pair pair_of(float x, float y)
{
    Pair p;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(p) : "f"(x), "f"(y));
    return p;
}
__device__ __forceinline__ float2 floats_of(Pair p)
{
    float2 f;
    asm("mov.b64 {%0, %1}, %2;\n" : "=f"(f.x), "=f"(f.y) : "l"(p));
    return f;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair p;
    asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(p) : "l"(a), "l"(b), "l"(c));
    return p;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair p;
    asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(p) : "l"(a), "l"(b));
    return p;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair p;
    asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(p) : "l"(a), "l"(b));
    return p;
}

// Eight channels.
struct Piece {
    Pair p[4];
};
template <int DTYPE>
__device__ __forceinline__ void open_piece(const Eight<DTYPE>& raw, Piece& v)
{
    float f[8];
    unpack_eight(raw, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) v.p[j] = pair_of(f[2 * j], f[2 * j + 1]);
}
template <int DTYPE>
__device__ __forceinline__ void close_piece(Eight<DTYPE>& raw, const Piece& v)
{
    float f[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 t = floats_of(v.p[j]);
        f[2 * j] = t.x;
        f[2 * j + 1] = t.y;
    }
    pack_eight(raw, f);
}
__device__ __forceinline__ void set_floats(Piece& v, const float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) v.p[j] = pair_of(f[2 * j], f[2 * j + 1]);
}
__device__ __forceinline__ void get_floats(const Piece& v, float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 t = floats_of(v.p[j]);
        f[2 * j] = t.x;
        f[2 * j + 1] = t.y;
    }
}

}  // namespace bacon
