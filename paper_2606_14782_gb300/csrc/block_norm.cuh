// What both kernels of the step between two blocks share.
#pragma once

#include "block_norm.h"
#include "common.cuh"
#include "values.cuh"

namespace bacon {
namespace {

// Sums over the threads of a row.
template <bool WARP>
struct RowSum {
    float* scratch;  // [2][32], zeros beyond the block's warps
    int lanes;       // of a row that has a warp's, a power of two
    int turn = 0;
    __device__ __forceinline__ float operator()(float v)
    {
        for (int off = (WARP ? lanes : 32) / 2; off; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
        if (WARP) return v;
        // two buffers in turn: who writes one again has been past the barrier
        // of the other, which everyone has left the first behind for
        float* const s = scratch + 32 * turn;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
        __syncthreads();
        const float4* const q = reinterpret_cast<const float4*>(s);
        float4 a = q[0];
        for (int i = 1; i < ((int)blockDim.x + 127) / 128; ++i) {
            const float4 c = q[i];
            a.x += c.x;
            a.y += c.y;
            a.z += c.z;
            a.w += c.w;
        }
        return (a.x + a.y) + (a.z + a.w);
    }
};

__device__ __forceinline__ float activate(float g, int kind)
{
    if (kind == BACON_GATE_TANH) return tanhf(g);
    const float s = 1.0f / (1.0f + expf(-g));
    if (kind == BACON_GATE_SIGMOID) return s;
    return g == -INFINITY ? 0.0f : g * s;  // the limit
}

// Statistics of rows that fp32 has no room for.  A row whose squares pass 3e38 is scaled
// by kScaled and gone through again; eps is nothing beside its mean square then, but
// where that is 0 (a row of one value and its mean) it keeps the root from being
// infinite.  A row that lies far off 0 for its spread has a mean whose rounding would
// show beside that spread: the mean is taken off the values, nearly all of them
// exactly, and the row gone through again; a row of one value is 0 then.  From 64 times
// the spread on, so that a mean off by 2^-22 of itself is off by 2^-16 of the spread.
constexpr float kScaled = 0x1p-100f, kScaledEps = 0x1p-126f;
__device__ __forceinline__ bool far_off(float mean, float square) { return square < mean * mean * 0x1p-12f; }

// sum / width; of a row gone through again with one step of correction: exact where the
// quotient is.
__device__ __forceinline__ float mean_of(float sum, int width, float per_channel, bool again)
{
    const float mean = sum * per_channel;
    return again ? fmaf(fmaf(-mean, (float)width, sum), per_channel, mean) : mean;
}

struct Norm {
    int kind;
    const void* weight;
    const void* bias;
};

}  // namespace
}  // namespace bacon
