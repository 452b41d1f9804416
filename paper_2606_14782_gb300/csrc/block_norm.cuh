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
    return g > -INFINITY ? g * s : 0.0f;  // the limit
}

struct Norm {
    int kind;
    const void* weight;
    const void* bias;
};

}  // namespace
}  // namespace bacon
