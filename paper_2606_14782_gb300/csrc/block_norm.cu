// Between two blocks: the norm of a block's output, its gate, the residual sum and
// the norm before the next block, one row (token) at a time.  Bound by bytes: y,
// x and a full gate are read once, the sum and its norm written once; a row stays
// in registers between the statistics and their use.
//
// A row belongs to a warp when it is narrow and to a block otherwise.  A thread
// has kChunks pieces of eight channels.  Pieces start at multiples of 16 bytes of
// y's memory: the channels before the first such address and behind the last are
// the ends of pieces that are read value by value, so that odd widths and rows
// that start anywhere still move 16 bytes at a time in between.
#include "block_norm.h"

#include "common.cuh"
#include "values.cuh"

namespace bacon {
namespace {

// Sums over the threads of a row.
template <bool WARP>
struct RowSum {
    float* scratch;  // [2][32]
    int turn = 0;
    __device__ __forceinline__ float operator()(float v)
    {
#pragma unroll
        for (int off = 16; off; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
        if (WARP) return v;
        // two buffers in turn: who writes one again has been past the barrier
        // of the other, which everyone has left the first behind for
        float* const s = scratch + 32 * turn;
        turn ^= 1;
        const int lane = threadIdx.x & 31, warps = blockDim.x / 32;
        if (lane == 0) s[threadIdx.x >> 5] = v;
        __syncthreads();
        v = lane < warps ? s[lane] : 0.0f;
#pragma unroll
        for (int off = 16; off; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
        return v;
    }
};

// A row's pieces: piece i of a thread holds the channels e(i) .. e(i) + 8, of which
// those in [0, width) exist.
struct Pieces {
    int width, lead, first, step;  // lead: channels that piece 0 lies before the row
    bool vectors;
    __device__ __forceinline__ int e(int i) const { return 8 * (first + i * step) - lead; }
    __device__ __forceinline__ bool some(int i) const { return e(i) < width; }
    __device__ __forceinline__ bool whole(int i) const
    {
        return vectors && e(i) >= 0 && e(i) + 8 <= width;
    }
};

template <int DTYPE>
__device__ __forceinline__ void load_piece(const Pieces& p, int i, const void* row, float (&v)[8])
{
    const int e = p.e(i);
    if (p.whole(i)) {
        Eight<DTYPE> raw;
        load_eight(raw, static_cast<const char*>(row) + (long long)e * Eight<DTYPE>::kBytes);
        unpack_eight(raw, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = e + j >= 0 && e + j < p.width ? load_one<DTYPE>(row, e + j) : 0.0f;
    }
}
template <int DTYPE>
__device__ __forceinline__ void store_piece(const Pieces& p, int i, void* row, const float (&v)[8])
{
    const int e = p.e(i);
    if (p.whole(i)) {
        Eight<DTYPE> raw;
        pack_eight(raw, v);
        store_eight(static_cast<char*>(row) + (long long)e * Eight<DTYPE>::kBytes, raw);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (e + j >= 0 && e + j < p.width) store_one<DTYPE>(row, e + j, v[j]);
    }
}
// Weights: the same for all rows, whose pieces start at other channels of them.
__device__ __forceinline__ void load_weights(const Pieces& p, int i, const void* w, int dtype,
                                             bool aligned, float (&v)[8])
{
    const int e = p.e(i);
    if (aligned && p.lead == 0 && p.whole(i)) {
        if (dtype == BACON_FP32) {
            Eight<BACON_FP32> raw;
            load_eight(raw, static_cast<const float*>(w) + e);
            unpack_eight(raw, v);
        } else {
            Eight<BACON_BF16> raw;
            load_eight(raw, static_cast<const uint16_t*>(w) + e);
            if (dtype == BACON_BF16) {
                unpack_eight(raw, v);
            } else {
                Eight<BACON_FP16> half;
#pragma unroll
                for (int j = 0; j < 4; ++j) half.w[j] = raw.w[j];
                unpack_eight(half, v);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = e + j >= 0 && e + j < p.width ? load_any(w, e + j, dtype) : 0.0f;
    }
}

__device__ __forceinline__ float activate(float g, int kind)
{
    if (kind == BACON_GATE_LINEAR) return g;
    if (kind == BACON_GATE_TANH) return tanhf(g);
    const float s = 1.0f / (1.0f + expf(-g));
    if (kind == BACON_GATE_SIGMOID) return s;
    return g > -INFINITY ? g * s : 0.0f;  // the limit
}

struct Norm {
    int kind;
    const void* weight;
    const void* bias;
    bool aligned;
};

// v becomes its norm.
template <int CHUNKS, typename SUM>
__device__ __forceinline__ void normalise(const bacon_block& b, const Norm& n, const Pieces& p,
                                          SUM& sum, float (&v)[CHUNKS][8])
{
    float mean, inverse, eps = b.eps;
    for (int pass = 0; pass < 2; ++pass) {
        mean = 0.0f;
        if (n.kind == BACON_NORM_LAYER) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) s += v[i][j];
            mean = sum(s) / (float)b.width;
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = p.e(i) + j;
                const float x = e >= 0 && e < p.width ? v[i][j] - mean : 0.0f;
                s = fmaf(x, x, s);
            }
        s = sum(s);
        inverse = 1.0f / sqrtf(s / (float)b.width + eps);
        if (s < INFINITY || pass) break;
        // once more with the row far smaller; eps is nothing beside its squares
        eps = 0.0f;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] *= 0x1p-100f;
    }
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        if (!p.some(i)) continue;
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - mean) * inverse;
        if (n.weight) {
            load_weights(p, i, n.weight, b.weight_dtype, n.aligned, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] *= b.weight_offset + w[j];
        }
        if (n.bias) {
            load_weights(p, i, n.bias, b.weight_dtype, n.aligned, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] += w[j];
        }
        // channels that are not there count as 0
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (p.e(i) + j < 0 || p.e(i) + j >= p.width) v[i][j] = 0.0f;
    }
}

struct Choices {
    bool vectors;       // pieces of y, x, gate, sum and normed start at 16 bytes together
    bool post_aligned, pre_aligned, gate_aligned;
};

template <int DTYPE, int RESIDUAL, int CHUNKS, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : 1024)
block_norm_kernel(const __grid_constant__ bacon_block b, const __grid_constant__ Choices choice)
{
    __shared__ float s_scratch[64];
    RowSum<WARP> sum{s_scratch};
    const int t = WARP ? blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && t >= b.tokens) return;
    constexpr int kBytes = Eight<DTYPE>::kBytes, kWide = Eight<RESIDUAL>::kBytes;
    const char* const y = static_cast<const char*>(b.y) + t * b.y_token * kBytes;
    Pieces p;
    p.width = b.width;
    p.vectors = choice.vectors;
    p.lead = choice.vectors ? (int)(reinterpret_cast<uintptr_t>(y) / kBytes) & (16 / kBytes - 1) : 0;
    p.first = WARP ? threadIdx.x & 31 : threadIdx.x;
    p.step = WARP ? 32 : blockDim.x;

    float v[CHUNKS][8], x[CHUNKS][8];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        if (p.some(i))
            load_piece<DTYPE>(p, i, y, v[i]);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
    const char* const x_row = static_cast<const char*>(b.x) + t * b.x_token * kWide;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        if (b.x && p.some(i))
            load_piece<RESIDUAL>(p, i, x_row, x[i]);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = 0.0f;
    }
    if (b.post != BACON_NORM_NONE)
        normalise(b, Norm{b.post, b.post_weight, b.post_bias, choice.post_aligned}, p, sum, v);
    if (b.gate) {
        const char* const gate = static_cast<const char*>(b.gate) + t * b.gate_token * kBytes;
        if (!b.gate_channel) {
            const float g = activate(load_one<DTYPE>(gate, 0), b.activation);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int e = p.e(i) + j;
                    v[i][j] = e >= 0 && e < p.width ? v[i][j] * g : 0.0f;
                }
        } else {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                if (!p.some(i)) continue;
                float g[8];
                if (b.gate_token)
                    load_piece<DTYPE>(p, i, gate, g);
                else
                    load_weights(p, i, gate, b.dtype, choice.gate_aligned, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= activate(g[j], b.activation);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = fmaf(b.scale, v[i][j], x[i][j]);
    if (b.sum) {
        char* const row = static_cast<char*>(b.sum) + t * b.sum_token * kWide;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            if (p.some(i)) store_piece<RESIDUAL>(p, i, row, v[i]);
    }
    if (!b.normed) return;
    normalise(b, Norm{b.pre, b.pre_weight, b.pre_bias, choice.pre_aligned}, p, sum, v);
    char* const row = static_cast<char*>(b.normed) + t * b.normed_token * kBytes;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
        if (p.some(i)) store_piece<DTYPE>(p, i, row, v[i]);
}

// Whether rows at p, `stride` values apart, have pieces that start where y's do.
bool together(const bacon_block& b, const void* p, long long stride, int bytes, int y_bytes)
{
    if (!p) return true;
    const long long unit = 16 / bytes;  // values of 16 bytes
    if (b.tokens > 1 && (stride - b.y_token) % unit) return false;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(b.y);
    return a % bytes == 0 && ((long long)(a / bytes) - (long long)(y / y_bytes)) % unit == 0;
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <int DTYPE, int RESIDUAL>
cudaError_t go(const bacon_block& b, cudaStream_t st)
{
    constexpr int kBytes = Eight<DTYPE>::kBytes, kWide = Eight<RESIDUAL>::kBytes;
    Choices c;
    c.vectors = together(b, b.x, b.x_token, kWide, kBytes) &&
                together(b, b.sum, b.sum_token, kWide, kBytes) &&
                together(b, b.normed, b.normed_token, kBytes, kBytes) &&
                (!b.gate || !b.gate_channel || !b.gate_token ||
                 together(b, b.gate, b.gate_token, kBytes, kBytes));
    c.post_aligned = aligned(b.post_weight) && aligned(b.post_bias);
    c.pre_aligned = aligned(b.pre_weight) && aligned(b.pre_bias);
    c.gate_aligned = aligned(b.gate);
    const int lead = c.vectors ? 16 / kBytes - 1 : 0;
    const int pieces = (b.width + lead + 7) / 8;  // of a row, at most
    if (pieces <= 32 * 4) {
        const unsigned blocks = (unsigned)((b.tokens + 3LL) / 4);
        if (pieces <= 32)
            return launch_first(block_norm_kernel<DTYPE, RESIDUAL, 1, true>, blocks, 128, 0, st, b, c);
        if (pieces <= 64)
            return launch_first(block_norm_kernel<DTYPE, RESIDUAL, 2, true>, blocks, 128, 0, st, b, c);
        return launch_first(block_norm_kernel<DTYPE, RESIDUAL, 4, true>, blocks, 128, 0, st, b, c);
    }
    const int per = pieces <= 1024 ? 1 : pieces <= 2048 ? 2 : 4;
    const unsigned threads = (unsigned)((pieces + per - 1) / per + 31) / 32 * 32;
    if (pieces > 4096) return launch_first(block_norm_kernel<DTYPE, RESIDUAL, 5, false>, b.tokens, 1024, 0, st, b, c);
    if (per == 1)
        return launch_first(block_norm_kernel<DTYPE, RESIDUAL, 1, false>, b.tokens, threads, 0, st, b, c);
    if (per == 2)
        return launch_first(block_norm_kernel<DTYPE, RESIDUAL, 2, false>, b.tokens, threads, 0, st, b, c);
    return launch_first(block_norm_kernel<DTYPE, RESIDUAL, 4, false>, b.tokens, threads, 0, st, b, c);
}

}  // namespace

cudaError_t launch_block_norm(const bacon_block& b, cudaStream_t st)
{
    const bool wide = b.residual_dtype == BACON_FP32;
    if (b.dtype == BACON_BF16)
        return wide ? go<BACON_BF16, BACON_FP32>(b, st) : go<BACON_BF16, BACON_BF16>(b, st);
    if (b.dtype == BACON_FP16)
        return wide ? go<BACON_FP16, BACON_FP32>(b, st) : go<BACON_FP16, BACON_FP16>(b, st);
    return go<BACON_FP32, BACON_FP32>(b, st);
}

}  // namespace bacon
