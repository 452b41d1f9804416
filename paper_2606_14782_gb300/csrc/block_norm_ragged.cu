// Between two blocks (block_norm.cu): rows of odd widths, or that start anywhere.  A
// thread has every threads-th channel of its row, so that a warp's accesses are of
// neighbours wherever the row starts; they are two or four bytes a lane.  2049 rows of
// 1111 channels, layer norms on both sides, fp16 with the sum in fp32: 11.7 us for 4.1
// of bytes; a row is a chain of its loads and four sums over a block, of which an SM
// has seven at a time.  (16-byte pieces whose ends are read value by value, with
// weights shifted into place: 16.3 us, three times the instructions.)  Wider rows spill 40
// bytes a thread from 8193 channels on and 196 from 16385 on: 2000 layer norms of 12001
// channels 112 us for 28, of 20001 358 for 47.
#include "block_norm.cuh"

namespace bacon {
namespace {

// Weights and biases of a norm.
template <int DTYPE, int COUNT>
__device__ __forceinline__ void weigh(const bacon_block& b, const Norm& n, int first, int step, float (&v)[COUNT])
{
    float w[COUNT];
    const auto load = [&](const void* from) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int e = first + i * step;
            w[i] = e < b.width ? load_one<DTYPE>(from, e) : 0.0f;
        }
    };
    if (n.weight) {
        load(n.weight);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] *= b.weight_offset + w[i];  // (0 stays 0)
    }
    if (n.bias) {
        load(n.bias);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] += w[i];
    }
}

// v becomes its norm; channels that are not there are 0 and stay so.
template <int DTYPE, int COUNT, typename SUM>
__device__ __forceinline__ void normalise(const bacon_block& b, float per_channel, const Norm& n, int first,
                                          int step, SUM& sum, float (&v)[COUNT])
{
    const bool layer = n.kind == BACON_NORM_LAYER;
    float mean = 0.0f, inverse, eps = b.eps;
    for (int pass = 0;; ++pass) {
        if (layer) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) s += v[i];
            mean = mean_of(sum(s), b.width, per_channel, pass > 0);
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const float x = first + i * step < b.width ? v[i] - mean : 0.0f;
            s = fmaf(x, x, s);
        }
        const float squares = sum(s), square = fmaf(squares, per_channel, eps);
        inverse = rsqrtf(square);
        // once more, far smaller or with the mean off (block_norm.cuh)
        const bool over = !(squares < INFINITY) && pass < 1;
        const bool far = layer && pass < 3 && far_off(mean, square);
        if (!over && !far) break;
        if (over) eps = kScaledEps;
        const float by = over ? kScaled : 1.0f, less = far ? mean : 0.0f;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = first + i * step < b.width ? fmaf(v[i], by, -less) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = first + i * step < b.width ? (v[i] - mean) * inverse : 0.0f;
    if (DTYPE != BACON_FP32 && b.weight_dtype == BACON_FP32)
        weigh<BACON_FP32>(b, n, first, step, v);
    else
        weigh<DTYPE>(b, n, first, step, v);
}

template <int DTYPE, int RESIDUAL, int COUNT, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : 1024)
ragged_norm_kernel(const __grid_constant__ bacon_block b, float per_channel)
{
    __shared__ __align__(16) float s_scratch[64];
    if (!WARP) {
        if (threadIdx.x < 64) s_scratch[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    RowSum<WARP> sum{s_scratch, 32};
    const long long t = WARP ? blockIdx.x * 4LL + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && t >= b.tokens) return;
    constexpr int kBytes = Eight<DTYPE>::kBytes, kWide = Eight<RESIDUAL>::kBytes;
    const int first = WARP ? threadIdx.x & 31 : threadIdx.x, step = WARP ? 32 : blockDim.x;
    const char* const y = static_cast<const char*>(b.y) + t * b.y_token * kBytes;
    const char* const x_row = static_cast<const char*>(b.x) + t * b.x_token * kWide;
    const char* const gate = static_cast<const char*>(b.gate) + t * b.gate_token * kBytes;
    constexpr bool kEarly = COUNT <= 16;  // x on its way with y: there are registers for it

    float v[COUNT], x[COUNT];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const int e = first + i * step;
        v[i] = e < b.width ? load_one<DTYPE>(y, e) : 0.0f;
        x[i] = kEarly && b.x && e < b.width ? load_one<RESIDUAL>(x_row, e) : 0.0f;
    }
    if (b.post != BACON_NORM_NONE)
        normalise<DTYPE>(b, per_channel, Norm{b.post, b.post_weight, b.post_bias}, first, step, sum, v);
    if (b.gate) {
        const int by = b.gate_channel;
        float g = by ? 0.0f : load_one<DTYPE>(gate, 0);
        if (!by && b.activation != BACON_GATE_LINEAR) g = activate(g, b.activation);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int e = first + i * step;
            if (e >= b.width) continue;
            if (by) {
                g = load_one<DTYPE>(gate, e);
                if (b.activation != BACON_GATE_LINEAR) g = activate(g, b.activation);
            }
            v[i] *= g;
        }
    }
    char* const sum_row = static_cast<char*>(b.sum) + t * b.sum_token * kWide;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const int e = first + i * step;
        if (!kEarly && b.x && e < b.width) x[i] = load_one<RESIDUAL>(x_row, e);
        v[i] = fmaf(b.scale, v[i], x[i]);
        if (b.sum && e < b.width) store_one<RESIDUAL>(sum_row, e, v[i]);
    }
    if (!b.normed) return;
    normalise<DTYPE>(b, per_channel, Norm{b.pre, b.pre_weight, b.pre_bias}, first, step, sum, v);
    char* const row = static_cast<char*>(b.normed) + t * b.normed_token * kBytes;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const int e = first + i * step;
        if (e < b.width) store_one<DTYPE>(row, e, v[i]);
    }
}

template <int DTYPE, int RESIDUAL>
cudaError_t ragged_rows(const bacon_block& b, cudaStream_t st)
{
    const float per_channel = 1.0f / (float)b.width;
    if (b.width <= 256) {
        const unsigned blocks = (unsigned)((b.tokens + 3LL) / 4);
        return launch_first(ragged_norm_kernel<DTYPE, RESIDUAL, 8, true>, blocks, 128, 0, st, b, per_channel);
    }
    // eight channels a thread, or more where a block has too few threads (12 in place of
    // 8 changes nothing, 16 takes 10 % longer)
    const auto threads = [&](int count) { return ((b.width + count - 1) / count + 31) / 32 * 32; };
    if (b.width <= 8192)
        return launch_first(ragged_norm_kernel<DTYPE, RESIDUAL, 8, false>, b.tokens, threads(8), 0, st, b,
                            per_channel);
    if (b.width <= 16384)
        return launch_first(ragged_norm_kernel<DTYPE, RESIDUAL, 16, false>, b.tokens, threads(16), 0, st, b,
                            per_channel);
    return launch_first(ragged_norm_kernel<DTYPE, RESIDUAL, 32, false>, b.tokens, threads(32), 0, st, b,
                        per_channel);
}

}  // namespace

cudaError_t launch_ragged_norm(const bacon_block& b, cudaStream_t st)
{
    const bool wide = b.residual_dtype == BACON_FP32;
    if (b.dtype == BACON_FP32) return ragged_rows<BACON_FP32, BACON_FP32>(b, st);
    if (b.dtype == BACON_BF16)
        return wide ? ragged_rows<BACON_BF16, BACON_FP32>(b, st) : ragged_rows<BACON_BF16, BACON_BF16>(b, st);
    return wide ? ragged_rows<BACON_FP16, BACON_FP32>(b, st) : ragged_rows<BACON_FP16, BACON_FP16>(b, st);
}

}  // namespace bacon
