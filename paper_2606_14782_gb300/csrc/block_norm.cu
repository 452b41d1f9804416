// Between two blocks: the norm of a block's output, its gate, the residual sum and
// the norm before the next block, one row (token) at a time.  Bound by bytes: y,
// x and a full gate are read once, the sum and its norm written once; a row stays
// in registers between the statistics and their use.
//
// Here are rows of whole pieces of eight channels that start at multiples of 16
// bytes (others: block_norm_ragged.cu).  A row belongs to some or all lanes of a warp
// when it is narrow and to a block otherwise, a thread has CHUNKS pieces of it as
// pairs of floats: products and sums are the two-float instructions, since what is
// left of the bound after the bytes is issuing instructions.  Blocks stay and go from row
// to row, and the next row is on its way while one is worked on (to four pieces).  65536 rows of 3584 channels,
// RMS norms on both sides and a gate, bf16: 292 us, 95 % of the measured copy
// bandwidth (one row after the other: 541; without TIGHT, below: 421); one row 2.3 us,
// a launch and the latency of a row's loads and its sums.  With the sum in fp32, 32768
// rows: 228 us for 209 of bytes (40 bytes a thread are spilled); in fp32, 16384 rows of
// 4096: 215 for 159 (120 bytes).  Eight pieces (over 16384 channels) spill 84 to 100
// bytes and have no row ahead: 2000 rows of 20000 81 us for 47.
#include "block_norm.cuh"

namespace bacon {
namespace {

// A row's pieces: piece i of a thread holds the channels e(i) .. e(i) + 8, which
// exist if e(i) < width.  TIGHT: all but the last are known to.
template <int CHUNKS, bool TIGHT>
struct Pieces {
    int width, first, step;
    __device__ __forceinline__ int e(int i) const { return 8 * (first + i * step); }
    __device__ __forceinline__ bool some(int i) const { return (TIGHT && i < CHUNKS - 1) || e(i) < width; }
};

template <int DTYPE>
__device__ __forceinline__ void load_piece(const void* row, int e, Piece& v)
{
    Eight<DTYPE> raw;
    load_eight(raw, static_cast<const char*>(row) + (long long)e * Eight<DTYPE>::kBytes);
    open_piece(raw, v);
}
template <int DTYPE>
__device__ __forceinline__ void store_piece(char* row, int e, const Piece& v)
{
    Eight<DTYPE> raw;
    close_piece(raw, v);
    store_eight(row + (long long)e * Eight<DTYPE>::kBytes, raw);
}

// Weights and biases of a norm.
template <int DTYPE, int CHUNKS, bool TIGHT>
__device__ __forceinline__ void weigh(const bacon_block& b, const Norm& n, const Pieces<CHUNKS, TIGHT>& p,
                                      Piece (&v)[CHUNKS])
{
    const Pair offset = pair_of(b.weight_offset, b.weight_offset);
    Piece w;
    if (n.weight) {
        if (b.weight_offset == 0.0f) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) {
                    load_piece<DTYPE>(n.weight, p.e(i), w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], w.p[j]);
                }
        } else {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) {
                    load_piece<DTYPE>(n.weight, p.e(i), w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], add2(w.p[j], offset));
                }
        }
    }
    if (n.bias)
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            if (p.some(i)) {
                load_piece<DTYPE>(n.bias, p.e(i), w);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = add2(v[i].p[j], w.p[j]);
            }
}

// v becomes its norm.
template <int DTYPE, int CHUNKS, bool TIGHT, typename SUM>
__device__ __forceinline__ void normalise(const bacon_block& b, float per_channel, const Norm& n,
                                          const Pieces<CHUNKS, TIGHT>& p, SUM& sum, Piece (&v)[CHUNKS])
{
    const bool layer = n.kind == BACON_NORM_LAYER;
    float mean = 0.0f, inverse, eps = b.eps;
    bool again = false;  // this row has been gone through before, and not for others alone
    for (int pass = 0;; ++pass) {
        if (layer) {
            Pair s = 0;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s = add2(s, v[i].p[j]);
            const float2 f = floats_of(s);
            mean = mean_of(sum(f.x + f.y), b.width, per_channel, again);
        }
        Pair s = 0;
        const Pair off = pair_of(-mean, -mean);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Pair x = v[i].p[j];
                if (layer) x = p.some(i) ? add2(x, off) : 0;
                s = fma2(x, x, s);
            }
        const float2 f = floats_of(s);
        const float squares = sum(f.x + f.y), square = fmaf(squares, per_channel, eps);
        inverse = rsqrtf(square);
        // once more, far smaller or with the mean off (block_norm.cuh).  The rows of a
        // warp go together, and the others find again what they had
        const bool over = !(squares < INFINITY) && pass < 1;
        const bool far = layer && pass < 3 && far_off(mean, square);
        if (TIGHT ? !(over || far) : !__any_sync(0xFFFFFFFFu, over || far)) break;
        again |= over || far;
        if (over) eps = kScaledEps;
        const float by = over ? kScaled : 1.0f, less = far ? -mean : -0.0f;
        const Pair times = pair_of(by, by), plus = pair_of(less, less);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].p[j] = p.some(i) ? fma2(v[i].p[j], times, plus) : 0;
    }
    const Pair by = pair_of(inverse, inverse), off = pair_of(-mean, -mean);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // channels that are not there stay 0
            if (layer) v[i].p[j] = p.some(i) ? add2(v[i].p[j], off) : 0;
            v[i].p[j] = mul2(v[i].p[j], by);
        }
    if (DTYPE != BACON_FP32 && b.weight_dtype == BACON_FP32)
        weigh<BACON_FP32>(b, n, p, v);
    else
        weigh<DTYPE>(b, n, p, v);
}

constexpr int most_threads(bool warp) { return warp ? 128 : 512; }

template <int DTYPE, int RESIDUAL, int CHUNKS, bool WARP>
__global__ void __launch_bounds__(most_threads(WARP))
block_norm_kernel(const __grid_constant__ bacon_block b, float per_channel, int lanes)
{
    __shared__ __align__(16) float s_scratch[64];
    if (!WARP) {
        if (threadIdx.x < 64) s_scratch[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    RowSum<WARP> sum{s_scratch, lanes};
    constexpr int kBytes = Eight<DTYPE>::kBytes, kWide = Eight<RESIDUAL>::kBytes;
    Pieces<CHUNKS, !WARP> p;
    p.width = b.width;
    p.first = WARP ? threadIdx.x & (lanes - 1) : threadIdx.x;
    p.step = WARP ? lanes : blockDim.x;
    const int rows = WARP ? blockDim.x / lanes : 1;
    const long long apart = (long long)gridDim.x * rows;
    long long t = (long long)blockIdx.x * rows + (WARP ? threadIdx.x / lanes : 0);
    // the first row of the warp: all of its rows go round together, those that are
    // not there as rows of no channels
    long long first = WARP ? t - (threadIdx.x & 31) / lanes : t;

    // a row ahead, where rows leave registers for it
    constexpr bool kAhead = CHUNKS <= 4;
    Eight<DTYPE> y_next[kAhead ? CHUNKS : 1];
    Eight<RESIDUAL> x_next[kAhead ? CHUNKS : 1];
    auto fetch = [&](long long row) {
        const char* const y = static_cast<const char*>(b.y) + row * b.y_token * kBytes;
        const char* const x = static_cast<const char*>(b.x) + row * b.x_token * kWide;
        p.width = !WARP || row < b.tokens ? b.width : 0;
#pragma unroll
        for (int i = 0; i < (kAhead ? CHUNKS : 1); ++i)
            if (p.some(i)) {
                load_eight(y_next[i], y + (long long)p.e(i) * kBytes);
                if (b.x) load_eight(x_next[i], x + (long long)p.e(i) * kWide);
            }
    };
    if (kAhead) {
#pragma unroll
        for (int i = 0; i < (kAhead ? CHUNKS : 1); ++i) {
#pragma unroll
            for (int j = 0; j < Eight<DTYPE>::kWords; ++j) y_next[i].w[j] = 0;
#pragma unroll
            for (int j = 0; j < Eight<RESIDUAL>::kWords; ++j) x_next[i].w[j] = 0;
        }
        if (first < b.tokens) fetch(t);
    }
    for (; first < b.tokens; t += apart, first += apart) {
        Piece v[CHUNKS], x[CHUNKS];
        const char* const y = static_cast<const char*>(b.y) + t * b.y_token * kBytes;
        const char* const x_row = static_cast<const char*>(b.x) + t * b.x_token * kWide;
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                open_piece(y_next[i], v[i]);
                open_piece(x_next[i], x[i]);
            }
            if (first + apart < b.tokens) fetch(t + apart);
            p.width = !WARP || t < b.tokens ? b.width : 0;
        } else {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = x[i].p[j] = 0;
                if (p.some(i)) load_piece<DTYPE>(y, p.e(i), v[i]);
            }
        }
        if (b.post != BACON_NORM_NONE)
            normalise<DTYPE>(b, per_channel, Norm{b.post, b.post_weight, b.post_bias}, p, sum, v);
        const char* const gate = static_cast<const char*>(b.gate) + t * b.gate_token * kBytes;
        if (b.gate && !b.gate_channel) {
            const float g = p.width ? load_one<DTYPE>(gate, 0) : 0.0f;
            const float a = b.activation == BACON_GATE_LINEAR ? g : activate(g, b.activation);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i))
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], pair_of(a, a));
        }
        if (b.gate && b.gate_channel) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                if (!p.some(i)) continue;
                Piece g;
                load_piece<DTYPE>(gate, p.e(i), g);
                if (b.activation != BACON_GATE_LINEAR) {
                    float f[8];
                    get_floats(g, f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = activate(f[j], b.activation);
                    set_floats(g, f);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], g.p[j]);
            }
        }
        const Pair scale = pair_of(b.scale, b.scale);
        if (!kAhead && b.x)
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) load_piece<RESIDUAL>(x_row, p.e(i), x[i]);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].p[j] = fma2(scale, v[i].p[j], x[i].p[j]);
        if (b.sum) {
            char* const row = static_cast<char*>(b.sum) + t * b.sum_token * kWide;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) store_piece<RESIDUAL>(row, p.e(i), v[i]);
        }
        if (!b.normed) continue;
        normalise<DTYPE>(b, per_channel, Norm{b.pre, b.pre_weight, b.pre_bias}, p, sum, v);
        char* const row = static_cast<char*>(b.normed) + t * b.normed_token * kBytes;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            if (p.some(i)) store_piece<DTYPE>(row, p.e(i), v[i]);
    }
}

template <int DTYPE, int RESIDUAL, int CHUNKS, bool WARP>
cudaError_t launch_rows(const bacon_block& b, int pieces, cudaStream_t st)
{
    int lanes = 32;  // of a narrow row: several rows a warp
    while (WARP && CHUNKS == 1 && lanes / 2 >= pieces) lanes /= 2;
    const int threads = WARP ? 128 : ((pieces + CHUNKS - 1) / CHUNKS + 31) / 32 * 32;
    const long long rows = WARP ? 128 / lanes : 1, wanted = (b.tokens + rows - 1) / rows;
    // as many blocks as the registers leave room for, if there are as many rows
    const long long most = 152LL * (!WARP ? 512 : CHUNKS == 1 ? 1024 : 384) / threads;
    const long long blocks = wanted < most || CHUNKS > 4 ? wanted : most;
    return launch_first(block_norm_kernel<DTYPE, RESIDUAL, CHUNKS, WARP>, (unsigned)blocks, threads, 0, st, b,
                        1.0f / (float)b.width, lanes);
}

template <int DTYPE, int RESIDUAL>
cudaError_t whole_rows(const bacon_block& b, cudaStream_t st)
{
    const int pieces = b.width / 8;
    if (pieces <= 32) return launch_rows<DTYPE, RESIDUAL, 1, true>(b, pieces, st);
    if (pieces <= 128) return launch_rows<DTYPE, RESIDUAL, 4, true>(b, pieces, st);
    // By the width alone, so that a row's bits do not depend on how many there are (one
    // piece a thread for few rows: 2.8 us for 3.1 of 32 rows of 2048, 4.0 for 3.8 of
    // 8192): the most pieces a thread of which all but the last are there in every
    // thread.  Fewer threads a row have fewer sums to share (two pieces: 566 us for 422
    // of the largest case, before pieces were known to exist).
    const auto tight = [&](int chunks) {
        const int threads = ((pieces + chunks - 1) / chunks + 31) / 32 * 32;
        return threads <= 512 && (chunks - 1) * threads <= pieces;
    };
    if (tight(4)) return launch_rows<DTYPE, RESIDUAL, 4, false>(b, pieces, st);
    if (tight(3)) return launch_rows<DTYPE, RESIDUAL, 3, false>(b, pieces, st);
    if (tight(2)) return launch_rows<DTYPE, RESIDUAL, 2, false>(b, pieces, st);
    return launch_rows<DTYPE, RESIDUAL, 8, false>(b, pieces, st);
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

cudaError_t launch_block_norm(const bacon_block& b, cudaStream_t st)
{
    const int bytes = b.dtype == BACON_FP32 ? 4 : 2, wide = b.residual_dtype == BACON_FP32 ? 4 : 2;
    const auto rows = [&](const void* p, long long stride, int size) {
        // (of one row too, so that it is the row that it is among others)
        return !p || (aligned(p) && stride * size % 16 == 0);
    };
    const bool whole = b.width % 8 == 0 && rows(b.y, b.y_token, bytes) && rows(b.x, b.x_token, wide) &&
                       rows(b.sum, b.sum_token, wide) && rows(b.normed, b.normed_token, bytes) &&
                       (!b.gate_channel || rows(b.gate, b.gate_token, bytes)) && aligned(b.post_weight) &&
                       aligned(b.post_bias) && aligned(b.pre_weight) && aligned(b.pre_bias);
    if (!whole) return launch_ragged_norm(b, st);
    if (b.dtype == BACON_FP32) return whole_rows<BACON_FP32, BACON_FP32>(b, st);
    if (b.dtype == BACON_BF16)
        return wide == 4 ? whole_rows<BACON_BF16, BACON_FP32>(b, st) : whole_rows<BACON_BF16, BACON_BF16>(b, st);
    return wide == 4 ? whole_rows<BACON_FP16, BACON_FP32>(b, st) : whole_rows<BACON_FP16, BACON_FP16>(b, st);
}

}  // namespace bacon
