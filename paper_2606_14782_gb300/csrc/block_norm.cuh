// The kernel of the step between two blocks, one row (token) at a time.  Bound by
// bytes: y, x and a full gate are read once, the sum and its norm written once; a
// row stays in registers between the statistics and their use.
//
// A row belongs to a warp when it is narrow and to a block otherwise.  A thread
// has CHUNKS pieces of eight channels, as four pairs of floats: products and sums
// are the two-float instructions, since what is left of the bound after the bytes
// is issuing instructions.  Blocks stay and go from row to row; the next row is on
// its way while one is worked on.
//
// Where rows do not start at multiples of 16 bytes (odd widths), pieces start at
// such addresses of y all the same: the channels before the first and behind the
// last are the ends of pieces that are read value by value, and 16 bytes move at a
// time in between.
#pragma once

#include "block_norm.h"
#include "common.cuh"
#include "values.cuh"

namespace bacon {
namespace {

// ------------------------------------------------------------ pairs of floats

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
__device__ __forceinline__ void open(const Eight<DTYPE>& raw, Piece& v)
{
    float f[8];
    unpack_eight(raw, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) v.p[j] = pair_of(f[2 * j], f[2 * j + 1]);
}
template <int DTYPE>
__device__ __forceinline__ void close(Eight<DTYPE>& raw, const Piece& v)
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

// ------------------------------------------------------------------- a row

// Sums over the threads of a row.
template <bool WARP>
struct RowSum {
    float* scratch;  // [2][32], zeros beyond the block's warps
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

// A row's pieces: piece i of a thread holds the channels e(i) .. e(i) + 8, of which
// those in [0, width) exist.  EVEN: all of a piece or nothing.
template <int CHUNKS, bool EVEN, bool TIGHT>
struct Pieces {
    // a block's even rows: the host chooses CHUNKS so that all but the last exist
    static constexpr bool kTight = TIGHT;
    int width, lead, first, step;  // lead: channels that piece 0 lies before the row
    bool vectors;
    __device__ __forceinline__ int e(int i) const { return 8 * (first + i * step) - (EVEN ? 0 : lead); }
    __device__ __forceinline__ bool some(int i) const
    {
        return (EVEN && kTight && i < CHUNKS - 1) || e(i) < width;
    }
    __device__ __forceinline__ bool all(int i) const
    {
        return EVEN ? some(i) : e(i) >= 0 && e(i) + 8 <= width;
    }
    __device__ __forceinline__ bool has(int i, int j) const { return e(i) + j >= 0 && e(i) + j < width; }
    // channels that are not there are 0
    __device__ __forceinline__ void trim(int i, Piece& v) const
    {
        if (all(i)) return;
        float f[8];
        get_floats(v, f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (EVEN || !has(i, j)) f[j] = 0.0f;
        set_floats(v, f);
    }
};

template <int DTYPE, int CHUNKS, bool EVEN, bool TIGHT>
__device__ __forceinline__ void load_piece(const Pieces<CHUNKS, EVEN, TIGHT>& p, int i, const char* row, Piece& v)
{
    const int e = p.e(i);
    if (EVEN || (p.vectors && p.all(i))) {
        Eight<DTYPE> raw;
        load_eight(raw, row + (long long)e * Eight<DTYPE>::kBytes);
        open(raw, v);
    } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = p.has(i, j) ? load_one<DTYPE>(row, e + j) : 0.0f;
        set_floats(v, f);
    }
}
template <int DTYPE, int CHUNKS, bool EVEN, bool TIGHT>
__device__ __forceinline__ void store_piece(const Pieces<CHUNKS, EVEN, TIGHT>& p, int i, char* row, const Piece& v)
{
    const int e = p.e(i);
    if (EVEN || (p.vectors && p.all(i))) {
        Eight<DTYPE> raw;
        close(raw, v);
        store_eight(row + (long long)e * Eight<DTYPE>::kBytes, raw);
    } else {
        float f[8];
        get_floats(v, f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (p.has(i, j)) store_one<DTYPE>(row, e + j, f[j]);
    }
}

// Values e .. e + 8 of an array that starts at 16 bytes, e anything >= 0: the two
// (fp32: three) groups of 16 bytes that hold them, shifted in three steps.
template <int DTYPE>
__device__ __forceinline__ void load_shifted(const char* w, int e, Piece& v)
{
    constexpr int kUnit = 16 / Eight<DTYPE>::kBytes, kWords = Eight<DTYPE>::kWords + 4;
    const uint4* const q = reinterpret_cast<const uint4*>(w) + e / kUnit;
    uint32_t x[kWords];
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
        const uint4 t = q[i];
        x[4 * i] = t.x;
        x[4 * i + 1] = t.y;
        x[4 * i + 2] = t.z;
        x[4 * i + 3] = t.w;
    }
    const int words = e % kUnit * Eight<DTYPE>::kBytes / 4;
    Eight<DTYPE> raw;
    if (words & 2)
#pragma unroll
        for (int i = 0; i + 2 < kWords; ++i) x[i] = x[i + 2];
    if (words & 1)
#pragma unroll
        for (int i = 0; i + 1 < kWords; ++i) x[i] = x[i + 1];
#pragma unroll
    for (int i = 0; i < Eight<DTYPE>::kWords; ++i)
        raw.w[i] = DTYPE != BACON_FP32 && (e & 1) ? __funnelshift_r(x[i], x[i + 1], 16) : x[i];
    open(raw, v);
}

// Weights, biases and a shared gate: the same for all rows, whose pieces may start
// at other channels of them.
template <int DTYPE, int CHUNKS, bool EVEN, bool TIGHT>
__device__ __forceinline__ void load_shared(const Pieces<CHUNKS, EVEN, TIGHT>& p, int i, const void* w, bool aligned, Piece& v)
{
    const int e = p.e(i);
    const char* const at = static_cast<const char*>(w);
    constexpr int kUnit = 16 / Eight<DTYPE>::kBytes;
    if (EVEN) {
        Eight<DTYPE> raw;
        load_eight(raw, at + (long long)e * Eight<DTYPE>::kBytes);
        open(raw, v);
    } else if (aligned && e >= 0 && e / kUnit * kUnit + 8 + kUnit <= p.width) {
        load_shifted<DTYPE>(at, e, v);
    } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = p.has(i, j) ? load_one<DTYPE>(w, e + j) : 0.0f;
        set_floats(v, f);
    }
}
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
    bool aligned;
};

// Weights and biases of a norm.
template <int DTYPE, int CHUNKS, bool EVEN, bool TIGHT>
__device__ __forceinline__ void weigh(const bacon_block& b, const Norm& n, const Pieces<CHUNKS, EVEN, TIGHT>& p,
                                      Piece (&v)[CHUNKS])
{
    const Pair offset = pair_of(b.weight_offset, b.weight_offset);
    Piece w;
    if (n.weight) {
        if (b.weight_offset == 0.0f) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) {
                    load_shared<DTYPE>(p, i, n.weight, n.aligned, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], w.p[j]);
                }
        } else {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) {
                    load_shared<DTYPE>(p, i, n.weight, n.aligned, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], add2(w.p[j], offset));
                }
        }
    }
    if (n.bias)
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            if (p.some(i)) {
                load_shared<DTYPE>(p, i, n.bias, n.aligned, w);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = add2(v[i].p[j], w.p[j]);
            }
}

// v becomes its norm.
template <int DTYPE, int CHUNKS, bool EVEN, bool TIGHT, typename SUM>
__device__ __forceinline__ void normalise(const bacon_block& b, float per_channel, const Norm& n,
                                          const Pieces<CHUNKS, EVEN, TIGHT>& p, SUM& sum, Piece (&v)[CHUNKS])
{
    float inverse, eps = b.eps;
    for (int pass = 0;; ++pass) {
        if (n.kind == BACON_NORM_LAYER) {
            Pair s = 0;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s = add2(s, v[i].p[j]);
            const float2 f = floats_of(s);
            const float mean = sum(f.x + f.y) * per_channel;
            const Pair off = pair_of(-mean, -mean);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = add2(v[i].p[j], off);
                p.trim(i, v[i]);
            }
        }
        Pair s = 0;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s = fma2(v[i].p[j], v[i].p[j], s);
        const float2 f = floats_of(s);
        const float squares = sum(f.x + f.y);
        inverse = rsqrtf(fmaf(squares, per_channel, eps));
        if (squares < INFINITY || pass) break;
        // once more with the row far smaller; eps is nothing beside its squares
        eps = 0.0f;
        const Pair small = pair_of(0x1p-100f, 0x1p-100f);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], small);
    }
    const Pair by = pair_of(inverse, inverse);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], by);
    if (DTYPE != BACON_FP32 && b.weight_dtype == BACON_FP32)
        weigh<BACON_FP32>(b, n, p, v);
    else
        weigh<DTYPE>(b, n, p, v);
    if (!EVEN)
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) p.trim(i, v[i]);
}

constexpr int most_threads(int chunks, bool warp) { return warp ? 128 : chunks == 1 ? 1024 : 512; }

template <int DTYPE, int RESIDUAL, int CHUNKS, bool WARP, bool EVEN>
__global__ void __launch_bounds__(most_threads(CHUNKS, WARP))
block_norm_kernel(const __grid_constant__ bacon_block b, const __grid_constant__ Choices choice)
{
    __shared__ __align__(16) float s_scratch[64];
    if (!WARP) {
        if (threadIdx.x < 64) s_scratch[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    RowSum<WARP> sum{s_scratch};
    constexpr int kBytes = Eight<DTYPE>::kBytes, kWide = Eight<RESIDUAL>::kBytes;
    Pieces<CHUNKS, EVEN, !WARP> p;
    p.width = b.width;
    p.vectors = choice.vectors;
    p.first = WARP ? threadIdx.x & 31 : threadIdx.x;
    p.step = WARP ? 32 : blockDim.x;
    const int rows = WARP ? blockDim.x / 32 : 1;
    const long long apart = (long long)gridDim.x * rows;
    long long t = (long long)blockIdx.x * rows + (WARP ? threadIdx.x >> 5 : 0);

    // a row ahead, where rows are even and leave registers for it
    constexpr bool kAhead = EVEN && CHUNKS <= 4, kEarly = CHUNKS <= 4;
    Eight<DTYPE> y_next[kAhead ? CHUNKS : 1];
    Eight<RESIDUAL> x_next[kAhead ? CHUNKS : 1];
    auto fetch = [&](long long row) {
        const char* const y = static_cast<const char*>(b.y) + row * b.y_token * kBytes;
        const char* const x = static_cast<const char*>(b.x) + row * b.x_token * kWide;
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
        if (t < b.tokens) fetch(t);
    }
    for (; t < b.tokens; t += apart) {
        Piece v[CHUNKS], x[CHUNKS];
        const char* const y = static_cast<const char*>(b.y) + t * b.y_token * kBytes;
        const char* const x_row = static_cast<const char*>(b.x) + t * b.x_token * kWide;
        p.lead = !EVEN && choice.vectors ? (int)(reinterpret_cast<uintptr_t>(y) / kBytes) & (16 / kBytes - 1) : 0;
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                open(y_next[i], v[i]);
                open(x_next[i], x[i]);
            }
            if (t + apart < b.tokens) fetch(t + apart);
        } else {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = x[i].p[j] = 0;
                if (!p.some(i)) continue;
                load_piece<DTYPE>(p, i, y, v[i]);
                if (kEarly && b.x) load_piece<RESIDUAL>(p, i, x_row, x[i]);
            }
        }
        if (b.post != BACON_NORM_NONE)
            normalise<DTYPE>(b, choice.per_channel, Norm{b.post, b.post_weight, b.post_bias, choice.post_aligned},
                             p, sum, v);
        const char* const gate = static_cast<const char*>(b.gate) + t * b.gate_token * kBytes;
        if (b.gate && !b.gate_channel) {
            const float g = load_one<DTYPE>(gate, 0);
            const float a = b.activation == BACON_GATE_LINEAR ? g : activate(g, b.activation);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(v[i].p[j], pair_of(a, a));
                p.trim(i, v[i]);
            }
        }
        if (b.gate && b.gate_channel) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                if (!p.some(i)) continue;
                Piece g;
                if (EVEN || b.gate_token)
                    load_piece<DTYPE>(p, i, gate, g);
                else
                    load_shared<DTYPE>(p, i, gate, choice.gate_aligned, g);
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
        if (!kEarly && b.x)
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) load_piece<RESIDUAL>(p, i, x_row, x[i]);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i].p[j] = fma2(scale, v[i].p[j], x[i].p[j]);
        if (b.sum) {
            char* const row = static_cast<char*>(b.sum) + t * b.sum_token * kWide;
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i)
                if (p.some(i)) store_piece<RESIDUAL>(p, i, row, v[i]);
        }
        if (!b.normed) continue;
        normalise<DTYPE>(b, choice.per_channel, Norm{b.pre, b.pre_weight, b.pre_bias, choice.pre_aligned}, p,
                         sum, v);
        char* const row = static_cast<char*>(b.normed) + t * b.normed_token * kBytes;
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i)
            if (p.some(i)) store_piece<DTYPE>(p, i, row, v[i]);
    }
}

template <int DTYPE, int RESIDUAL, int CHUNKS, bool WARP, bool EVEN>
cudaError_t launch_rows(const bacon_block& b, const Choices& c, int pieces, cudaStream_t st)
{
    const int threads = WARP ? 128 : ((pieces + CHUNKS - 1) / CHUNKS + 31) / 32 * 32;
    const long long rows = WARP ? 4 : 1, wanted = (b.tokens + rows - 1) / rows;
    // as many blocks as the registers leave room for, or half as many rows
    const long long most = 152LL * (CHUNKS == 1 ? 1024 : CHUNKS == 2 ? 768 : WARP ? 384 : 512) / threads;
    const long long blocks = wanted < most || !(EVEN && CHUNKS <= 4) ? wanted : most;
    return launch_first(block_norm_kernel<DTYPE, RESIDUAL, CHUNKS, WARP, EVEN>, (unsigned)blocks, threads, 0,
                        st, b, c);
}

}  // namespace
}  // namespace bacon
