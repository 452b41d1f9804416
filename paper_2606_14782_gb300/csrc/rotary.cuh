// Rotary positions of rows, eight values a lane: what bacon_rotary_apply and
// bacon_cache_store_rotated share, so that both give the same bits.
#pragma once

#include "common.cuh"
#include "values.cuh"

namespace bacon {

constexpr int kMaxPairsOfHead = BACON_MAX_HEAD / 2;
constexpr int kMostHeads = 16;  // of a group

// A handle's table and a call's choices; travels as a kernel parameter (1.2 KB),
// so that a handle has no device memory and a captured call outlives it.
struct RotaryTable {
    // theta_i / 2 pi in units of 2^-64 turns: times an integer position, modulo
    // 2^64, it is the angle without a whole turn, exact however far the position
    uint64_t turns[kMaxPairsOfHead];
    uint8_t axis[kMaxPairsOfHead];
    int head_dim, rotary_dim, interleaved, axes;
    float amplitude;
    // of a call
    int transposed;
    int weight_dtype;
    float eps, weight_offset, per_value;  // per_value: 1 / head_dim
    long long tokens;          // of an axis
    const int32_t* positions;  // [axes][tokens]
};

// How a lane that has eight neighbouring values gets the other of each pair ...
enum { kPairLane = 0,    // from another lane: half a rotation is a multiple of eight values
       kPairOwn = 1,     // it has it itself: interleaved
       kPairMemory = 2,  // it reads it again, and rows may start anywhere
       // ... and lanes that have eight whole pairs (rotary.cu)
       kPairHalves = 3,  // eight values and their eight others, half a rotation on
       kPairSixteen = 4 };  // sixteen neighbours, interleaved

// Cosines and sines of two angles given in units of 2^-32 turns: the nearest
// quarter turn comes off, the rest, at most an eighth of a turn either way, goes
// into the Taylor series of both (to x^9 and x^10, what follows is below 2^-29),
// and the quarter says which of the two is the cosine and with what sign.
__device__ __forceinline__ void two_angles(uint32_t u0, uint32_t u1, float (&cosine)[2], float (&sine)[2])
{
    const uint32_t u[2] = {u0, u1};
    uint32_t quarter[2];
    float rest[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        quarter[i] = (u[i] + 0x20000000u) >> 30;
        rest[i] = (float)(int32_t)(u[i] - (quarter[i] << 30));
    }
    const auto both = [](float v) { return pair_of(v, v); };
    const Pair x = mul2(pair_of(rest[0], rest[1]), both(1.4629180792671596e-9f));  // 2 pi / 2^32
    const Pair z = mul2(x, x);
    Pair s = fma2(z, both(1.0f / 362880), both(-1.0f / 5040));
    s = fma2(z, s, both(1.0f / 120));
    s = fma2(z, s, both(-1.0f / 6));
    s = fma2(mul2(x, z), s, x);
    Pair c = fma2(z, both(-1.0f / 3628800), both(1.0f / 40320));
    c = fma2(z, c, both(-1.0f / 720));
    c = fma2(z, c, both(1.0f / 24));
    c = fma2(z, c, both(-0.5f));
    c = fma2(z, c, both(1.0f));
    const float2 fs = floats_of(s), fc = floats_of(c);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float a = i ? fs.y : fs.x, b = i ? fc.y : fc.x;
        const bool odd = quarter[i] & 1;
        sine[i] = __uint_as_float(__float_as_uint(odd ? b : a) ^ (quarter[i] & 2) << 30);
        cosine[i] = __uint_as_float(__float_as_uint(odd ? a : b) ^ ((quarter[i] + 1) & 2) << 30);
    }
}

// A token's positions, and pair i's angle there in units of 2^-32 turns: exact
// modulo a turn however far the position.
struct RotaryPlace {
    int p[3];
};
__device__ __forceinline__ RotaryPlace place_of(const RotaryTable& a, long long t)
{
    RotaryPlace at;
    at.p[0] = at.p[1] = at.p[2] = a.positions[t];
    if (a.axes > 1) {
        at.p[1] = a.positions[a.tokens + t];
        at.p[2] = a.positions[2 * a.tokens + t];
    }
    return at;
}
__device__ __forceinline__ uint32_t phase_of(const RotaryPlace& at, uint64_t turns, int axis)
{
    const int p = axis == 0 ? at.p[0] : axis == 1 ? at.p[1] : at.p[2];
    return (uint32_t)((uint64_t)(int64_t)p * turns >> 32);
}

// What a lane keeps of the table for the values e0 .. e0 + 8: its pairs' turns (0
// beyond the rotation) and, two bits each, their axes.
template <int PAIR>
struct RotaryLane {
    static constexpr int kStep = PAIR == kPairOwn ? 2 : 1;  // values that an angle serves
    uint64_t turns[8 / kStep];
    uint32_t axes;
};
template <int PAIR>
__device__ __forceinline__ RotaryLane<PAIR> lane_of(const RotaryTable& a, int e0)
{
    constexpr int kStep = RotaryLane<PAIR>::kStep;
    const int half = a.rotary_dim / 2;
    const bool interleaved = PAIR == kPairOwn || (PAIR == kPairMemory && a.interleaved);
    RotaryLane<PAIR> lane;
    lane.axes = 0;
#pragma unroll
    for (int j = 0; j < 8; j += kStep) {
        const int e = e0 + j;
        lane.turns[j / kStep] = 0;
        if (e >= a.rotary_dim) continue;
        const int i = interleaved ? e >> 1 : e < half ? e : e - half;
        lane.turns[j / kStep] = a.turns[i];
        if (a.axes > 1) lane.axes |= (uint32_t)a.axis[i] << (2 * (j / kStep));
    }
    return lane;
}

// Factors of the values e0 .. e0 + 8 of a row at a place: y_e = x_e c_e + x_pair
// s_e.  Values beyond the rotation have 1 and -0, which with a pair of 0 leaves
// them as they are, -0 too.
template <int PAIR>
__device__ __forceinline__ void factors_of(const RotaryTable& a, const RotaryLane<PAIR>& lane,
                                           const RotaryPlace& at, int e0, Piece& cosines, Piece& sines)
{
    constexpr int kStep = RotaryLane<PAIR>::kStep;
    const int half = a.rotary_dim / 2;
    const bool interleaved = PAIR == kPairOwn || (PAIR == kPairMemory && a.interleaved);
    const float turned = a.transposed ? -a.amplitude : a.amplitude;
    float c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; j += 2 * kStep) {
        const int i = j / kStep;
        float cosine[2], sine[2];
        two_angles(phase_of(at, lane.turns[i], lane.axes >> (2 * i) & 3),
                   phase_of(at, lane.turns[i + 1], lane.axes >> (2 * i + 2) & 3), cosine, sine);
#pragma unroll
        for (int k = 0; k < 2 * kStep; ++k) {
            const int e = e0 + j + k, from = k / kStep;
            const float f = sine[from] * turned;
            c[j + k] = e < a.rotary_dim ? cosine[from] * a.amplitude : 1.0f;
            s[j + k] = e < a.rotary_dim ? ((interleaved ? e & 1 : e >= half) ? f : -f) : -0.0f;
        }
    }
    set_floats(cosines, c);
    set_floats(sines, s);
}

// The other value of each pair of the values 8 q .. of a row, 0 beyond the rotation.
// `raw` (v unpacked) are the lane's own, q its place among those that have the row
// at `row`, which start at a lane of the same alignment; the whole warp calls it,
// and `mine` says whether there is such a row.
template <int DTYPE, int PAIR>
__device__ __forceinline__ void pairs_of(const RotaryTable& a, const Eight<DTYPE>& raw, const Piece& v,
                                         const void* row, bool mine, int q, Piece& other)
{
    const int e0 = 8 * q;
    if (PAIR == kPairLane) {
        const int lanes = a.rotary_dim / 16;
        const int away = q < lanes ? lanes : q < 2 * lanes ? -lanes : 0;
        Eight<DTYPE> o;
#pragma unroll
        for (int i = 0; i < Eight<DTYPE>::kWords; ++i)
            o.w[i] = __shfl_sync(0xFFFFFFFFu, raw.w[i], (threadIdx.x & 31) + away);
        if (a.rotary_dim < a.head_dim && away == 0)
#pragma unroll
            for (int i = 0; i < Eight<DTYPE>::kWords; ++i) o.w[i] = 0;
        open_piece(o, other);
    } else if (PAIR == kPairOwn) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = floats_of(v.p[j]);
            other.p[j] = pair_of(f.y, f.x);
            if (a.rotary_dim < a.head_dim && e0 + 2 * j >= a.rotary_dim) other.p[j] = 0;
        }
    } else {
        const int half = a.rotary_dim / 2;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = e0 + j;
            f[j] = 0.0f;
            if (mine && e < a.rotary_dim)
                f[j] = load_one<DTYPE>(row, a.interleaved ? e ^ 1 : e < half ? e + half : e - half);
        }
        set_floats(other, f);
    }
}

// Weights of a norm into the factors: y = inv (x (w c) + other (w_other s)).
// Whole warps call it; without a weight the factors stay.
template <int DTYPE, int PAIR>
__device__ __forceinline__ void weigh_as(const RotaryTable& a, const void* weight, int q, Piece& c, Piece& s)
{
    const int e0 = 8 * q;
    const bool mine = weight && e0 < a.head_dim;
    Eight<DTYPE> raw;
    Piece w, other;
#pragma unroll
    for (int i = 0; i < Eight<DTYPE>::kWords; ++i) raw.w[i] = 0;
    if (PAIR != kPairMemory) {
        if (mine) load_eight(raw, static_cast<const char*>(weight) + e0 * Eight<DTYPE>::kBytes);
        open_piece(raw, w);
    } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = mine && e0 + j < a.head_dim ? load_one<DTYPE>(weight, e0 + j) : 0.0f;
        set_floats(w, f);
    }
    pairs_of<DTYPE, PAIR>(a, raw, w, weight, mine, q, other);
    if (!mine) return;
    const Pair offset = pair_of(a.weight_offset, a.weight_offset);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c.p[j] = mul2(c.p[j], add2(w.p[j], offset));
        s.p[j] = mul2(s.p[j], add2(other.p[j], offset));
    }
}
template <int DTYPE, int PAIR>
__device__ __forceinline__ void weigh(const RotaryTable& a, const void* weight, int q, Piece& c, Piece& s)
{
    if (DTYPE != BACON_FP32 && a.weight_dtype == BACON_FP32)
        weigh_as<BACON_FP32, PAIR>(a, weight, q, c, s);
    else
        weigh_as<DTYPE, PAIR>(a, weight, q, c, s);
}

// 1 / sqrt(mean x^2 + eps) of rows that groups of 2^log_lanes lanes have; the
// whole warp calls it, and rows without a norm have 1.  Rows whose squares pass
// fp32 are scaled, x and other too.
__device__ __forceinline__ float row_inverse(const RotaryTable& a, int log_lanes, bool norm, Piece& x,
                                             Piece& other)
{
    const auto squares = [&] {
        Pair t = mul2(x.p[0], x.p[0]);
#pragma unroll
        for (int j = 1; j < 4; ++j) t = fma2(x.p[j], x.p[j], t);
        const float2 f = floats_of(t);
        float sum = f.x + f.y;
        for (int off = 0; off < log_lanes; ++off) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1 << off);
        return sum;
    };
    float sum = squares(), eps = a.eps;
    const bool passed = norm && !(sum < INFINITY);
    if (__any_sync(0xFFFFFFFFu, passed)) {
        if (passed) {
            eps = 0.0f;  // far below such a mean
            const Pair small = pair_of(0x1p-100f, 0x1p-100f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x.p[j] = mul2(x.p[j], small);
                other.p[j] = mul2(other.p[j], small);
            }
        }
        sum = squares();
    }
    return norm ? rsqrtf(fmaf(sum, a.per_value, eps)) : 1.0f;
}

__device__ __forceinline__ void turn_piece(const Piece& x, const Piece& other, const Piece& c, const Piece& s,
                                           Piece& y)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) y.p[j] = fma2(x.p[j], c.p[j], mul2(other.p[j], s.p[j]));
}
__device__ __forceinline__ void scale_piece(Piece& y, float by)
{
    const Pair p = pair_of(by, by);
#pragma unroll
    for (int j = 0; j < 4; ++j) y.p[j] = mul2(y.p[j], p);
}

// First (A) and second (B) values of eight pairs, of two groups of eight values.
template <int DTYPE, bool SIXTEEN>
__device__ __forceinline__ void open_pairs(const Eight<DTYPE>& one, const Eight<DTYPE>& two, Piece& A, Piece& B)
{
    float f[8], g[8];
    unpack_eight(one, f);
    unpack_eight(two, g);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        A.p[j] = SIXTEEN ? pair_of(f[4 * j], f[4 * j + 2]) : pair_of(f[2 * j], f[2 * j + 1]);
        B.p[j] = SIXTEEN ? pair_of(f[4 * j + 1], f[4 * j + 3]) : pair_of(g[2 * j], g[2 * j + 1]);
        A.p[j + 2] = SIXTEEN ? pair_of(g[4 * j], g[4 * j + 2]) : pair_of(f[2 * j + 4], f[2 * j + 5]);
        B.p[j + 2] = SIXTEEN ? pair_of(g[4 * j + 1], g[4 * j + 3]) : pair_of(g[2 * j + 4], g[2 * j + 5]);
    }
}
template <int DTYPE, bool SIXTEEN>
__device__ __forceinline__ void close_pairs(Eight<DTYPE>& one, Eight<DTYPE>& two, const Piece& A, const Piece& B)
{
    float x[8], y[8];
    get_floats(A, x);
    get_floats(B, y);
    if (SIXTEEN) {
        float f[8], g[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[2 * j] = x[j];
            f[2 * j + 1] = y[j];
            g[2 * j] = x[j + 4];
            g[2 * j + 1] = y[j + 4];
        }
        pack_eight(one, f);
        pack_eight(two, g);
    } else {
        pack_eight(one, x);
        pack_eight(two, y);
    }
}

template <int DTYPE>
struct TypeTag {
    static constexpr int kType = DTYPE;
};

// The same of rows that lanes have eight pairs of, q a lane's place among those of
// its row: each group of eight values is summed like a lane's there, and the groups
// meet in the same order, so that a row's bits do not depend on how it is read.
template <int DTYPE, bool SIXTEEN>
__device__ __forceinline__ float pairs_inverse(const RotaryTable& a, int log_lanes, int q, bool norm,
                                               const Eight<DTYPE>& one, const Eight<DTYPE>& two, Piece& A,
                                               Piece& B)
{
    const auto squares = [&](float scale) {
        float sums[2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            Piece x;
            open_piece(z ? two : one, x);
            Pair t = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Pair v = scale == 1.0f ? x.p[j] : mul2(x.p[j], pair_of(scale, scale));
                t = j ? fma2(v, v, t) : mul2(v, v);
            }
            const float2 f = floats_of(t);
            sums[z] = f.x + f.y;
        }
        if (!SIXTEEN) {
            // lane q gets the groups 2 q and 2 q + 1, neighbours as in the row
            const int half = a.rotary_dim / 16, first = threadIdx.x & 31 & ~((1 << log_lanes) - 1);
            float mine[2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const int g = 2 * q + z;
                const int from = first + (g < half ? g : g < 2 * half ? g - half : q);
                const float x = __shfl_sync(0xFFFFFFFFu, sums[0], from), y = __shfl_sync(0xFFFFFFFFu, sums[1], from);
                mine[z] = (g < 2 * half ? g >= half : z) ? y : x;
            }
            sums[0] = mine[0];
            sums[1] = mine[1];
        }
        float sum = sums[0] + sums[1];
        for (int off = 0; off < log_lanes; ++off) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1 << off);
        return sum;
    };
    float sum = squares(1.0f), eps = a.eps;
    const bool passed = norm && !(sum < INFINITY);
    if (__any_sync(0xFFFFFFFFu, passed)) {
        if (passed) {
            eps = 0.0f;
            scale_piece(A, 0x1p-100f);
            scale_piece(B, 0x1p-100f);
        }
        sum = squares(passed ? 0x1p-100f : 1.0f);
    }
    return norm ? rsqrtf(fmaf(sum, a.per_value, eps)) : 1.0f;
}

// offset + weight of eight pairs.
template <int DTYPE, bool SIXTEEN>
__device__ __forceinline__ void weights_of(const RotaryTable& a, const void* weight, int e0, int e1, Piece& A,
                                           Piece& B)
{
    const auto as = [&](auto kind) {
        constexpr int kType = decltype(kind)::kType, kBytes = Eight<kType>::kBytes;
        Eight<kType> one, two;
        load_eight(one, static_cast<const char*>(weight) + e0 * kBytes);
        load_eight(two, static_cast<const char*>(weight) + e1 * kBytes);
        open_pairs<kType, SIXTEEN>(one, two, A, B);
    };
    if (DTYPE != BACON_FP32 && a.weight_dtype == BACON_FP32)
        as(TypeTag<BACON_FP32>{});
    else
        as(TypeTag<DTYPE>{});
    const Pair offset = pair_of(a.weight_offset, a.weight_offset);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        A.p[j] = add2(A.p[j], offset);
        B.p[j] = add2(B.p[j], offset);
    }
}

// Rows of one call: bacon_rows without what the host has checked.
struct RotaryRows {
    const char* in;
    char* out;
    const void* weight;
    int heads;
    long long in_request, in_token, in_head;  // bytes
    long long out_request, out_token, out_head;
};
struct RotaryArgs {
    RotaryTable table;
    RotaryRows rows[2];  // Q, K
    int dtype, requests, tokens;
    int q_pair;      // how a call's rows are turned, but for K that is stored
    int vectors;     // rows start at multiples of 16 bytes
};
cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t st);

// How the rows of a call are dealt out: a group of 2^log_lanes lanes turns up to
// per[0] heads of Q of a token, chunks[0] such pieces a token, or per[1] of K; first
// come all pieces of Q, so that the groups of a warp have about as much to do.
struct RotaryDeal {
    int log_lanes, per[2], chunks[2];
};

// A group's piece of a call's rows.
struct RotaryTask {
    bool active;
    unsigned t;        // token
    int key, count;    // Q or K, heads
    int most;          // heads of any group of the warp
    const char* in;
    char* out;
    const void* weight;
    long long in_step, out_step;  // bytes from a head to the next
};
__device__ __forceinline__ RotaryTask task_of(const RotaryArgs& a, const RotaryDeal& deal, unsigned item)
{
    RotaryTask task;
    const unsigned before = (unsigned)a.table.tokens * deal.chunks[0];
    task.key = item >= before;
    if (task.key) item -= before;
    const RotaryRows& rows = a.rows[task.key];
    task.t = deal.chunks[task.key] ? item / deal.chunks[task.key] : a.table.tokens;
    task.active = task.t < a.table.tokens;
    const int first = task.active ? (int)(item % deal.chunks[task.key]) * deal.per[task.key] : 0;
    task.count = task.active ? min(deal.per[task.key], rows.heads - first) : 0;
    task.most = __reduce_max_sync(0xFFFFFFFFu, task.count);
    const unsigned r = task.t / a.tokens, n = task.t % a.tokens;
    task.in = rows.in + r * rows.in_request + n * rows.in_token + first * rows.in_head;
    task.out = rows.out + r * rows.out_request + n * rows.out_token + first * rows.out_head;
    task.weight = task.active ? rows.weight : nullptr;
    task.in_step = rows.in_head;
    task.out_step = rows.out_head;
    return task;
}

// Group tasks with eight values a lane; whole warps call it.
template <int DTYPE, int PAIR, bool NORM>
__device__ __forceinline__ void rotate_eights(const RotaryArgs& a, const RotaryDeal& deal, unsigned item)
{
    constexpr int kBytes = Eight<DTYPE>::kBytes, kBatch = 2;
    const RotaryTable& tab = a.table;
    const int q = threadIdx.x & ((1 << deal.log_lanes) - 1), e0 = 8 * q;
    RotaryTask task = task_of(a, deal, item);
    const bool inside = e0 < tab.head_dim;
    const int count = inside ? task.count : 0;
    const bool vectors = PAIR != kPairMemory || a.vectors;
    const bool norm = NORM && task.weight;
    // beyond the rotation rows stay as they are
    const bool changes = norm || e0 < tab.rotary_dim;
    const bool writes = changes || task.in != task.out;

    Piece c, s;
    for (int base = 0; base < task.most; base += kBatch) {
        Eight<DTYPE> raw[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
#pragma unroll
            for (int i = 0; i < Eight<DTYPE>::kWords; ++i) raw[b].w[i] = 0;
            if (base + b < count && vectors) load_eight(raw[b], task.in + b * task.in_step + e0 * kBytes);
        }
        if (base == 0) {
            if (task.active && inside)
                factors_of<PAIR>(tab, lane_of<PAIR>(tab, e0), place_of(tab, task.t), e0, c, s);
            if (NORM) weigh<DTYPE, PAIR>(tab, inside ? task.weight : nullptr, q, c, s);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (base + b >= task.most) break;
            const bool mine = base + b < count;
            const char* const row = task.in + b * task.in_step;
            char* const to = task.out + b * task.out_step;
            Piece x, other, y;
            if (vectors) {
                open_piece(raw[b], x);
            } else {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    f[j] = mine && e0 + j < tab.head_dim ? load_one<DTYPE>(row, e0 + j) : 0.0f;
                set_floats(x, f);
            }
            pairs_of<DTYPE, PAIR>(tab, raw[b], x, row, mine, q, other);
            if (PAIR == kPairMemory) __syncwarp();  // a row in place is read before it is written
            float inv = 1.0f;
            if (NORM) inv = row_inverse(tab, deal.log_lanes, norm, x, other);
            turn_piece(x, other, c, s, y);
            if (NORM) scale_piece(y, inv);
            if (!mine || !writes) continue;
            if (vectors) {
                Eight<DTYPE> w = raw[b];
                if (changes) close_piece(w, y);
                store_eight(to + e0 * kBytes, w);
            } else {
                float f[8];
                get_floats(y, f);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e0 + j < tab.head_dim) store_one<DTYPE>(to, e0 + j, f[j]);
            }
        }
        task.in += kBatch * task.in_step;
        task.out += kBatch * task.out_step;
    }
}

// Where a lane's two groups of eight values lie: eight pairs, or beyond the
// rotation sixteen neighbours that stay.
struct RotarySpan {
    int e0, e1;
    bool turning;
};
template <bool SIXTEEN>
__device__ __forceinline__ RotarySpan span_of(const RotaryTable& a, int q)
{
    RotarySpan s;
    s.turning = 16 * q < a.rotary_dim;
    s.e0 = SIXTEEN || !s.turning ? 16 * q : 8 * q;
    s.e1 = SIXTEEN || !s.turning ? s.e0 + 8 : s.e0 + a.rotary_dim / 2;
    return s;
}

// y_A = A cA + B sA, y_B = B cB + A sB; without a norm cB is cA.
struct PairFactors {
    Piece cA, sA, cB, sB;
};
template <int DTYPE, bool SIXTEEN, bool NORM>
__device__ __forceinline__ void pair_factors(const RotaryTable& tab, const RotaryPlace& at, const void* weight,
                                             int q, const RotarySpan& span, PairFactors& f)
{
    if (!span.turning && !(NORM && weight)) return;  // nobody looks at them
    const float turned = tab.transposed ? -tab.amplitude : tab.amplitude;
    float c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = 1.0f, s[j] = 0.0f;
    if (span.turning)
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float cosine[2], sine[2];
            uint32_t u[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int i = 8 * q + j + k;
                u[k] = phase_of(at, tab.turns[i], tab.axes > 1 ? tab.axis[i] : 0);
            }
            two_angles(u[0], u[1], cosine, sine);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                c[j + k] = cosine[k] * tab.amplitude;
                s[j + k] = sine[k] * turned;
            }
        }
    set_floats(f.cA, c);
    set_floats(f.sB, s);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = -s[j];
    set_floats(f.sA, s);
    f.cB = f.cA;
    if (NORM && weight) {
        Piece wA, wB;
        weights_of<DTYPE, SIXTEEN>(tab, weight, span.e0, span.e1, wA, wB);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f.cA.p[j] = mul2(f.cA.p[j], wA.p[j]);
            f.sA.p[j] = mul2(f.sA.p[j], wB.p[j]);
            f.cB.p[j] = mul2(f.cB.p[j], wB.p[j]);
            f.sB.p[j] = mul2(f.sB.p[j], wA.p[j]);
        }
    }
}

// Turns a lane's pairs of a row; beyond the rotation and without a norm they stay
// bit for bit.  With NORM whole warps call it.
template <int DTYPE, bool SIXTEEN, bool NORM>
__device__ __forceinline__ void turn_pairs(const RotaryTable& tab, int log_lanes, int q, bool norm,
                                           const RotarySpan& span, const PairFactors& f, Eight<DTYPE>& one,
                                           Eight<DTYPE>& two)
{
    Piece A, B, yA, yB;
    open_pairs<DTYPE, SIXTEEN>(one, two, A, B);
    float inv = 1.0f;
    if (NORM) inv = pairs_inverse<DTYPE, SIXTEEN>(tab, log_lanes, q, norm, one, two, A, B);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        // (beyond the rotation nothing of the other, were it an infinity)
        const Pair fromB = !NORM || span.turning ? mul2(B.p[j], f.sA.p[j]) : 0;
        const Pair fromA = !NORM || span.turning ? mul2(A.p[j], f.sB.p[j]) : 0;
        yA.p[j] = fma2(A.p[j], f.cA.p[j], fromB);
        yB.p[j] = fma2(B.p[j], NORM ? f.cB.p[j] : f.cA.p[j], fromA);
    }
    if (NORM) {
        scale_piece(yA, inv);
        scale_piece(yB, inv);
    }
    if (span.turning || (NORM && norm)) close_pairs<DTYPE, SIXTEEN>(one, two, yA, yB);
}

// Group tasks with eight pairs a lane, with the same products and sums as with eight
// values a lane.  Whole warps call it.
template <int DTYPE, bool SIXTEEN, bool NORM>
__device__ __forceinline__ void rotate_pairs(const RotaryArgs& a, const RotaryDeal& deal, unsigned item)
{
    // rows on their way together: what the registers hold (with norms two took 105 us for
    // 96 of 95000 tokens of 8 heads in 16 bits, four of fp32 42 for 33 of 2800 of 64)
    constexpr int kBytes = Eight<DTYPE>::kBytes, kBatch = DTYPE == BACON_FP32 ? 2 : 4;
    const RotaryTable& tab = a.table;
    const int q = threadIdx.x & ((1 << deal.log_lanes) - 1);
    RotaryTask task = task_of(a, deal, item);
    const RotarySpan span = span_of<SIXTEEN>(tab, q);
    const bool inside = 16 * q < tab.head_dim;
    // beyond the rotation rows in place stay as they are
    const int count = inside && (span.turning || (NORM && task.weight) || task.in != task.out) ? task.count : 0;
    task.in += span.e0 * kBytes;
    task.out += span.e0 * kBytes;
    const int apart = (span.e1 - span.e0) * kBytes;

    PairFactors f;
    for (int base = 0; base < task.most; base += kBatch) {
        Eight<DTYPE> one[kBatch], two[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            if (base + b < count) {
                load_eight(one[b], task.in + b * task.in_step);
                load_eight(two[b], task.in + b * task.in_step + apart);
            }
        if (base == 0 && inside && task.active)
            pair_factors<DTYPE, SIXTEEN, NORM>(tab, place_of(tab, task.t), task.weight, q, span, f);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (NORM && base + b >= task.most) break;
            const bool mine = base + b < count;
            if (!NORM && !mine) break;
            if (NORM && !mine)
#pragma unroll
                for (int i = 0; i < Eight<DTYPE>::kWords; ++i) one[b].w[i] = two[b].w[i] = 0;
            turn_pairs<DTYPE, SIXTEEN, NORM>(tab, deal.log_lanes, q, task.weight != nullptr, span, f, one[b], two[b]);
            if (!mine) continue;
            store_eight(task.out + b * task.out_step, one[b]);
            store_eight(task.out + b * task.out_step + apart, two[b]);
        }
        task.in += kBatch * task.in_step;
        task.out += kBatch * task.out_step;
    }
}

template <int DTYPE, int PAIR, bool NORM>
__device__ __forceinline__ void rotate_piece(const RotaryArgs& a, const RotaryDeal& deal, unsigned item)
{
    if constexpr (PAIR == kPairHalves)
        rotate_pairs<DTYPE, false, NORM>(a, deal, item);
    else if constexpr (PAIR == kPairSixteen)
        rotate_pairs<DTYPE, true, NORM>(a, deal, item);
    else
        rotate_eights<DTYPE, PAIR, NORM>(a, deal, item);
}

// Deals out rows: as few heads share a group and its angles as give every SM
// `threads` threads.  Returns the pieces.
inline long long deal_rows(const RotaryArgs& a, int values, int threads, RotaryDeal* deal)
{
    *deal = RotaryDeal{};
    while (values << deal->log_lanes < a.table.head_dim) ++deal->log_lanes;
    const long long rows = a.table.tokens * (a.rows[0].heads + a.rows[1].heads);
    int most = 1;
    while (most < kMostHeads && rows / most > (152LL * threads >> deal->log_lanes)) most *= 2;
    for (int i = 0; i < 2; ++i) {
        const int heads = a.rows[i].heads, chunks = (heads + most - 1) / most;
        deal->chunks[i] = chunks;
        deal->per[i] = chunks ? (heads + chunks - 1) / chunks : 0;
    }
    return a.table.tokens * (deal->chunks[0] + deal->chunks[1]);
}
inline int values_of_lane(int pair) { return pair == kPairHalves || pair == kPairSixteen ? 16 : 8; }

}  // namespace bacon
