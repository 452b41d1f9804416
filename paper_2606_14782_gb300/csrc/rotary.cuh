// Rotary positions of rows, eight values a lane: what bacon_rotary_apply and
// bacon_cache_store_rotated share, so that both give the same bits.
#pragma once

#include "common.cuh"
#include "values.cuh"

namespace bacon {

constexpr int kMaxPairsOfHead = BACON_MAX_HEAD / 2;

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

// How a lane gets the other value of each of its pairs.
enum { kPairLane = 0,    // from another lane: half a rotation is a multiple of eight values
       kPairOwn = 1,     // it has it itself: interleaved
       kPairMemory = 2 };  // it reads it again, and rows may start anywhere

// Cosine and signed sine of token t's angles for the values e0 .. e0 + 8 of a
// row: y_e = x_e c_e + x_pair s_e.  Values beyond the rotation have 1 and -0, which
// with a pair of 0 leaves them as they are, -0 too.
template <int PAIR>
__device__ __forceinline__ void angles_of(const RotaryTable& a, long long t, int e0, Piece& cosines,
                                          Piece& sines)
{
    const int half = a.rotary_dim / 2;
    int p[3] = {0, 0, 0};
    p[0] = a.positions[t];
    if (a.axes > 1) {
        p[1] = a.positions[a.tokens + t];
        p[2] = a.positions[2 * a.tokens + t];
    }
    const bool interleaved = PAIR == kPairOwn || (PAIR == kPairMemory && a.interleaved);
    float c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (PAIR == kPairOwn && (j & 1)) {
            c[j] = c[j - 1];  // (a rotation ends with a pair)
            s[j] = e0 + j < a.rotary_dim ? -s[j - 1] : -0.0f;
            continue;
        }
        const int e = e0 + j;
        c[j] = 1.0f;
        s[j] = -0.0f;
        if (e >= a.rotary_dim) continue;
        const int i = interleaved ? e >> 1 : e < half ? e : e - half;
        const bool second = interleaved ? e & 1 : e >= half;
        int at = p[0];
        if (a.axes > 1) {
            const int x = a.axis[i];
            at = x == 0 ? p[0] : x == 1 ? p[1] : p[2];
        }
        const uint64_t phase = (uint64_t)(int64_t)at * a.turns[i];
        // 2^-32 turns, in (-1, 1] half turns
        const float turn = (float)(int32_t)(phase >> 32) * 0x1p-31f;
        float sine, cosine;
        sincospif(turn, &sine, &cosine);
        c[j] = cosine * a.amplitude;
        sine *= a.amplitude;
        s[j] = second != (a.transposed != 0) ? sine : -sine;
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
    int pair;        // how pairs are got
    int vectors;     // rows start at multiples of 16 bytes
};
cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t st);

// How the rows of a call are dealt out: a group of 2^log_lanes lanes turns `per`
// heads of Q or of K of a token, of chunks[0] and chunks[1] such pieces.
struct RotaryDeal {
    int log_lanes, per, chunks[2];
};
constexpr int kRotaryBatch = 4;  // rows of a group that are on their way together

// Piece `item` of the call's rows; whole warps call it.
template <int DTYPE, int PAIR, bool NORM>
__device__ __forceinline__ void rotate_piece(const RotaryArgs& a, const RotaryDeal& deal, unsigned item)
{
    constexpr int kBytes = Eight<DTYPE>::kBytes;
    const RotaryTable& tab = a.table;
    const int q = threadIdx.x & ((1 << deal.log_lanes) - 1), e0 = 8 * q;
    const unsigned every = deal.chunks[0] + deal.chunks[1], t = item / every;
    int first = (int)(item % every);
    const bool key = first >= deal.chunks[0];
    const RotaryRows& rows = a.rows[key];
    if (key) first -= deal.chunks[0];
    first *= deal.per;
    const bool active = t < tab.tokens && e0 < tab.head_dim;
    const int count = active ? min(deal.per, rows.heads - first) : 0;
    const unsigned r = t / a.tokens, n = t % a.tokens;
    const char* in = rows.in + r * rows.in_request + n * rows.in_token + first * rows.in_head;
    char* out = rows.out + r * rows.out_request + n * rows.out_token + first * rows.out_head;
    const bool vectors = PAIR != kPairMemory || a.vectors;
    const bool norm = NORM && rows.weight;
    // beyond the rotation rows stay as they are
    const bool turns = norm || e0 < tab.rotary_dim;
    const bool writes = turns || in != out;

    Piece c, s;
    for (int base = 0; base < deal.per; base += kRotaryBatch) {  // the same for the whole warp
        Eight<DTYPE> raw[kRotaryBatch];
#pragma unroll
        for (int b = 0; b < kRotaryBatch; ++b) {
#pragma unroll
            for (int i = 0; i < Eight<DTYPE>::kWords; ++i) raw[b].w[i] = 0;
            if (base + b < count && vectors) load_eight(raw[b], in + b * rows.in_head + e0 * kBytes);
        }
        if (base == 0) {
            if (active) angles_of<PAIR>(tab, t, e0, c, s);
            if (NORM) weigh<DTYPE, PAIR>(tab, active ? rows.weight : nullptr, q, c, s);
        }
#pragma unroll
        for (int b = 0; b < kRotaryBatch; ++b) {
            if (base + b >= deal.per) break;
            const bool mine = base + b < count;
            const char* const row = in + b * rows.in_head;
            char* const to = out + b * rows.out_head;
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
                if (turns) close_piece(w, y);
                store_eight(to + e0 * kBytes, w);
            } else {
                float f[8];
                get_floats(y, f);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e0 + j < tab.head_dim) store_one<DTYPE>(to, e0 + j, f[j]);
            }
        }
        in += kRotaryBatch * rows.in_head;
        out += kRotaryBatch * rows.out_head;
    }
}

// Pieces of `heads` rows for the deal's `per`.
inline int chunks_of(int heads, int per) { return (heads + per - 1) / per; }

}  // namespace bacon
