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
    float eps, weight_offset;
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
__device__ __forceinline__ void angles_of(const RotaryTable& a, long long t, int e0, float (&c)[8],
                                          float (&s)[8])
{
    const int half = a.rotary_dim / 2;
    int p[3] = {0, 0, 0};
    p[0] = a.positions[t];
    if (a.axes > 1) {
        p[1] = a.positions[a.tokens + t];
        p[2] = a.positions[2 * a.tokens + t];
    }
    const bool interleaved = PAIR == kPairOwn || (PAIR == kPairMemory && a.interleaved);
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
}

// The other value of each pair of the values e0 .. of a row, 0 beyond the
// rotation.  `raw` (x unpacked) are the lane's own, `q` its place among those
// that have the row at `row`, which start at a lane of the same alignment; the
// whole warp calls it, and `mine` says whether there is such a row.
template <int DTYPE, int PAIR>
__device__ __forceinline__ void pairs_of(const RotaryTable& a, const Eight<DTYPE>& raw,
                                         const float (&x)[8], const void* row, bool mine, int q,
                                         float (&other)[8])
{
    const int e0 = 8 * q;
    if (PAIR == kPairLane) {
        const int lanes = a.rotary_dim / 16;
        const int away = q < lanes ? lanes : q < 2 * lanes ? -lanes : 0;
        Eight<DTYPE> o;
#pragma unroll
        for (int i = 0; i < Eight<DTYPE>::kWords; ++i) {
            o.w[i] = __shfl_sync(0xFFFFFFFFu, raw.w[i], (threadIdx.x & 31) + away);
            if (away == 0) o.w[i] = 0;
        }
        unpack_eight(o, other);
        return;
    }
    if (PAIR == kPairOwn) {
#pragma unroll
        for (int j = 0; j < 8; ++j) other[j] = e0 + j < a.rotary_dim ? x[j ^ 1] : 0.0f;
        return;
    }
    const int half = a.rotary_dim / 2;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = e0 + j;
        other[j] = 0.0f;
        if (mine && e < a.rotary_dim)
            other[j] = load_one<DTYPE>(row, a.interleaved ? e ^ 1 : e < half ? e + half : e - half);
    }
}

// Weights of a norm into the factors: y = inv (x (w c) + other (w_other s)).
__device__ __forceinline__ void weigh(const RotaryTable& a, const void* weight, int e0,
                                      bool interleaved, float (&c)[8], float (&s)[8])
{
    const int half = a.rotary_dim / 2;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = e0 + j;
        if (e >= a.head_dim) continue;
        c[j] *= a.weight_offset + load_any(weight, e, a.weight_dtype);
        if (e >= a.rotary_dim) continue;
        const int o = interleaved ? e ^ 1 : e < half ? e + half : e - half;
        s[j] *= a.weight_offset + load_any(weight, o, a.weight_dtype);
    }
}

// 1 / sqrt(mean x^2 + eps) of rows that groups of 2^log_lanes lanes have; the
// whole warp calls it, and rows without a norm have 1.  Rows whose squares pass
// fp32 are scaled, x and other too.
__device__ __forceinline__ float row_inverse(const RotaryTable& a, int log_lanes, bool norm,
                                             float (&x)[8], float (&other)[8])
{
    auto squares = [&] {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], sum);
        for (int off = 0; off < log_lanes; ++off) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1 << off);
        return sum;
    };
    float sum = squares(), eps = a.eps;
    const bool passed = norm && !(sum < INFINITY);
    if (__any_sync(0xFFFFFFFFu, passed)) {
        if (passed) {
            eps = 0.0f;  // far below such a mean
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] *= 0x1p-100f;
                other[j] *= 0x1p-100f;
            }
        }
        sum = squares();
    }
    return norm ? 1.0f / sqrtf(sum / (float)a.head_dim + eps) : 1.0f;
}

__device__ __forceinline__ void turn_eight(const float (&x)[8], const float (&other)[8],
                                           const float (&c)[8], const float (&s)[8], float inv,
                                           float (&y)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = fmaf(x[j], c[j], other[j] * s[j]) * inv;
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
// heads of a token, of `chunks` such pieces.
struct RotaryDeal {
    int log_lanes, per, chunks;
};
constexpr int kRotaryBatch = 4;  // rows of a group that are on their way together

// Piece `item` of the call's rows; whole warps call it.
template <int DTYPE, int PAIR, bool NORM>
__device__ __forceinline__ void rotate_piece(const RotaryArgs& a, const RotaryDeal& deal,
                                             unsigned item)
{
    const RotaryTable& tab = a.table;
    const int q = threadIdx.x & ((1 << deal.log_lanes) - 1), e0 = 8 * q;
    const unsigned t = item / deal.chunks;
    const int first = (int)(item % deal.chunks) * deal.per;
    const bool active = t < tab.tokens;
    const int count = active ? min(deal.per, a.rows[0].heads + a.rows[1].heads - first) : 0;
    const bool inside = e0 < tab.head_dim;
    const unsigned r = t / a.tokens, n = t % a.tokens;
    const bool interleaved = PAIR == kPairOwn || (PAIR == kPairMemory && tab.interleaved);
    const bool vectors = PAIR != kPairMemory || a.vectors;

    float c[8], s[8], wc[8], ws[8];
    int weighed = -1;
    for (int base = 0; base < deal.per; base += kRotaryBatch) {  // the same for the whole warp
        Eight<DTYPE> raw[kRotaryBatch];
        const char* in[kRotaryBatch];
        char* out[kRotaryBatch];
        bool mine[kRotaryBatch];
#pragma unroll
        for (int b = 0; b < kRotaryBatch; ++b) {
            int h = first + base + b;
            const bool key = h >= a.rows[0].heads;
            const RotaryRows& rows = a.rows[key];
            if (key) h -= a.rows[0].heads;
            in[b] = rows.in + r * rows.in_request + n * rows.in_token + h * rows.in_head;
            out[b] = rows.out + r * rows.out_request + n * rows.out_token + h * rows.out_head;
            mine[b] = base + b < count && inside;
            // beyond the rotation a row in place stays as it is
            if (!NORM && in[b] == out[b] && e0 >= tab.rotary_dim) mine[b] = false;
#pragma unroll
            for (int i = 0; i < Eight<DTYPE>::kWords; ++i) raw[b].w[i] = 0;
            if (mine[b] && vectors) load_eight(raw[b], in[b] + e0 * Eight<DTYPE>::kBytes);
        }
        if (base == 0 && active) angles_of<PAIR>(tab, t, e0, c, s);
#pragma unroll
        for (int b = 0; b < kRotaryBatch; ++b) {
            if (base + b >= deal.per) break;
            float x[8], other[8], y[8];
            unpack_eight(raw[b], x);
            if (!vectors && mine[b])
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e0 + j < tab.head_dim) x[j] = load_one<DTYPE>(in[b], e0 + j);
            pairs_of<DTYPE, PAIR>(tab, raw[b], x, in[b], mine[b], q, other);
            if (PAIR == kPairMemory) __syncwarp();  // a row in place is read before it is written
            if (NORM) {
                const int key = first + base + b >= a.rows[0].heads;
                const void* const weight = a.rows[key].weight;
                if (key != weighed) {
                    weighed = key;
#pragma unroll
                    for (int j = 0; j < 8; ++j) wc[j] = c[j], ws[j] = s[j];
                    if (weight && active) weigh(tab, weight, e0, interleaved, wc, ws);
                }
                const float inv = row_inverse(tab, deal.log_lanes, weight != nullptr, x, other);
                turn_eight(x, other, wc, ws, inv, y);
            } else {
                turn_eight(x, other, c, s, 1.0f, y);
            }
            if (!mine[b]) continue;
            if (vectors) {
                Eight<DTYPE> w = raw[b];  // beyond the rotation, without a norm
                if (e0 < tab.rotary_dim || (NORM && a.rows[first + base + b >= a.rows[0].heads].weight))
                    pack_eight(w, y);
                store_eight(out[b] + e0 * Eight<DTYPE>::kBytes, w);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e0 + j < tab.head_dim) store_one<DTYPE>(out[b], e0 + j, y[j]);
            }
        }
    }
}

}  // namespace bacon
