// C ABI of rotary positions, the norms between blocks and the rules on logits:
// argument checks and handles.
#include <cmath>
#include <new>
#include <utility>

#include "bacon.h"
#include "block_norm.h"
#include "cache.h"
#include "common.cuh"
#include "host.h"
#include "logits.h"
#include "rotary.cuh"
#include "step_host.h"

using namespace bacon;

struct bacon_rotary {
    RotaryTable table{};
};

struct bacon_logits {
    int device = 0;
    int vocab = 0;
    int* err = nullptr;
};

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr float kLeastEps = 1e-20f;

int size_of(int dtype) { return dtype == BACON_FP32 ? 4 : 2; }
bool known(int dtype) { return dtype == BACON_BF16 || dtype == BACON_FP16 || dtype == BACON_FP32; }
bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// theta / 2 pi in units of 2^-64 turns, |theta| below 2^20; whole turns do not count at
// whole positions.  In integers, to less than a unit: a double's quotient is off by
// 2^-53 of itself, which a position of 2^31 makes 2^-22 turns for each turn of theta.
uint64_t turns_of(double theta)
{
    constexpr uint64_t kHigh = 0x28be60db9391054a, kLow = 0x7f09d5f47d4d3770;  // 2^128 / 2 pi
    int exponent;
    const uint64_t mantissa = (uint64_t)std::ldexp(std::frexp(std::fabs(theta), &exponent), 53);
    const unsigned __int128 low = (unsigned __int128)mantissa * kLow;
    const unsigned __int128 turns = (unsigned __int128)mantissa * kHigh + (uint64_t)(low >> 64);
    const int shift = 53 - exponent;  // theta is mantissa 2^-shift, `turns` in units of 2^-64 of those
    const uint64_t units = shift < 128 ? (uint64_t)(turns >> shift) : 0;
    return theta < 0.0 ? 0 - units : units;
}

// Whether rows of d values at (n0, n1, n2) places with these strides are apart.
bool apart(int d, const long long (&sizes)[3], const long long (&strides)[3])
{
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            if (strides[order[j]] > strides[order[j + 1]]) std::swap(order[j], order[j + 1]);
    long long extent = d;
    for (int i : order) {
        if (sizes[i] <= 1) continue;
        if (strides[i] < extent) return false;
        extent += strides[i] * (sizes[i] - 1);
    }
    return true;
}

// Checks rows of Q or K and fills `out`; `vectors` stays if they start at 16 bytes.
bacon_status take_rows(const bacon_rows& r, const char* what, int requests, int tokens, int d,
                       int dtype, int weight_dtype, bool writes, RotaryRows* out, bool* vectors)
{
    const int bytes = size_of(dtype);
    if (r.heads < 0) return fail(BACON_EINVAL, "%s: heads must not be negative", what);
    if (r.heads == 0) return BACON_OK;
    if (!r.in || !aligned_to(r.in, bytes) || (writes && (!r.out || !aligned_to(r.out, bytes))))
        return fail(BACON_EINVAL, "%s: rows must be non-null and aligned to their type", what);
    if (r.weight && !aligned_to(r.weight, size_of(weight_dtype)))
        return fail(BACON_EINVAL, "%s: the weight must be aligned to its type", what);
    const long long strides[6] = {r.in_request, r.in_token, r.in_head,
                                  r.out_request, r.out_token, r.out_head};
    for (int i = 0; i < (writes ? 6 : 3); ++i)
        if (strides[i] < 0 || strides[i] >= 1ll << 56)
            return fail(BACON_EINVAL, "%s: a stride is out of range", what);
    if (writes && !apart(d, {requests, tokens, r.heads}, {r.out_request, r.out_token, r.out_head}))
        return fail(BACON_EINVAL, "%s: rows of the output overlap", what);
    if (!aligned16(r.in) || (writes && !aligned16(r.out)) || !aligned16(r.weight)) *vectors = false;
    const int places[3] = {requests, tokens, r.heads};
    for (int i = 0; i < (writes ? 6 : 3); ++i)
        if (places[i % 3] > 1 && strides[i] * bytes % 16) *vectors = false;
    out->in = static_cast<const char*>(r.in);
    out->out = writes ? static_cast<char*>(r.out) : nullptr;
    out->weight = r.weight;
    out->heads = r.heads;
    out->in_request = r.in_request * bytes;
    out->in_token = r.in_token * bytes;
    out->in_head = r.in_head * bytes;
    out->out_request = r.out_request * bytes;
    out->out_token = r.out_token * bytes;
    out->out_head = r.out_head * bytes;
    return BACON_OK;
}

}  // namespace

namespace bacon {

bacon_status rotary_args(const bacon_rotary* rotary, int requests, int tokens, const bacon_rows* q,
                         const bacon_rows* k, bool k_writes, int dtype, int weight_dtype, float eps,
                         float weight_offset, int transposed, const int32_t* positions,
                         RotaryArgs* out)
{
    if (!rotary) return fail(BACON_EINVAL, "null rotary");
    if (requests < 0 || tokens < 0) return fail(BACON_EINVAL, "sizes must not be negative");
    if (!known(dtype)) return fail(BACON_EINVAL, "unknown dtype %d", dtype);
    const bool norm = (q && q->heads && q->weight) || (k && k->heads && k->weight);
    if (norm && weight_dtype != dtype && weight_dtype != BACON_FP32)
        return fail(BACON_EINVAL, "weights are of the rows' type or fp32");
    if (norm && transposed)
        return fail(BACON_EINVAL, "the transposed rotation takes no weights");
    if (norm && !(std::isfinite(eps) && eps >= kLeastEps && std::isfinite(weight_offset)))
        return fail(BACON_EINVAL, "eps must be at least 1e-20 and finite, the offset finite");
    RotaryArgs a{};
    a.table = rotary->table;
    const int d = a.table.head_dim;
    bool vectors = d % 8 == 0;
    const bacon_rows* const rows[2] = {q, k};
    for (int i = 0; i < 2; ++i)
        if (rows[i] && requests && tokens)
            if (bacon_status rc = take_rows(*rows[i], i ? "k" : "q", requests, tokens, d, dtype,
                                            weight_dtype, i == 0 || k_writes, &a.rows[i], &vectors))
                return rc;
    const long long every = (long long)a.rows[0].heads + a.rows[1].heads;
    if ((long long)requests * tokens * (every > 0 ? every : 1) >= 1ll << 31)
        return fail(BACON_EINVAL, "a call takes fewer than 2^31 rows");
    if (requests && tokens && every && !positions) return fail(BACON_EINVAL, "null positions");
    if (!aligned_to(positions, 4)) return fail(BACON_EINVAL, "positions must be aligned to their type");
    a.table.transposed = transposed != 0;
    a.table.weight_dtype = weight_dtype;
    a.table.eps = eps;
    a.table.weight_offset = weight_offset;
    a.table.tokens = (long long)requests * tokens;
    a.table.positions = positions;
    a.dtype = dtype;
    a.requests = requests;
    a.tokens = tokens;
    a.vectors = vectors;
    const int pair = !vectors                        ? kPairMemory
                     : a.table.interleaved           ? kPairOwn
                     : a.table.rotary_dim % 16 == 0 ? kPairLane
                                                     : kPairMemory;
    // lanes with eight pairs: where sixteen values lie on one side of the rotation's end
    const bool pairs = d % 16 == 0 && a.table.rotary_dim % 16 == 0;
    a.q_pair = pair == kPairMemory || !pairs ? pair : a.table.interleaved ? kPairSixteen : kPairHalves;
    *out = a;
    return BACON_OK;
}

}  // namespace bacon

extern "C" {

bacon_status bacon_rotary_frequencies(int rotary_dim, double base, int scaling, double factor,
                                      double original, double low, double high, double* out)
{
    g_last_error.clear();
    if (!out) return fail(BACON_EINVAL, "null argument");
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > BACON_MAX_HEAD)
        return fail(BACON_EINVAL, "rotary_dim must be even, in [2, %d], got %d", BACON_MAX_HEAD,
                    rotary_dim);
    if (!(std::isfinite(base) && base > 1.0)) return fail(BACON_EINVAL, "base must be above 1");
    if (scaling < BACON_ROPE_PLAIN || scaling > BACON_ROPE_DIMS)
        return fail(BACON_EINVAL, "unknown scaling %d", scaling);
    if (scaling != BACON_ROPE_PLAIN && !(std::isfinite(factor) && factor > 0.0))
        return fail(BACON_EINVAL, "factor must be positive");
    if (scaling == BACON_ROPE_BASE && rotary_dim == 2)
        return fail(BACON_EINVAL, "one pair has no base to scale");
    const bool ramp = scaling == BACON_ROPE_ROTATIONS || scaling == BACON_ROPE_DIMS;
    if (ramp && !(std::isfinite(original) && original > 0.0 && low > 0.0 && low < high &&
                  std::isfinite(high)))
        return fail(BACON_EINVAL, "original must be positive and 0 < low < high");
    const int half = rotary_dim / 2;
    if (scaling == BACON_ROPE_BASE) {
        base *= std::pow(factor, rotary_dim / (rotary_dim - 2.0));
        if (!(std::isfinite(base) && base > 0.0)) return fail(BACON_EINVAL, "the scaled base is out of range");
    }
    // the pair that turns r times over the original length
    const auto pair_of = [&](double r) {
        return rotary_dim * std::log(original / (kTwoPi * r)) / (2.0 * std::log(base));
    };
    double first = 0.0, last = 0.0;
    if (scaling == BACON_ROPE_DIMS) {
        first = std::fmax(std::floor(pair_of(high)), 0.0);
        last = std::ceil(pair_of(low));  // it may lie behind the last pair
    }
    for (int i = 0; i < half; ++i) {
        double theta = std::pow(base, -2.0 * i / rotary_dim), kept = 1.0;
        if (scaling == BACON_ROPE_LINEAR) kept = 0.0;
        if (scaling == BACON_ROPE_ROTATIONS) kept = (original * theta / kTwoPi - low) / (high - low);
        if (scaling == BACON_ROPE_DIMS) kept = 1.0 - (i - first) / std::fmax(last - first, 0.5);
        kept = std::fmin(std::fmax(kept, 0.0), 1.0);
        if (scaling != BACON_ROPE_PLAIN && scaling != BACON_ROPE_BASE)
            theta = kept * theta + (1.0 - kept) * theta / factor;
        out[i] = theta;
    }
    return BACON_OK;
}

bacon_status bacon_rotary_create(bacon_rotary** out, int head_dim, int rotary_dim, int interleaved,
                                 float amplitude, const double* frequencies, const uint8_t* axis)
{
    g_last_error.clear();
    if (!out || !frequencies) return fail(BACON_EINVAL, "null argument");
    *out = nullptr;
    if (head_dim < 2 || head_dim % 2 || head_dim > BACON_MAX_HEAD)
        return fail(BACON_EINVAL, "head_dim must be even, in [2, %d], got %d", BACON_MAX_HEAD, head_dim);
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > head_dim)
        return fail(BACON_EINVAL, "rotary_dim must be even, in [2, head_dim], got %d", rotary_dim);
    if (!std::isfinite(amplitude)) return fail(BACON_EINVAL, "amplitude must be finite");
    bacon_rotary* r = new (std::nothrow) bacon_rotary;
    if (!r) return fail(BACON_ENOMEM, "host allocation failed");
    RotaryTable& t = r->table;
    t.head_dim = head_dim;
    t.rotary_dim = rotary_dim;
    t.interleaved = interleaved != 0;
    t.amplitude = amplitude;
    t.per_value = 1.0f / (float)head_dim;
    t.axes = axis ? 3 : 1;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        if (!std::isfinite(frequencies[i]) || std::fabs(frequencies[i]) > 1e6 ||
            (axis && axis[i] > 2)) {
            delete r;
            return fail(BACON_EINVAL, "frequency or axis %d is out of range", i);
        }
        t.turns[i] = turns_of(frequencies[i]);
        t.axis[i] = axis ? axis[i] : 0;
    }
    *out = r;
    return BACON_OK;
}

void bacon_rotary_destroy(bacon_rotary* rotary) { delete rotary; }

bacon_status bacon_rotary_apply(const bacon_rotary* rotary, int requests, int tokens,
                                const bacon_rows* q, const bacon_rows* k, int dtype,
                                int weight_dtype, float eps, float weight_offset, int transposed,
                                const int32_t* positions, bacon_stream stream)
{
    g_last_error.clear();
    RotaryArgs a;
    if (bacon_status rc = rotary_args(rotary, requests, tokens, q, k, true, dtype, weight_dtype, eps,
                                      weight_offset, transposed, positions, &a))
        return rc;
    if (a.table.tokens == 0 || a.rows[0].heads + a.rows[1].heads == 0) return BACON_OK;
    BACON_CUDA(launch_rotary(a, static_cast<cudaStream_t>(stream)), "rotary launch");
    return BACON_OK;
}

bacon_status bacon_block_norm(const bacon_block* block, bacon_stream stream)
{
    g_last_error.clear();
    if (!block) return fail(BACON_EINVAL, "null argument");
    const bacon_block b = *block;
    if (b.tokens < 0 || b.width < 1 || b.width > BACON_MAX_WIDTH)
        return fail(BACON_EINVAL, "tokens must not be negative, width in [1, %d]", BACON_MAX_WIDTH);
    if (!known(b.dtype) || (b.residual_dtype != b.dtype && b.residual_dtype != BACON_FP32) ||
        (b.weight_dtype != b.dtype && b.weight_dtype != BACON_FP32))
        return fail(BACON_EINVAL, "unknown dtype, or a residual or weight dtype that is neither dtype nor fp32");
    if (b.post < BACON_NORM_NONE || b.post > BACON_NORM_LAYER || b.pre < BACON_NORM_NONE ||
        b.pre > BACON_NORM_LAYER)
        return fail(BACON_EINVAL, "unknown norm");
    if (b.activation < BACON_GATE_LINEAR || b.activation > BACON_GATE_SILU)
        return fail(BACON_EINVAL, "unknown activation %d", b.activation);
    if (!std::isfinite(b.scale) || !std::isfinite(b.weight_offset) || !std::isfinite(b.eps) ||
        b.eps < kLeastEps)
        return fail(BACON_EINVAL, "scale and weight_offset must be finite, eps at least 1e-20");
    if (b.tokens == 0) return BACON_OK;
    if (!b.sum && !b.normed) return fail(BACON_EINVAL, "neither sum nor normed is wanted");
    if (b.normed && b.pre == BACON_NORM_NONE) return fail(BACON_EINVAL, "normed needs a pre norm");
    if (!b.y) return fail(BACON_EINVAL, "null y");
    const int bytes = size_of(b.dtype), wide = size_of(b.residual_dtype), thin = size_of(b.weight_dtype);
    if (!aligned_to(b.y, bytes) || !aligned_to(b.gate, bytes) || !aligned_to(b.normed, bytes) ||
        !aligned_to(b.x, wide) || !aligned_to(b.sum, wide) || !aligned_to(b.post_weight, thin) ||
        !aligned_to(b.post_bias, thin) || !aligned_to(b.pre_weight, thin) || !aligned_to(b.pre_bias, thin))
        return fail(BACON_EINVAL, "a pointer is not aligned to its type");
    const long long most = 1ll << 56;
    for (long long s : {b.y_token, b.x_token, b.gate_token, b.sum_token, b.normed_token})
        if (s < 0 || s >= most) return fail(BACON_EINVAL, "a stride is out of range");
    if (b.tokens > 1 && ((b.sum && b.sum_token < b.width) || (b.normed && b.normed_token < b.width)))
        return fail(BACON_EINVAL, "rows of an output overlap");
    BACON_CUDA(launch_block_norm(b, static_cast<cudaStream_t>(stream)), "norm launch");
    return BACON_OK;
}

bacon_status bacon_logits_create(bacon_logits** out, int vocab)
{
    g_last_error.clear();
    if (!out) return fail(BACON_EINVAL, "null argument");
    *out = nullptr;
    if (vocab < 1 || vocab > BACON_MAX_VOCAB)
        return fail(BACON_EINVAL, "vocab must be in [1, %d], got %d", BACON_MAX_VOCAB, vocab);
    bacon_logits* l = new (std::nothrow) bacon_logits;
    if (!l) return fail(BACON_ENOMEM, "host allocation failed");
    l->vocab = vocab;
    cudaError_t e = cudaGetDevice(&l->device);
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&l->err), sizeof(int));
    if (e == cudaSuccess) e = clear_now(l->err, sizeof(int));
    if (e != cudaSuccess) {
        bacon_logits_destroy(l);
        const bacon_status rc = cuda_fail(e, "logits creation");
        return e == cudaErrorMemoryAllocation ? fail(BACON_ENOMEM, "device allocation failed") : rc;
    }
    *out = l;
    return BACON_OK;
}

void bacon_logits_destroy(bacon_logits* logits)
{
    if (!logits) return;
    DeviceGuard dg(logits->device);
    if (logits->err) cudaFree(logits->err);
    delete logits;
}

bacon_status bacon_logits_process(bacon_logits* logits, const bacon_logits_rows* rows,
                                  bacon_stream stream)
{
    g_last_error.clear();
    if (!logits || !rows) return fail(BACON_EINVAL, "null argument");
    bacon_logits_rows r = *rows;
    const int vocab = logits->vocab;
    if (r.rows < 0 || r.rows > 1 << 26) return fail(BACON_EINVAL, "rows must be in [0, 2^26]");
    if (!known(r.dtype) || (r.out && r.out_dtype != r.dtype && r.out_dtype != BACON_FP32))
        return fail(BACON_EINVAL, "unknown dtype, or an out dtype that is neither dtype nor fp32");
    if (!r.out) r.out_dtype = r.dtype;
    if (r.rows == 0) return BACON_OK;
    if (!r.out && !r.best && !r.logprob && !r.lse) return fail(BACON_EINVAL, "nothing is wanted");
    if (r.biases < 0 || r.biases > BACON_MAX_BIASES)
        return fail(BACON_EINVAL, "biases must be in [0, %d], got %d", BACON_MAX_BIASES, r.biases);
    if (r.tokens && r.lengths &&
        (r.requests < 1 || r.capacity < 0 || r.capacity > BACON_MAX_HISTORY || r.token_stride < 0))
        return fail(BACON_EINVAL, "requests must be positive, capacity in [0, %d]", BACON_MAX_HISTORY);
    if (r.tokens && !r.lengths) return fail(BACON_EINVAL, "tokens need lengths");
    if (r.biases && (!r.bias_tokens || !r.bias_values))
        return fail(BACON_EINVAL, "null list of biases");
    if (!r.logits) return fail(BACON_EINVAL, "null logits");
    if (!aligned_to(r.logits, size_of(r.dtype)) || !aligned_to(r.out, size_of(r.out_dtype)))
        return fail(BACON_EINVAL, "a pointer is not aligned to its type");
    for (const void* p : {(const void*)r.tokens, (const void*)r.request, (const void*)r.prompt,
                          (const void*)r.lengths, (const void*)r.repetition, (const void*)r.frequency,
                          (const void*)r.presence, (const void*)r.temperature, (const void*)r.bias_tokens,
                          (const void*)r.bias_values, (const void*)r.mask, (const void*)r.best,
                          (const void*)r.logprob, (const void*)r.lse})
        if (!aligned_to(p, 4)) return fail(BACON_EINVAL, "a pointer is not aligned to its type");
    const long long most = 1ll << 56;
    if (r.row_stride < 0 || r.row_stride >= most || r.out_stride < 0 || r.out_stride >= most ||
        r.token_stride >= most || r.mask_stride < 0 || r.mask_stride >= most)
        return fail(BACON_EINVAL, "a stride is out of range");
    if (r.rows > 1 && r.out && r.out_stride < vocab)
        return fail(BACON_EINVAL, "rows of the output overlap");
    if (r.out == r.logits && (r.out_dtype != r.dtype || (r.rows > 1 && r.out_stride != r.row_stride)))
        return fail(BACON_EINVAL, "logits in place keep their type and stride");
    if (!r.biases) r.bias_tokens = nullptr, r.bias_values = nullptr;
    DeviceGuard dg(logits->device);
    BACON_CUDA(launch_logits(r, vocab, logits->err, static_cast<cudaStream_t>(stream)), "logits launch");
    return BACON_OK;
}

bacon_status bacon_logits_sync(bacon_logits* logits, bacon_stream stream)
{
    g_last_error.clear();
    if (!logits) return fail(BACON_EINVAL, "null logits");
    DeviceGuard dg(logits->device);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    int flag = 0;
    BACON_CUDA(cudaMemcpyAsync(&flag, logits->err, sizeof(int), cudaMemcpyDeviceToHost, st),
               "error flag read");
    BACON_CUDA(cudaStreamSynchronize(st), "stream synchronisation");
    if (!flag) return BACON_OK;
    BACON_CUDA(cudaMemsetAsync(logits->err, 0, sizeof(int), st), "error flag reset");
    BACON_CUDA(cudaStreamSynchronize(st), "stream synchronisation");
    if (flag == kLogitsBadHistory)
        return fail(BACON_EINVAL, "a length, prompt or request was outside the history");
    if (flag == kLogitsBadBias) return fail(BACON_EINVAL, "a bias is of no token");
    if (flag == kLogitsBadValue)
        return fail(BACON_EINVAL, "a penalty or temperature was out of its range");
    return fail(BACON_ECUDA, "unknown device error code %d", flag);
}

}  // extern "C"
