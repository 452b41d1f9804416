// The step between two blocks: rows whose pieces are all whole, and which kernel has
// a call's rows (block_norm.cuh says how they work).
#include "block_norm.cuh"

namespace bacon {
namespace {

// Whether rows at p, `stride` values apart, have pieces that start where y's do.
bool together(const bacon_block& b, const void* p, long long stride, int bytes, int y_bytes)
{
    if (!p) return true;
    const long long unit = 16 / bytes;  // values of 16 bytes
    if (b.tokens > 1 && (stride - b.y_token) % unit) return false;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(b.y);
    return ((long long)(a / bytes) - (long long)(y / y_bytes)) % unit == 0;
}

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <int DTYPE, int RESIDUAL>
cudaError_t even_rows(const bacon_block& b, const Choices& c, cudaStream_t st)
{
    const int pieces = b.width / 8;
    if (pieces <= 32) return launch_rows<DTYPE, RESIDUAL, 1, true, true>(b, c, pieces, st);
    if (pieces <= 128) return launch_rows<DTYPE, RESIDUAL, 4, true, true>(b, c, pieces, st);
    const bool few = b.tokens <= 152 * 2;
    if (few && pieces <= 1024) return launch_rows<DTYPE, RESIDUAL, 1, false, true>(b, c, pieces, st);
    // the most pieces a thread of which all but the last are there in every thread
    const auto tight = [&](int chunks) {
        const int threads = ((pieces + chunks - 1) / chunks + 31) / 32 * 32;
        return threads <= 512 && (chunks - 1) * threads <= pieces;
    };
    if (tight(4)) return launch_rows<DTYPE, RESIDUAL, 4, false, true>(b, c, pieces, st);
    if (tight(3)) return launch_rows<DTYPE, RESIDUAL, 3, false, true>(b, c, pieces, st);
    if (tight(2)) return launch_rows<DTYPE, RESIDUAL, 2, false, true>(b, c, pieces, st);
    return launch_rows<DTYPE, RESIDUAL, 8, false, true>(b, c, pieces, st);
}

}  // namespace

cudaError_t launch_block_norm(const bacon_block& b, cudaStream_t st)
{
    const int bytes = b.dtype == BACON_FP32 ? 4 : 2, wide = b.residual_dtype == BACON_FP32 ? 4 : 2;
    Choices c;
    const bool full = b.gate && b.gate_channel && b.gate_token;
    c.vectors = together(b, b.x, b.x_token, wide, bytes) && together(b, b.sum, b.sum_token, wide, bytes) &&
                together(b, b.normed, b.normed_token, bytes, bytes) &&
                (!full || together(b, b.gate, b.gate_token, bytes, bytes));
    c.post_aligned = aligned(b.post_weight) && aligned(b.post_bias);
    c.pre_aligned = aligned(b.pre_weight) && aligned(b.pre_bias);
    c.gate_aligned = full || !b.gate_channel || aligned(b.gate);
    c.per_channel = 1.0f / (float)b.width;
    const bool even = c.vectors && b.width % 8 == 0 && aligned(b.y) &&
                      (b.tokens == 1 || b.y_token * bytes % 16 == 0) && c.post_aligned && c.pre_aligned &&
                      c.gate_aligned;
    if (!even) return launch_ragged_norm(b, c, st);
    if (b.dtype == BACON_FP32) return even_rows<BACON_FP32, BACON_FP32>(b, c, st);
    if (b.dtype == BACON_BF16)
        return wide == 4 ? even_rows<BACON_BF16, BACON_FP32>(b, c, st) : even_rows<BACON_BF16, BACON_BF16>(b, c, st);
    return wide == 4 ? even_rows<BACON_FP16, BACON_FP32>(b, c, st) : even_rows<BACON_FP16, BACON_FP16>(b, c, st);
}

}  // namespace bacon
