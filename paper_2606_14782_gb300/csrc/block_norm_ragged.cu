// The step between two blocks: rows whose pieces have ends that are not whole, or
// that start anywhere (block_norm.cuh says how they work).
#include "block_norm.cuh"

namespace bacon {
namespace {

template <int DTYPE, int RESIDUAL>
cudaError_t ragged_rows(const bacon_block& b, const Choices& c, cudaStream_t st)
{
    const int lead = c.vectors ? 16 / Eight<DTYPE>::kBytes - 1 : 0;
    const int pieces = (b.width + lead + 7) / 8;  // of a row, at most
    if (pieces <= 32) return launch_rows<DTYPE, RESIDUAL, 1, true, false>(b, c, pieces, st);
    if (pieces <= 1024) return launch_rows<DTYPE, RESIDUAL, 2, false, false>(b, c, pieces, st);
    return launch_rows<DTYPE, RESIDUAL, 9, false, false>(b, c, pieces, st);
}

}  // namespace

cudaError_t launch_ragged_norm(const bacon_block& b, const Choices& c, cudaStream_t st)
{
    const bool wide = b.residual_dtype == BACON_FP32;
    if (b.dtype == BACON_FP32) return ragged_rows<BACON_FP32, BACON_FP32>(b, c, st);
    if (b.dtype == BACON_BF16)
        return wide ? ragged_rows<BACON_BF16, BACON_FP32>(b, c, st) : ragged_rows<BACON_BF16, BACON_BF16>(b, c, st);
    return wide ? ragged_rows<BACON_FP16, BACON_FP32>(b, c, st) : ragged_rows<BACON_FP16, BACON_FP16>(b, c, st);
}

}  // namespace bacon
