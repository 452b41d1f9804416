// Kernel interface of the step between two blocks.
#pragma once

#include <cuda_runtime.h>

#include "bacon.h"

namespace bacon {

// What the host found of a call's addresses.
struct Choices {
    bool vectors;  // pieces of y, x, gate, sum and normed start at 16 bytes together
    bool post_aligned, pre_aligned, gate_aligned;
    float per_channel;  // 1 / width
};

// The call with all checks done, and its rows that are not of whole pieces.
cudaError_t launch_block_norm(const bacon_block& b, cudaStream_t st);
cudaError_t launch_ragged_norm(const bacon_block& b, const Choices& c, cudaStream_t st);

}  // namespace bacon
