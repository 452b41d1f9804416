// Kernel interface of the step between two blocks.
#pragma once

#include <cuda_runtime.h>

#include "bacon.h"

namespace bacon {

// The call with all checks done; rows that are not of whole pieces of 16 bytes.
cudaError_t launch_block_norm(const bacon_block& b, cudaStream_t st);
cudaError_t launch_ragged_norm(const bacon_block& b, cudaStream_t st);

}  // namespace bacon
