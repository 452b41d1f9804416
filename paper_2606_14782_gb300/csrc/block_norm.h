// Kernel interface of the step between two blocks.
#pragma once

#include <cuda_runtime.h>

#include "bacon.h"

namespace bacon {

// The call with all checks done.
cudaError_t launch_block_norm(const bacon_block& b, cudaStream_t st);

}  // namespace bacon
