// Kernel interface of the rules on logits.
#pragma once

#include <cuda_runtime.h>

#include "bacon.h"

namespace bacon {

// Codes of the handle's error word (bacon_logits_sync names them).
constexpr int kLogitsBadHistory = 1;  // a length, prompt or request outside the history
constexpr int kLogitsBadBias = 2;     // a bias of no token
constexpr int kLogitsBadValue = 3;    // a parameter out of its range

// The call with all checks done.
cudaError_t launch_logits(const bacon_logits_rows& r, int vocab, int* err, cudaStream_t st);

}  // namespace bacon
