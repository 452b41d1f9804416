// A rotary call's arguments, checked: shared by its own call and the cache's.
#pragma once

#include "bacon.h"

namespace bacon {

struct RotaryArgs;
bacon_status rotary_args(const bacon_rotary* rotary, int requests, int tokens, const bacon_rows* q,
                         const bacon_rows* k, bool k_writes, int dtype, int weight_dtype, float eps,
                         float weight_offset, int transposed, const int32_t* positions,
                         RotaryArgs* out);

}  // namespace bacon
