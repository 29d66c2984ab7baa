// Sizes and types as the host side of the operators counts them, without HIP.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../../include/comp_ams_operators.h"

namespace cams_ops {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline size_t type_size(int32_t type) { return type == COMP_AMS_F32 ? 4 : 2; }
inline bool known_type(int32_t type) { return type == COMP_AMS_F32 || type == COMP_AMS_BF16 || type == COMP_AMS_F16; }

}  // namespace cams_ops
