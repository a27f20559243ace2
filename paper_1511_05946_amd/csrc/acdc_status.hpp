// The HIP error behind ACDC_ERR_HIP, shared by the library's C entry points.
#pragma once

#include <hip/hip_runtime.h>

namespace acdc {

// Remembers e for acdc_last_hip_error (per thread); returns ACDC_ERR_HIP.
int hip_fail(hipError_t e);

}  // namespace acdc
