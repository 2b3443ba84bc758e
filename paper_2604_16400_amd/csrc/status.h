// Failures of HIP calls behind the C ABI.
#pragma once
#include <hip/hip_runtime.h>

namespace collm {

// COLLM_E_HIP; keeps the text for collm_last_error()
int hip_fail(hipError_t e, const char *what);

#define HIP_TRY(expr)                                              \
    do {                                                           \
        hipError_t e_ = (expr);                                    \
        if (e_ != hipSuccess) return ::collm::hip_fail(e_, #expr); \
    } while (0)

}  // namespace collm
