// Errors of the HIP runtime as status codes.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ffsnap.h"

namespace ffsnap {

// Keeps the error's text for ff_strerror on this thread; FF_ERR_HIP.
int hip_fail(hipError_t e);

}  // namespace ffsnap

#define FF_HIP_TRY(expr)                                   \
    do {                                                   \
        hipError_t e_ = (expr);                            \
        if (e_ != hipSuccess) return ffsnap::hip_fail(e_); \
    } while (0)
