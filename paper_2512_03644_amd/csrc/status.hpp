// Errors of the HIP runtime as status codes.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ffsnap.h"

namespace ffsnap {

// Keeps the error's text for ff_strerror on this thread; FF_ERR_HIP.  The runtime's own record of it is cleared: a later call asks
// there whether its launch has failed.
int hip_fail(hipError_t e);
// The same for an allocation: FF_ERR_NOMEM if there was no memory.
inline int alloc_fail(hipError_t e)
{
    const int rc = hip_fail(e);
    return e == hipErrorOutOfMemory ? FF_ERR_NOMEM : rc;
}

}  // namespace ffsnap

#define FF_HIP_TRY(expr)                                   \
    do {                                                   \
        hipError_t e_ = (expr);                            \
        if (e_ != hipSuccess) return ffsnap::hip_fail(e_); \
    } while (0)
