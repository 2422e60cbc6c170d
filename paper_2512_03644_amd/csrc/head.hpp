// Cross entropy over a vocabulary from hidden states, and its gradients (head.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ffsnap.h"

namespace ffsnap {

uint64_t head_workspace(const ff_head_batch& b, bool grad);
hipError_t launch_head(const ff_head_batch& b, float* logp, void* dhidden, uint64_t dhidden_stride, void* dweight, uint64_t dweight_stride,
                       ff_head_stats* stats, void* workspace, hipStream_t stream);

}  // namespace ffsnap
