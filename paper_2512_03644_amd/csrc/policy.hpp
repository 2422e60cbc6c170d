// Clipped policy loss with a KL term, and its gradient (policy.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ffsnap.h"

namespace ffsnap {

// What a token adds to the sums.
struct PolicyPart {
    double loss, kl;
    uint32_t what, unused;  // kTokenCounts, ...
};
constexpr uint32_t kTokenCounts = 1, kTokenClipped = 2, kTokenInvalid = 4;

uint64_t policy_workspace(uint64_t n_tokens, uint64_t vocab);
hipError_t launch_policy(const ff_policy_batch& b, float* logp, float* token_loss, void* dlogits, uint64_t grad_stride,
                         ff_policy_stats* stats, void* workspace, hipStream_t stream);

}  // namespace ffsnap
