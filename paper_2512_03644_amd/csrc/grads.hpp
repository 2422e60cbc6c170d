// Gradient norm and clipping over a list of tensors (grads.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

#include "../../include/ffsnap.h"
#include "fused.hpp"

namespace ffsnap {

// What a wavefront takes at a time: up to kGradItemBytes of one tensor, in rows of 1 KiB.
struct GradItem {
    uint64_t begin;   // byte offset in the tensor
    uint32_t tensor;  // place in the list
    uint32_t what;    // bits 0..29 bytes, 30..31 the format (kGradF32, ...)
};
constexpr uint32_t kGradItemBytes = 8192;
constexpr uint32_t kGradF32 = 0, kGradBf16 = 1, kGradF16 = 2;

// Items of all tensors in the list's order, and the first item of every group of kGradsPerLaunch tensors, whose
// addresses fit a launch's arguments (one entry more: the end).  False if there would be more than 2^31.
bool build_grad_items(const ff_segment* segs, uint64_t n, std::vector<GradItem>& items, std::vector<uint32_t>& begin);

constexpr uint32_t kGradWaves = 4;  // of a workgroup
// Workgroups over n items: no more than the chip holds at once, each goes on to further items.
constexpr uint32_t kGradGroups = 512;
inline uint32_t grad_groups(uint32_t n_items)
{
    const uint32_t g = (n_items + kGradWaves - 1) / kGradWaves;
    return g < 1 ? 1 : g > kGradGroups ? kGradGroups : g;
}

// What a workgroup leaves for the sum of all.
struct GradPart {
    double sumsq;
    uint64_t n_nonfinite;
};

struct GradWork {
    const GradItem* items = nullptr;    // DEVICE
    const uint64_t* address = nullptr;  // DEVICE: of every tensor; null where every call brings its own
    std::vector<uint32_t> launch;       // build_grad_items
    uint64_t n = 0;                     // tensors
};

// What launch_grad_norm is given, zero before the first call.
uint64_t grad_workspace(const GradWork& work);

// grads: HOST array of addresses, or null for the list's own.
hipError_t launch_grad_norm(const GradWork& work, const void* const* grads, double inv_scale, double max_norm,
                            void* workspace, ff_grad_stats* stats, hipStream_t stream);
hipError_t launch_grad_join(const ff_grad_stats* parts, uint64_t n, double inv_scale, double max_norm,
                            ff_grad_stats* stats, hipStream_t stream);
hipError_t launch_grad_clip(const GradWork& work, const void* const* grads, const ff_grad_stats* stats,
                            hipStream_t stream);

}  // namespace ffsnap
