// Layer norm and its gradients (norm.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ffsnap {

struct NormArgs {
    const uint8_t* x;
    uint64_t n_rows, width, x_stride;
    const uint8_t *weight, *bias;  // bias: or null
    float eps;
    float *mean, *rstd;  // forward: or null
    // forward: y; backward: dx
    uint8_t* out;
    uint64_t out_stride;
    // backward
    const uint8_t* dy;
    uint64_t dy_stride;
    uint8_t *dweight, *dbias;  // or null
    float* parts;              // [workgroup][dweight, dbias][width]
};

uint64_t norm_workspace(uint64_t n_rows, uint64_t width);
hipError_t launch_norm(const NormArgs& a, uint32_t dtype, hipStream_t stream);
hipError_t launch_norm_grad(const NormArgs& a, uint32_t dtype, hipStream_t stream);

}  // namespace ffsnap
