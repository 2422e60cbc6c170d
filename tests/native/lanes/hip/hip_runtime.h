// Stand-in for the HIP runtime's header with which a kernel's source runs on the CPU (see lanes.hpp): just what embed.hip and norm.hip
// and the headers under them use.
#pragma once
#include <math.h>
#include <stdint.h>

#include "../lanes.hpp"

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __launch_bounds__(threads)
#define __shared__ static

struct dim3 {
    uint32_t x, y, z;
    dim3(uint32_t x = 1, uint32_t y = 1, uint32_t z = 1) : x(x), y(y), z(z) {}
};
struct uint2 {
    uint32_t x, y;
};
typedef int hipError_t;
typedef void* hipStream_t;
constexpr hipError_t hipSuccess = 0;
inline hipError_t hipGetLastError() { return hipSuccess; }

#define threadIdx (lanes::thread())
#define blockIdx (lanes::g_block)
#define gridDim (lanes::g_grid)

inline void __syncthreads() { lanes::meet_workgroup(); }
inline uint64_t __ballot(bool x) { return lanes::ballot(x); }
inline int __popcll(uint64_t x) { return __builtin_popcountll(x); }
template <class T>
T __shfl_xor(T v, int d) { return lanes::exchange(v, lanes::lane() ^ d); }
template <class T>
T __shfl_down(T v, int d) { return lanes::exchange(v, lanes::lane() + d < 64 ? lanes::lane() + d : lanes::lane()); }
template <class T>
T __shfl_up(T v, int d) { return lanes::exchange(v, lanes::lane() >= d ? lanes::lane() - d : lanes::lane()); }
// (lanes take turns: nothing comes between)
inline uint32_t atomicAdd(uint32_t* p, uint32_t v)
{
    const uint32_t old = *p;
    *p += v;
    return old;
}

#define __builtin_amdgcn_readfirstlane(x) lanes::exchange(x, 0)
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) \
    lanes::launch(grid, block, [&] { kernel(__VA_ARGS__); })
