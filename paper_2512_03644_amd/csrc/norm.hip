// Layer norm, forward and backward, for gfx950.
//
// y = (x - mean) rstd w + b, rstd = 1 / sqrt(var + eps).  A group of threads -- a wavefront, or a workgroup -- holds a row in registers: the mean
// first, then the squares of what is left of it, so that a large mean costs the variance nothing.  Backward, with xh = (x - mean) rstd and g =
// dy w: dx = rstd (g - mean(g) - xh mean(g xh)); dw = sum of dy xh, db = sum of dy over the rows: a group keeps
// them in registers over the rows that it takes, and leaves its part in the workspace; a second launch joins the parts in their order.
//
// What bounds it: memory.
#include "norm.hpp"

#include <algorithm>

#include "rows.h"

namespace ffsnap {

namespace {

constexpr int kBlock = 256;             // threads of a workgroup whose wavefronts take rows of their own
constexpr uint32_t kMostGroups = 1024;  // that leave parts of dw and db

template <int GROUP>
constexpr int block_of()
{
    return GROUP == kWaveSize ? kBlock : GROUP;
}

// Sums over the group, the same in every thread.  `turn`: 0 and 1 in turn.
template <int GROUP, int N>
__device__ __forceinline__ void sum_over(float (&v)[N], int turn)
{
    for (int d = 32; d; d /= 2)
        for (int i = 0; i < N; i++) v[i] += __shfl_xor(v[i], d);
    if constexpr (GROUP > kWaveSize) {
        __shared__ float part[2][N][GROUP / kWaveSize];
        if (threadIdx.x % kWaveSize == 0)
            for (int i = 0; i < N; i++) part[turn][i][threadIdx.x / kWaveSize] = v[i];
        __syncthreads();
        for (int i = 0; i < N; i++) {
            v[i] = 0;
            for (int k = 0; k < GROUP / kWaveSize; k++) v[i] += part[turn][i][k];
        }
    }
}

__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

// Of the eight elements from `at` on, those that the row has.
__device__ __forceinline__ f32x8 cut(f32x8 v, uint32_t at, uint32_t width)
{
    if (at + kLaneItems > width)
        for (uint32_t i = 0; i < kLaneItems; i++) v[i] = at + i < width ? v[i] : 0.f;
    return v;
}

template <uint32_t DTYPE, int GROUP, int K>
__global__ __launch_bounds__(block_of<GROUP>()) void norm_kernel(const NormArgs a)
{
    using I = Items<DTYPE>;
    constexpr uint32_t kPer = block_of<GROUP>() / GROUP;
    const uint32_t width = static_cast<uint32_t>(a.width), thread = threadIdx.x % GROUP;
    const float each = 1.f / static_cast<float>(width);
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * kPer;
    int turn = 0;
    for (uint64_t r = static_cast<uint64_t>(blockIdx.x) * kPer + threadIdx.x / GROUP; r < a.n_rows; r += step) {
        const uint8_t* const row = a.x + r * a.x_stride * I::kBytes;
        typename I::Held h[K];
        float s[1] = {0.f};
        static_for<K>([&](auto i) {
            const uint32_t at = (i * GROUP + thread) * kLaneItems;
            if (at < width) {
                h[int(i)] = I::load(row, at, width);
                s[0] += sum8(I::wide(h[int(i)]));
            }
        });
        sum_over<GROUP>(s, turn);
        turn ^= 1;
        const float mean = s[0] * each;
        s[0] = 0.f;
        static_for<K>([&](auto i) {
            const uint32_t at = (i * GROUP + thread) * kLaneItems;
            if (at < width) {
                const f32x8 d = cut(I::wide(h[int(i)]) - mean, at, width);
                s[0] += sum8(d * d);
            }
        });
        sum_over<GROUP>(s, turn);
        turn ^= 1;
        const float rstd = 1.f / sqrtf(s[0] * each + a.eps);
        static_for<K>([&](auto i) {
            const uint32_t at = (i * GROUP + thread) * kLaneItems;
            if (at < width) {
                f32x8 y = (I::wide(h[int(i)]) - mean) * rstd * I::wide(I::load(a.weight, at, width));
                if (a.bias) y += I::wide(I::load(a.bias, at, width));
                I::store(a.out + r * a.out_stride * I::kBytes, at, width, I::narrow(y));
            }
        });
        if (thread == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

template <uint32_t DTYPE, int GROUP, int K>
__global__ __launch_bounds__(block_of<GROUP>()) void norm_grad_kernel(const NormArgs a)
{
    using I = Items<DTYPE>;
    constexpr uint32_t kPer = block_of<GROUP>() / GROUP;
    const uint32_t width = static_cast<uint32_t>(a.width), thread = threadIdx.x % GROUP;
    const float each = 1.f / static_cast<float>(width);
    const uint32_t group = blockIdx.x * kPer + threadIdx.x / GROUP;
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * kPer;
    typename I::Held w[K];
    f32x8 dw[K], db[K];
    static_for<K>([&](auto i) {
        const uint32_t at = (i * GROUP + thread) * kLaneItems;
        if (at < width) w[int(i)] = I::load(a.weight, at, width);
        dw[int(i)] = db[int(i)] = f32x8{};
    });
    int turn = 0;
    for (uint64_t r = group; r < a.n_rows; r += step) {
        const uint8_t *const row = a.x + r * a.x_stride * I::kBytes, *const grad = a.dy + r * a.dy_stride * I::kBytes;
        const float mean = a.mean[r], rstd = a.rstd[r];
        typename I::Held x[K], dy[K];
        static_for<K>([&](auto i) {
            const uint32_t at = (i * GROUP + thread) * kLaneItems;
            if (at < width) {
                x[int(i)] = I::load(row, at, width);
                dy[int(i)] = I::load(grad, at, width);
            }
        });
        float s[2] = {0.f, 0.f};
        static_for<K>([&](auto i) {
            const uint32_t at = (i * GROUP + thread) * kLaneItems;
            if (at < width) {
                const f32x8 normed = (I::wide(x[int(i)]) - mean) * rstd, d = I::wide(dy[int(i)]), g = d * I::wide(w[int(i)]);
                s[0] += sum8(g);
                s[1] += sum8(g * normed);
                dw[int(i)] += d * normed;
                db[int(i)] += d;
            }
        });
        sum_over<GROUP>(s, turn);
        turn ^= 1;
        const float c0 = s[0] * each, c1 = s[1] * each;
        static_for<K>([&](auto i) {
            const uint32_t at = (i * GROUP + thread) * kLaneItems;
            if (at < width) {
                const f32x8 normed = (I::wide(x[int(i)]) - mean) * rstd, g = I::wide(dy[int(i)]) * I::wide(w[int(i)]);
                I::store(a.out + r * a.out_stride * I::kBytes, at, width, I::narrow(rstd * (g - c0 - normed * c1)));
            }
        });
    }
    if (!a.dweight && !a.dbias) return;
    uint8_t* const out = reinterpret_cast<uint8_t*>(a.parts + 2ull * group * width);
    static_for<K>([&](auto i) {
        const uint32_t at = (i * GROUP + thread) * kLaneItems;
        if (at < width) {
            Items<FF_F32>::store(out, at, width, Items<FF_F32>::narrow(dw[int(i)]));
            Items<FF_F32>::store(out + 4ull * width, at, width, Items<FF_F32>::narrow(db[int(i)]));
        }
    });
}

// Columns of dw (blockIdx.y 0) and db (1): the parts of all groups.
constexpr uint32_t kColumns = 64, kJoinRows = 16;
template <uint32_t DTYPE>
__global__ __launch_bounds__(kColumns* kJoinRows) void norm_join_kernel(const NormArgs a, const uint32_t groups)
{
    using I = Items<DTYPE>;
    __shared__ float part[kJoinRows][kColumns];
    uint8_t* const out = blockIdx.y ? a.dbias : a.dweight;
    const uint32_t width = static_cast<uint32_t>(a.width), c = threadIdx.x % kColumns, k = threadIdx.x / kColumns;
    const uint32_t at = blockIdx.x * kColumns + c;
    if (!out) return;
    float s = 0.f;
    if (at < width)
        for (uint32_t g = k; g < groups; g += kJoinRows) s += as_global(a.parts)[(2ull * g + blockIdx.y) * width + at];
    part[k][c] = s;
    __syncthreads();
    if (k || at >= width) return;
    for (uint32_t i = 1; i < kJoinRows; i++) s += part[i][c];
    I::put(out + static_cast<uint64_t>(at) * I::kBytes, s);
}

// fn(group size, K): the fewest threads that hold a row of this width.
template <class Fn>
void choose(uint64_t width, Fn&& fn)
{
    using std::integral_constant;
    if (width <= 512) fn(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (width <= 2048) fn(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (width <= 4096) fn(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (width <= 8192) fn(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    else fn(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

// Workgroups of the backward pass, and the groups in them.
uint32_t grad_groups(uint64_t n_rows, uint64_t width, uint32_t* blocks)
{
    uint32_t groups = 0;
    choose(width, [&](auto group, auto) {
        constexpr uint32_t per = block_of<group>() / group;
        *blocks = static_cast<uint32_t>(std::min<uint64_t>((n_rows + per - 1) / per, kMostGroups / per));
        *blocks = std::max(*blocks, 1u);
        groups = *blocks * per;
    });
    return groups;
}

template <uint32_t DTYPE>
hipError_t forward(const NormArgs& a, hipStream_t stream)
{
    choose(a.width, [&](auto group, auto k) {
        constexpr int threads = block_of<group>();
        constexpr uint32_t per = threads / group;
        const uint32_t blocks = static_cast<uint32_t>(std::min<uint64_t>((a.n_rows + per - 1) / per, 1u << 20));
        hipLaunchKernelGGL((norm_kernel<DTYPE, group, k>), dim3(blocks), dim3(threads), 0, stream, a);
    });
    return hipGetLastError();
}

template <uint32_t DTYPE>
hipError_t backward(const NormArgs& a, hipStream_t stream)
{
    uint32_t blocks, groups = grad_groups(a.n_rows, a.width, &blocks);
    choose(a.width, [&](auto group, auto k) {
        hipLaunchKernelGGL((norm_grad_kernel<DTYPE, group, k>), dim3(blocks), dim3(block_of<group>()), 0, stream, a);
    });
    if (a.dweight || a.dbias)
        hipLaunchKernelGGL(norm_join_kernel<DTYPE>, dim3(static_cast<uint32_t>((a.width + kColumns - 1) / kColumns), 2), dim3(kColumns * kJoinRows), 0, stream,
                           a, groups);
    return hipGetLastError();
}

}  // namespace

uint64_t norm_workspace(uint64_t n_rows, uint64_t width)
{
    uint32_t blocks;
    return grad_groups(n_rows, width, &blocks) * 8ull * width;
}

hipError_t launch_norm(const NormArgs& a, uint32_t dtype, hipStream_t stream)
{
    if (!a.n_rows) return hipSuccess;
    return dtype == FF_BF16 ? forward<FF_BF16>(a, stream) : dtype == FF_F16 ? forward<FF_F16>(a, stream) : forward<FF_F32>(a, stream);
}

hipError_t launch_norm_grad(const NormArgs& a, uint32_t dtype, hipStream_t stream)
{
    return dtype == FF_BF16 ? backward<FF_BF16>(a, stream) : dtype == FF_F16 ? backward<FF_F16>(a, stream) : backward<FF_F32>(a, stream);
}

}  // namespace ffsnap
