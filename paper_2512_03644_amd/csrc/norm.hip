// Layer norm, forward and backward, for gfx950.
//
// y = (x - mean) rstd w + b, rstd = 1 / sqrt(var + eps).  A group of threads -- a wavefront, or a workgroup -- holds a row in registers: the mean
// first, then the squares of what is left of it, so that a large mean costs the variance nothing.  Quotients by the width are exact where they can be (Divisor):
// of a row of one value of few bits nothing is left, whatever the value.  Backward, with xh = (x - mean) rstd and g =
// dy w: dx = rstd (g - mean(g) - xh mean(g xh)); dw = sum of dy xh, db = sum of dy over the rows: a group keeps
// them in registers over the rows that it takes, and leaves its part in the workspace; a second launch joins the parts in their order.
//
// What bounds it: memory.  Forward, 16,384 rows of 8192 bf16 elements 80 to 82 us (6.6 TB/s), backward 138 to 143 (5.7 TB/s); a row of 4096 2.7 us, launch included.
#include "norm.hpp"

#include <algorithm>

#include "rows.h"

namespace ffsnap {

namespace {

constexpr int kBlock = 256;             // threads of a workgroup whose wavefronts take rows of their own
// (us, 512 / 2048 / 16,384 workgroups: 16,384 rows of 8192 bf16 elements 85 / 80 / 92, 4096 of 4096 14.3 / 12.0 / 12.8)
constexpr uint32_t kForwardBlocks = 2048;
// Workgroups of the backward pass, each of which leaves a part of dw and db: those of 512 threads and more have a compute unit to themselves.  (Us, with all
// gradients, half as many / these / twice as many: 16,384 rows of 4096 89 / 78 / 88; of 8192 - / 138 / 143; 4096 of 1024 12.3 / 12.5 / 15.3.)
constexpr uint32_t kMostBlocks = 512, kMostWideBlocks = 256;
// Up to so many rows, dw and db are summed straight from them, in the same launch.  (Us, so / in two launches: 200 rows of 4096 8.7 / 11.2, 1000 of 8192 21 / 18.4.)
constexpr uint32_t kFewRows = 512;

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

// Quotients by the width: the product with its reciprocal, and what that leaves of the sum divided likewise.  A quotient that 32 bits hold comes out
// exactly.  (The division that the compiler makes takes ten operations, and 155 us of 16,384 rows of 8192 bf16 elements backward instead of 143.)
struct Divisor {
    float of, each;
    __device__ explicit Divisor(uint32_t width) : of(static_cast<float>(width)), each(1.f / of) {}
    __device__ __forceinline__ float quotient(float s) const
    {
        const float q = s * each;
        return __builtin_isfinite(q) ? fmaf(fmaf(-q, of, s), each, q) : q;
    }
};

// fn(i, at) for the thread's K places in a row.
template <int GROUP, int K, class Fn>
__device__ __forceinline__ void places(uint32_t thread, uint32_t width, Fn&& fn)
{
    static_for<K>([&](auto i) {
        const uint32_t at = (i * GROUP + thread) * kLaneItems;
        if (at < width) fn(i, at);
    });
}

template <class I, int GROUP, int K, bool PAST>
__global__ __launch_bounds__(block_of<GROUP>()) void norm_kernel(const NormArgs a)
{
    constexpr uint32_t kPer = block_of<GROUP>() / GROUP;
    const uint32_t width = static_cast<uint32_t>(a.width), thread = threadIdx.x % GROUP;
    const Divisor of(width);
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * kPer;
    typename I::Held w[K], b[K], h[K], next[K];
    auto fetch = [&](typename I::Held (&to)[K], uint64_t r) {
        places<GROUP, K>(thread, width, [&](auto i, uint32_t at) { to[int(i)] = I::load(a.x + r * a.x_stride * I::kBytes, at, width); });
    };
    uint64_t r = static_cast<uint64_t>(blockIdx.x) * kPer + threadIdx.x / GROUP;
    if (r < a.n_rows) fetch(next, r);
    places<GROUP, K>(thread, width, [&](auto i, uint32_t at) {
        w[int(i)] = I::load(a.weight, at, width);
        if (a.bias) b[int(i)] = I::load(a.bias, at, width);
    });
    int turn = 0;
    for (; r < a.n_rows; r += step) {
        static_for<K>([&](auto i) { h[int(i)] = next[int(i)]; });
        if (r + step < a.n_rows) fetch(next, r + step);
        float s[1] = {0.f};
        places<GROUP, K>(thread, width, [&](auto i, uint32_t at) { s[0] += sum8(I::cut(I::wide(h[int(i)]), at, width)); });
        sum_over<GROUP>(s, turn);
        turn ^= 1;
        const float mean = of.quotient(s[0]);
        s[0] = 0.f;
        places<GROUP, K>(thread, width, [&](auto i, uint32_t at) {
            const f32x8 d = I::cut(I::wide(h[int(i)]) - mean, at, width);
            s[0] += sum8(d * d);
        });
        sum_over<GROUP>(s, turn);
        turn ^= 1;
        const float rstd = 1.f / sqrtf(of.quotient(s[0]) + a.eps);
        places<GROUP, K>(thread, width, [&](auto i, uint32_t at) {
            f32x8 y = (I::wide(h[int(i)]) - mean) * rstd * I::wide(w[int(i)]);
            if (a.bias) y += I::wide(b[int(i)]);
            I::template store<PAST>(a.out + r * a.out_stride * I::kBytes, at, width, I::narrow(y));
        });
        if (thread == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

// 32 columns of dw and db, from all rows.
constexpr uint32_t kColumns = 32;
template <class I, int THREADS>
__device__ __forceinline__ void columns(const NormArgs& a, const uint32_t block)
{
    constexpr uint32_t kAcross = THREADS / kColumns, kAhead = 8;
    __shared__ float part[2][kAcross][kColumns + 1];
    const uint32_t width = static_cast<uint32_t>(a.width), n = static_cast<uint32_t>(a.n_rows), c = threadIdx.x % kColumns, k = threadIdx.x / kColumns;
    const uint32_t at = block * kColumns + c;
    float dw = 0.f, db = 0.f;
    if (at < width)
        for (uint32_t first = k; first < n; first += kAcross * kAhead) {
            float x[kAhead], dy[kAhead], mean[kAhead], rstd[kAhead];
            static_for<kAhead>([&](auto i) {
                const uint64_t r = first + i * kAcross < n ? first + i * kAcross : k;
                x[int(i)] = I::one(a.x + (r * a.x_stride + at) * I::kBytes);
                dy[int(i)] = I::one(a.dy + (r * a.dy_stride + at) * I::kBytes);
                mean[int(i)] = a.mean[r];
                rstd[int(i)] = a.rstd[r];
            });
            static_for<kAhead>([&](auto i) {
                if (first + i * kAcross >= n) return;
                dw += dy[int(i)] * ((x[int(i)] - mean[int(i)]) * rstd[int(i)]);
                db += dy[int(i)];
            });
        }
    part[0][k][c] = dw;
    part[1][k][c] = db;
    __syncthreads();
    if (k >= 2 || at >= width) return;
    uint8_t* const out = k ? a.dbias : a.dweight;
    if (!out) return;
    float s = 0.f;
    for (uint32_t i = 0; i < kAcross; i++) s += part[k][i][c];
    I::put(out + static_cast<uint64_t>(at) * I::kBytes, s);
}

// `column_blocks` workgroups behind the others make dw and db; with none of them, the rows' groups leave their parts.
template <class I, int GROUP, int K, bool PAST>
__global__ __launch_bounds__(block_of<GROUP>()) void norm_grad_kernel(const NormArgs a, const uint32_t column_blocks)
{
    const uint32_t blocks = gridDim.x - column_blocks;
    if (blockIdx.x >= blocks) {
        columns<I, block_of<GROUP>()>(a, blockIdx.x - blocks);
        return;
    }
    constexpr uint32_t kPer = block_of<GROUP>() / GROUP;
    const uint32_t width = static_cast<uint32_t>(a.width), thread = threadIdx.x % GROUP;
    const Divisor of(width);
    const uint32_t group = blockIdx.x * kPer + threadIdx.x / GROUP;
    const uint64_t step = static_cast<uint64_t>(blocks) * kPer;
    // The widest rows leave no registers for the next row, nor for this one while its sums are made: it is read again, from the caches.
    constexpr bool kHold = GROUP * K <= 1024;
    typename I::Held w[K];
    f32x8 dw[K], db[K];
    struct Row {
        typename I::Held x[K], dy[K];
        float mean, rstd;
    } next;
    auto load_x = [&](uint64_t r, uint32_t at) { return I::template load<PAST>(a.x + r * a.x_stride * I::kBytes, at, width); };
    auto load_dy = [&](uint64_t r, uint32_t at) { return I::template load<PAST>(a.dy + r * a.dy_stride * I::kBytes, at, width); };
    auto load_w = [&](uint32_t at) { return I::load(a.weight, at, width); };
    auto fetch = [&](Row& to, uint64_t r) {
        to.mean = a.mean[r];
        to.rstd = a.rstd[r];
        if constexpr (kHold)
            places<GROUP, K>(thread, width, [&](auto i, uint32_t at) {
                to.x[int(i)] = load_x(r, at);
                to.dy[int(i)] = load_dy(r, at);
            });
    };
    uint64_t r = group;
    if (r < a.n_rows) fetch(next, r);
    if constexpr (kHold) places<GROUP, K>(thread, width, [&](auto i, uint32_t at) { w[int(i)] = load_w(at); });
    static_for<K>([&](auto i) { dw[int(i)] = db[int(i)] = f32x8{}; });
    int turn = 0;
    for (; r < a.n_rows; r += step) {
        const Row now = next;
        if (r + step < a.n_rows) fetch(next, r + step);
        // fn(i, at, x normed, dy, dy * weight)
        auto each_place = [&](auto&& fn) {
            places<GROUP, K>(thread, width, [&](auto i, uint32_t at) {
                const f32x8 x = I::wide(kHold ? now.x[int(i)] : load_x(r, at)), d = I::cut(I::wide(kHold ? now.dy[int(i)] : load_dy(r, at)), at, width);
                fn(i, at, (x - now.mean) * now.rstd, d, d * I::wide(kHold ? w[int(i)] : load_w(at)));
            });
        };
        float s[2] = {0.f, 0.f};
        each_place([&](auto i, uint32_t, f32x8 normed, f32x8 d, f32x8 g) {
            s[0] += sum8(g);
            s[1] += sum8(g * normed);
            dw[int(i)] += d * normed;
            db[int(i)] += d;
        });
        sum_over<GROUP>(s, turn);
        turn ^= 1;
        const float c0 = of.quotient(s[0]), c1 = of.quotient(s[1]);
        each_place([&](auto, uint32_t at, f32x8 normed, f32x8, f32x8 g) {
            I::template store<PAST>(a.out + r * a.out_stride * I::kBytes, at, width, I::narrow(now.rstd * (g - c0 - normed * c1)));
        });
    }
    if (column_blocks || (!a.dweight && !a.dbias)) return;
    if constexpr (kPer > 1) {  // the workgroup's groups into one, in their order
        __shared__ f32x8 both[2 * K][GROUP];
        for (uint32_t g = kPer - 1; g > 0; g--) {
            if (threadIdx.x / GROUP == g)
                static_for<K>([&](auto i) {
                    both[2 * i][thread] = dw[int(i)];
                    both[2 * i + 1][thread] = db[int(i)];
                });
            __syncthreads();
            if (threadIdx.x / GROUP == g - 1)
                static_for<K>([&](auto i) {
                    dw[int(i)] += both[2 * i][thread];
                    db[int(i)] += both[2 * i + 1][thread];
                });
            __syncthreads();
        }
        if (threadIdx.x >= GROUP) return;
    }
    uint8_t* const out = reinterpret_cast<uint8_t*>(a.parts + 2ull * blockIdx.x * width);
    places<GROUP, K>(thread, width, [&](auto i, uint32_t at) {
        I::Wide::store(out, at, width, I::Wide::narrow(dw[int(i)]));
        I::Wide::store(out + 4ull * width, at, width, I::Wide::narrow(db[int(i)]));
    });
}

// Columns of dw (blockIdx.y 0) and db (1): the parts of all workgroups.
constexpr uint32_t kJoinRows = 32, kJoinAhead = 8;
template <class I>
__global__ __launch_bounds__(kColumns* kJoinRows) void norm_join_kernel(const NormArgs a, const uint32_t blocks)
{
    __shared__ float part[kJoinRows][kColumns + 1];
    uint8_t* const out = blockIdx.y ? a.dbias : a.dweight;
    const uint32_t width = static_cast<uint32_t>(a.width), c = threadIdx.x % kColumns, k = threadIdx.x / kColumns;
    const uint32_t at = blockIdx.x * kColumns + c;
    if (!out) return;
    float s = 0.f;
    if (at < width)
        for (uint32_t g = k; g < blocks; g += kJoinRows * kJoinAhead) {
            float x[kJoinAhead];
            static_for<kJoinAhead>([&](auto i) {
                const uint32_t row = g + i * kJoinRows;
                x[int(i)] = row < blocks ? as_global(a.parts)[(2ull * row + blockIdx.y) * width + at] : 0.f;
            });
            static_for<kJoinAhead>([&](auto i) { s += x[int(i)]; });
        }
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
    else if (width <= 1024) fn(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (width <= 2048) fn(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (width <= 4096) fn(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (width <= 8192) fn(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    else fn(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

// Workgroups of the backward pass.
uint32_t grad_blocks(uint64_t n_rows, uint64_t width)
{
    uint32_t blocks = 0;
    choose(width, [&](auto group, auto) {
        constexpr uint32_t per = block_of<group>() / group;
        blocks = static_cast<uint32_t>(std::max<uint64_t>(std::min<uint64_t>((n_rows + per - 1) / per, group >= 512 ? kMostWideBlocks : kMostBlocks), 1));
    });
    return blocks;
}

template <class I>
bool past(const NormArgs& a)
{
    return a.n_rows * a.width * I::kBytes >= kPastBytes;
}

template <class I>
hipError_t forward(const NormArgs& a, hipStream_t stream)
{
    choose(a.width, [&](auto group, auto k) {
        constexpr int threads = block_of<group>();
        constexpr uint32_t per = threads / group;
        const uint32_t blocks = static_cast<uint32_t>(std::min<uint64_t>((a.n_rows + per - 1) / per, kForwardBlocks));
        const auto kernel = past<I>(a) ? norm_kernel<I, group, k, true> : norm_kernel<I, group, k, false>;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, stream, a);
    });
    return hipGetLastError();
}

template <class I>
hipError_t backward(const NormArgs& a, hipStream_t stream)
{
    const uint32_t blocks = grad_blocks(a.n_rows, a.width);
    // (not from rows that the launch replaces)
    const bool sums = a.dweight || a.dbias, few = a.n_rows <= kFewRows && a.out != a.x && a.out != a.dy;
    const uint32_t all = static_cast<uint32_t>((a.width + kColumns - 1) / kColumns), column_blocks = sums && few ? all : 0;
    choose(a.width, [&](auto group, auto k) {
        const auto kernel = past<I>(a) ? norm_grad_kernel<I, group, k, true> : norm_grad_kernel<I, group, k, false>;
        hipLaunchKernelGGL(kernel, dim3(blocks + column_blocks), dim3(block_of<group>()), 0, stream, a, column_blocks);
    });
    if (sums && !few) hipLaunchKernelGGL(norm_join_kernel<I>, dim3(all, 2), dim3(kColumns * kJoinRows), 0, stream, a, blocks);
    return hipGetLastError();
}

}  // namespace

uint64_t norm_workspace(uint64_t n_rows, uint64_t width)
{
    return grad_blocks(n_rows, width) * 8ull * width;
}

hipError_t launch_norm(const NormArgs& a, uint32_t dtype, hipStream_t stream)
{
    hipError_t err = hipSuccess;
    if (a.n_rows) with_items(dtype, a.width, [&](auto items) { err = forward<decltype(items)>(a, stream); });
    return err;
}

hipError_t launch_norm_grad(const NormArgs& a, uint32_t dtype, hipStream_t stream)
{
    hipError_t err = hipSuccess;
    with_items(dtype, a.width, [&](auto items) { err = backward<decltype(items)>(a, stream); });
    return err;
}

}  // namespace ffsnap
