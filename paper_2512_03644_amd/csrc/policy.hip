// Clipped policy loss with a KL term, and its gradient, for gfx950.
//
// One workgroup takes the row of one token.  Every thread keeps the running maximum of its logits and the sum
// of their exponentials against it; the workgroup joins those, and what hangs on the token's log-probability
// alone -- ratio, clipping, KL term, the slope of the loss in it -- is a handful of operations in 64 bits.  The
// gradient is the slope times ([j is the target] - softmax), from the row read a second time.  What
// tokens add to the sums goes to memory and is joined by a last workgroup in the tokens' order.
#include "policy.hpp"

#include <hip/hip_fp16.h>

#include "fold.h"

namespace ffsnap {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWaveSize;
constexpr float kLog2E = 1.44269504088896340736f;

__device__ __forceinline__ float f16_to_f32(uint32_t bits) { return __half2float(__ushort_as_half(static_cast<unsigned short>(bits))); }

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 16 bytes of a row: kItem elements as floats, and back, rounded to nearest even.
template <uint32_t DTYPE>
struct Slot;
template <>
struct Slot<FF_F32> {
    static constexpr int kItems = 4, kBytes = 4;
    static __device__ __forceinline__ void read(const u32x4 w, float (&z)[4])
    {
        static_for<4>([&](auto k) { z[int(k)] = __uint_as_float(w[int(k)]); });
    }
    static __device__ __forceinline__ u32x4 write(const float (&z)[4])
    {
        return u32x4{__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3])};
    }
    static __device__ __forceinline__ float one(const uint8_t* p) { return *as_global(reinterpret_cast<const float*>(p)); }
    static __device__ __forceinline__ void put(uint8_t* p, float v) { *as_global(reinterpret_cast<float*>(p)) = v; }
};
template <>
struct Slot<FF_BF16> {
    static constexpr int kItems = 8, kBytes = 2;
    static __device__ __forceinline__ void read(const u32x4 w, float (&z)[8])
    {
        static_for<4>([&](auto k) {
            z[2 * k] = __uint_as_float(w[int(k)] << 16);
            z[2 * k + 1] = __uint_as_float(w[int(k)] & 0xFFFF0000u);
        });
    }
    static __device__ __forceinline__ uint32_t pair(float a, float b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    }
    static __device__ __forceinline__ u32x4 write(const float (&z)[8])
    {
        return u32x4{pair(z[0], z[1]), pair(z[2], z[3]), pair(z[4], z[5]), pair(z[6], z[7])};
    }
    static __device__ __forceinline__ float one(const uint8_t* p)
    {
        return __uint_as_float(uint32_t(*as_global(reinterpret_cast<const uint16_t*>(p))) << 16);
    }
    static __device__ __forceinline__ void put(uint8_t* p, float v)
    {
        *as_global(reinterpret_cast<uint16_t*>(p)) = static_cast<uint16_t>(pair(v, 0.f));
    }
};
template <>
struct Slot<FF_F16> {
    static constexpr int kItems = 8, kBytes = 2;
    static __device__ __forceinline__ void read(const u32x4 w, float (&z)[8])
    {
        static_for<4>([&](auto k) {
            z[2 * k] = f16_to_f32(w[int(k)] & 0xFFFFu);
            z[2 * k + 1] = f16_to_f32(w[int(k)] >> 16);
        });
    }
    static __device__ __forceinline__ uint32_t pair(float a, float b)
    {
        return __half_as_ushort(__float2half_rn(a)) | uint32_t(__half_as_ushort(__float2half_rn(b))) << 16;
    }
    static __device__ __forceinline__ u32x4 write(const float (&z)[8])
    {
        return u32x4{pair(z[0], z[1]), pair(z[2], z[3]), pair(z[4], z[5]), pair(z[6], z[7])};
    }
    static __device__ __forceinline__ float one(const uint8_t* p)
    {
        return f16_to_f32(*as_global(reinterpret_cast<const uint16_t*>(p)));
    }
    static __device__ __forceinline__ void put(uint8_t* p, float v)
    {
        *as_global(reinterpret_cast<uint16_t*>(p)) = static_cast<uint16_t>(pair(v, 0.f));
    }
};

// The largest of some logits, and the sum of exp(z - base(m)) over them.  Logits of -inf add nothing, and a row
// of nothing else is left with m = -inf and s = 0; a NaN, which the maximum passes over, or +inf makes s NaN.
struct Running {
    float m, s;
};
__device__ __forceinline__ float base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float exp_from(float z, float b) { return __builtin_amdgcn_exp2f((z - b) * kLog2E); }
__device__ __forceinline__ Running join(const Running x, const Running y)
{
    const float m = fmaxf(x.m, y.m), b = base(m);
    return {m, x.s * exp_from(x.m, b) + y.s * exp_from(y.m, b)};
}
template <int N>
__device__ __forceinline__ void add(Running& r, const float (&z)[N])
{
    float m = r.m;
    static_for<N>([&](auto k) { m = fmaxf(m, z[int(k)]); });
    const float b = base(m);
    float s = r.s * exp_from(r.m, b);
    static_for<N>([&](auto k) { s += exp_from(z[int(k)], b); });
    r = {m, s};
}

// What hangs on the token's log-probability.  By one thread.
__device__ void token(const ff_policy_batch& b, const uint64_t t, const float m, const double total, const float z_y,
                      float* logp_out, float* loss_out, PolicyPart* part, float& share, float& target_grad)
{
    const double logp = (static_cast<double>(z_y) - static_cast<double>(m)) - log(total);
    const double w = b.weights[t], gain = b.advantages[t];
    const double r = exp(logp - static_cast<double>(b.old_logp[t]));
    const double lo = 1.0 - static_cast<double>(b.clip_low), hi = 1.0 + static_cast<double>(b.clip_high);
    const double kept = r * gain, cut = (r < lo ? lo : r > hi ? hi : r) * gain;
    const bool clipped = cut < kept;
    double loss = clipped ? -cut : -kept, slope = clipped ? 0.0 : -kept, kl = 0.0;
    if (b.ref_logp) {
        const double d = static_cast<double>(b.ref_logp[t]) - logp, e = expm1(d);
        kl = d == INFINITY ? d : e - d;
        if (b.beta > 0.f) {
            loss += static_cast<double>(b.beta) * kl;
            slope -= static_cast<double>(b.beta) * e;
        }
    }
    logp_out[t] = static_cast<float>(logp);
    loss_out[t] = static_cast<float>(loss);
    part[t] = PolicyPart{w * loss, w * kl, kTokenCounts | (clipped ? kTokenClipped : 0u), 0u};
    const double c = w * slope * static_cast<double>(b.loss_scale);
    share = static_cast<float>(-c / total);
    target_grad = static_cast<float>(c * -expm1(logp));
}

template <uint32_t DTYPE>
__global__ __launch_bounds__(kThreads) void policy_kernel(const ff_policy_batch b, float* __restrict__ logp,
                                                          float* __restrict__ token_loss, uint8_t* dlogits, uint64_t grad_stride,
                                                          PolicyPart* __restrict__ parts)
{
    using S = Slot<DTYPE>;
    constexpr int N = S::kItems;
    __shared__ Running joined[kWaves];
    __shared__ float factors[2];
    const uint64_t t = blockIdx.x;
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x / kWaveSize;
    const uint32_t vocab = static_cast<uint32_t>(b.vocab), slots = vocab / N;
    const uint8_t* const row = static_cast<const uint8_t*>(b.logits) + t * b.row_stride * S::kBytes;
    uint8_t* const out = dlogits + t * grad_stride * S::kBytes;
    const int64_t y = b.targets[t];
    const bool wanted = b.weights[t] != 0.f, inside = y >= 0 && y < static_cast<int64_t>(vocab);
    const uint32_t rest = slots * N + threadIdx.x;  // elements behind the last whole slot, one to a thread
    Running r = {-INFINITY, 0.f};
    if (wanted && inside) {
        for (uint32_t k = threadIdx.x; k < slots; k += kThreads) {
            float z[N];
            S::read(load16_unaligned<false>(row + 16ull * k), z);
            add(r, z);
        }
        if (rest < vocab) {
            const float z[1] = {S::one(row + uint64_t(rest) * S::kBytes)};
            add(r, z);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) r = join(r, Running{__shfl_xor(r.m, d), __shfl_xor(r.s, d)});
        if (lane == 0) joined[wave] = r;
        __syncthreads();
        r = joined[0];
        for (int w = 1; w < kWaves; w++) r = join(r, joined[w]);
    }
    if (!wanted || !inside || (r.m == -INFINITY && r.s == 0.f)) {
        if (threadIdx.x == 0) {
            logp[t] = token_loss[t] = 0.f;
            parts[t] = PolicyPart{0, 0, wanted ? kTokenInvalid : 0u, 0u};
        }
        if (dlogits) {
            for (uint32_t k = threadIdx.x; k < slots; k += kThreads) store16_unaligned<false>(out + 16ull * k, u32x4{0, 0, 0, 0});
            if (rest < vocab) S::put(out + uint64_t(rest) * S::kBytes, 0.f);
        }
        return;
    }
    if (threadIdx.x == 0) {
        float share, target_grad;
        token(b, t, r.m, r.s, S::one(row + y * S::kBytes), logp, token_loss, parts, share, target_grad);
        factors[0] = share;
        factors[1] = target_grad;
    }
    if (!dlogits) return;
    __syncthreads();
    const float share = factors[0], target_grad = factors[1], from = base(r.m);
    for (uint32_t k = threadIdx.x; k < slots; k += kThreads) {
        float z[N];
        S::read(load16_unaligned<false>(row + 16ull * k), z);
        static_for<N>([&](auto i) {
            z[int(i)] = share * exp_from(z[int(i)], from);
            if (N * k + i == static_cast<uint32_t>(y)) z[int(i)] = target_grad;
        });
        store16_unaligned<false>(out + 16ull * k, S::write(z));
    }
    if (rest < vocab) {
        const float z = S::one(row + uint64_t(rest) * S::kBytes);
        S::put(out + uint64_t(rest) * S::kBytes, rest == static_cast<uint32_t>(y) ? target_grad : share * exp_from(z, from));
    }
}

constexpr int kFinishThreads = 256;
__global__ __launch_bounds__(kFinishThreads) void policy_finish_kernel(const PolicyPart* __restrict__ parts, uint64_t n,
                                                                       ff_policy_stats* __restrict__ stats)
{
    double sums[2] = {0, 0};
    unsigned long long counts[3] = {0, 0, 0};
    for (uint64_t i = threadIdx.x; i < n; i += kFinishThreads) {
        sums[0] += parts[i].loss;
        sums[1] += parts[i].kl;
        static_for<3>([&](auto k) { counts[int(k)] += parts[i].what >> k & 1u; });
    }
    __shared__ double all_sums[2][kFinishThreads / kWaveSize];
    __shared__ unsigned long long all_counts[3][kFinishThreads / kWaveSize];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        static_for<2>([&](auto k) { sums[int(k)] += __shfl_xor(sums[int(k)], d); });
        static_for<3>([&](auto k) { counts[int(k)] += __shfl_xor(counts[int(k)], d); });
    }
    const int wave = threadIdx.x / kWaveSize;
    if (threadIdx.x % kWaveSize == 0) {
        static_for<2>([&](auto k) { all_sums[int(k)][wave] = sums[int(k)]; });
        static_for<3>([&](auto k) { all_counts[int(k)][wave] = counts[int(k)]; });
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kFinishThreads / kWaveSize; w++) {
        static_for<2>([&](auto k) { sums[int(k)] += all_sums[int(k)][w]; });
        static_for<3>([&](auto k) { counts[int(k)] += all_counts[int(k)][w]; });
    }
    *stats = ff_policy_stats{static_cast<float>(sums[0]), static_cast<float>(sums[1]), counts[0], counts[1], counts[2]};
}

}  // namespace

uint64_t policy_workspace(uint64_t n_tokens, uint64_t)
{
    return n_tokens * sizeof(PolicyPart);
}

hipError_t launch_policy(const ff_policy_batch& b, float* logp, float* token_loss, void* dlogits, uint64_t grad_stride,
                         ff_policy_stats* stats, void* workspace, hipStream_t stream)
{
    PolicyPart* const parts = static_cast<PolicyPart*>(workspace);
    if (b.n_tokens) {
        const auto kernel = b.dtype == FF_F32 ? policy_kernel<FF_F32> : b.dtype == FF_BF16 ? policy_kernel<FF_BF16> : policy_kernel<FF_F16>;
        hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(b.n_tokens)), dim3(kThreads), 0, stream, b, logp, token_loss,
                           static_cast<uint8_t*>(dlogits), grad_stride, parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(policy_finish_kernel, dim3(1), dim3(kFinishThreads), 0, stream, parts, b.n_tokens, stats);
    return hipGetLastError();
}

}  // namespace ffsnap
