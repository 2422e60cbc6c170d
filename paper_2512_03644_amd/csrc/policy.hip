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

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The sum of exp(z - base) over some logits, base the largest of them so far: -inf as long as all are, and the sum is 0;
// or NaN, as ever after a NaN or +inf.  (With a base that is only moved where a logit is far above it, an exponent rounded to 24
// bits takes 7e-8 off the log-probability of a likely token, against 1e-8.)
constexpr float kLog2E = 0x1.715476p+0f, kLog2ELow = 0x1.4ae0bep-26f;  // log2(e) to 48 bits

__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// What rounding the constant to 24 bits takes off would add up over the vocabulary, always to the same side.
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(fmaf(d, kLog2E, d * kLog2ELow)); }
// What a sum against `from` is against `to`: with what the exponent loses in 24 bits, as this is not one error of many.
__device__ __forceinline__ double moved(double sum, float from, float to)
{
    const float d = fmaxf(from - to, -1000.f), t = d * kLog2E, low = fmaf(d, kLog2E, -t) + d * kLog2ELow;
    const float e = __builtin_amdgcn_exp2f(t);
    return from == -INFINITY ? sum : sum * (static_cast<double>(e) * (1.0 + 0.6931471805599453 * static_cast<double>(low)));
}

// 16 bytes of a row as floats.  gradient(), write(): what the softmax is multiplied by, -factor / total, is for 32-bit elements the
// first of two factors; for 16-bit ones its logarithm joins the exponent, rounded to 24 bits and so to 2^-18 of the
// gradient, and its sign goes on to the rounded elements two at a time.
struct Slot32 {
    static constexpr int kItems = 4, kBytes = 4;
    static __device__ __forceinline__ void read(const u32x4 w, float (&z)[4])
    {
        static_for<4>([&](auto k) { z[int(k)] = __uint_as_float(w[int(k)]); });
    }
    static __device__ __forceinline__ float one(const uint8_t* p) { return *as_global(reinterpret_cast<const float*>(p)); }
    static __device__ __forceinline__ void put(uint8_t* p, float v) { *as_global(reinterpret_cast<float*>(p)) = v; }
    static __device__ __forceinline__ void set_factors(float* f, double factor, double total)
    {
        f[0] = static_cast<float>(-factor / total);
        f[1] = 0.f;
    }
    static __device__ __forceinline__ float gradient(float d, float f0) { return f0 * exp_of(d); }
    static __device__ __forceinline__ float signed_by(float g, float) { return g; }
    static __device__ __forceinline__ u32x4 write(const float (&z)[4], float)
    {
        return u32x4{__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3])};
    }
    static __device__ __forceinline__ u32x4 with(u32x4 w, uint32_t i, float v)
    {
        static_for<4>([&](auto k) { w[int(k)] = i == k ? __float_as_uint(v) : w[int(k)]; });
        return w;
    }
};
template <bool BF16>
struct Slot16 {
    static constexpr int kItems = 8, kBytes = 2;
    static __device__ __forceinline__ float low(uint32_t w)
    {
        return BF16 ? __uint_as_float(w << 16) : __half2float(__ushort_as_half(static_cast<unsigned short>(w & 0xFFFFu)));
    }
    static __device__ __forceinline__ float high(uint32_t w)
    {
        return BF16 ? __uint_as_float(w & 0xFFFF0000u) : __half2float(__ushort_as_half(static_cast<unsigned short>(w >> 16)));
    }
    static __device__ __forceinline__ uint32_t pair(float a, float b)
    {
        if (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
        return __half_as_ushort(__float2half_rn(a)) | uint32_t(__half_as_ushort(__float2half_rn(b))) << 16;
    }
    static __device__ __forceinline__ void read(const u32x4 w, float (&z)[8])
    {
        static_for<4>([&](auto k) {
            z[2 * k] = low(w[int(k)]);
            z[2 * k + 1] = high(w[int(k)]);
        });
    }
    static __device__ __forceinline__ float one(const uint8_t* p) { return low(*as_global(reinterpret_cast<const uint16_t*>(p))); }
    static __device__ __forceinline__ void put(uint8_t* p, float v)
    {
        *as_global(reinterpret_cast<uint16_t*>(p)) = static_cast<uint16_t>(pair(v, 0.f));
    }
    static __device__ __forceinline__ void set_factors(float* f, double factor, double total)
    {
        f[0] = static_cast<float>(log2(fabs(factor)) - log2(total));
        f[1] = __uint_as_float(factor > 0 ? 0x80008000u : 0u);
    }
    static __device__ __forceinline__ float gradient(float d, float f0) { return __builtin_amdgcn_exp2f(fmaf(d, kLog2E, f0)); }
    static __device__ __forceinline__ float signed_by(float g, float f1)
    {
        return __uint_as_float(__float_as_uint(g) ^ (__float_as_uint(f1) & 0x80000000u));
    }
    static __device__ __forceinline__ u32x4 write(const float (&z)[8], float f1)
    {
        const uint32_t s = __float_as_uint(f1);
        return u32x4{pair(z[0], z[1]) ^ s, pair(z[2], z[3]) ^ s, pair(z[4], z[5]) ^ s, pair(z[6], z[7]) ^ s};
    }
    static __device__ __forceinline__ u32x4 with(u32x4 w, uint32_t i, float v)
    {
        const uint32_t bits = pair(v, v), half = i % 2 ? 0xFFFF0000u : 0xFFFFu;
        static_for<4>([&](auto k) { w[int(k)] = i / 2 == k ? (w[int(k)] & ~half) | (bits & half) : w[int(k)]; });
        return w;
    }
};
template <uint32_t DTYPE>
struct SlotOf {
    using Type = Slot16<DTYPE == FF_BF16>;
};
template <>
struct SlotOf<FF_F32> {
    using Type = Slot32;
};

template <int N>
__device__ __forceinline__ void add(float& base, double& sum, const float (&z)[N])
{
    float m = z[0];
    static_for<N - 1>([&](auto k) { m = fmaxf(m, z[k + 1]); });
    if (__any(m > base)) {
        if (m > base) {
            sum = moved(sum, base, m);
            base = m;
        }
    }
    const float b = base_of(base);
    float s[N];
    static_for<N>([&](auto k) { s[int(k)] = exp_of(z[int(k)] - b); });
    for (int d = 1; d < N; d *= 2)
        for (int k = 0; k + d < N; k += 2 * d) s[k] += s[k + d];
    sum += static_cast<double>(s[0]);
}

// What hangs on the token's log-probability.  By one wavefront; total: of exp(z - base).
struct Token {
    double old_logp, ref_logp, gain, weight;
    float z;  // the target's logit
};
__device__ __forceinline__ void token(const ff_policy_batch& b, const Token& k, const double base, const double total, const int lane,
                                      double& logp, double& loss, double& kl, bool& clipped, double& factor)
{
    logp = (static_cast<double>(k.z) - base) - log(total);
    const double lo = 1.0 - static_cast<double>(b.clip_low), hi = 1.0 + static_cast<double>(b.clip_high);
    const double r = exp(logp - k.old_logp);
    const double kept = r * k.gain, cut = (r < lo ? lo : r > hi ? hi : r) * k.gain;
    clipped = cut < kept;
    loss = clipped ? -cut : -kept;
    double slope = clipped ? 0.0 : -kept;
    kl = 0.0;
    if (b.ref_logp) {
        const double d = k.ref_logp - logp, e = expm1(d);
        kl = d == INFINITY ? d : e - d;
        if (b.beta > 0.f) {
            loss += static_cast<double>(b.beta) * kl;
            slope -= static_cast<double>(b.beta) * e;
        }
    }
    factor = k.weight * slope * static_cast<double>(b.loss_scale);
}

// One workgroup, one row.  A thread holds K slots of 16 bytes of it in registers (slot i * THREADS + thread); of longer rows what is
// behind is read again for the gradient.
template <uint32_t DTYPE, int THREADS, int K>
__global__ __launch_bounds__(THREADS) void policy_kernel(const ff_policy_batch b, float* __restrict__ logp_out,
                                                         float* __restrict__ loss_out, uint8_t* dlogits, uint64_t grad_stride,
                                                         PolicyPart* __restrict__ parts)
{
    using S = typename SlotOf<DTYPE>::Type;
    constexpr int N = S::kItems, kWaves = THREADS / kWaveSize;
    __shared__ float bases[kWaves];
    __shared__ double sums[kWaves];
    __shared__ float factors[3];
    const uint64_t t = blockIdx.x;
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const uint32_t vocab = static_cast<uint32_t>(b.vocab), slots = vocab / N;
    const uint8_t* const row = static_cast<const uint8_t*>(b.logits) + t * b.row_stride * S::kBytes;
    uint8_t* const out = dlogits + t * grad_stride * S::kBytes;
    const int64_t y = b.targets[t];
    const float w = b.weights[t];
    const bool wanted = w != 0.f, inside = y >= 0 && y < static_cast<int64_t>(vocab);
    const uint32_t rest = slots * N + threadIdx.x;  // elements behind the last whole slot, one to a thread
    const uint32_t wave_first = wave * kWaveSize;   // a wavefront's first slot of a round
    bool empty = true;
    double total = 0;
    float base = 0;
    u32x4 held[K];
    Token k;
    if (wanted && inside) {
        const uint32_t last = slots ? slots - 1 : 0;
        static_for<K>([&](auto i) {
            const uint32_t slot = i * THREADS + threadIdx.x;
            if (i * THREADS + wave_first < slots) held[int(i)] = load16_unaligned<true>(row + 16ull * (slot < slots ? slot : last));
        });
        k.z = S::one(row + y * S::kBytes);
        k.old_logp = b.old_logp[t];
        k.ref_logp = b.ref_logp ? b.ref_logp[t] : 0.f;
        k.gain = b.advantages[t];
        k.weight = w;
        double sum = 0;
        float own = -INFINITY;  // the thread's base
        static_for<K>([&](auto i) {
            if (i * THREADS + wave_first < slots) {
                float z[N];
                S::read(held[int(i)], z);
                if (i * THREADS + wave_first + kWaveSize > slots) {  // the row's last wavefront
                    const bool mine = i * THREADS + threadIdx.x < slots;
                    static_for<N>([&](auto j) { z[int(j)] = mine ? z[int(j)] : -INFINITY; });
                }
                add(own, sum, z);
            }
        });
        for (uint32_t first = K * THREADS + wave_first; first < slots; first += THREADS) {
            const uint32_t slot = first + lane;
            float z[N];
            S::read(load16_unaligned<false>(row + 16ull * (slot < slots ? slot : last)), z);
            static_for<N>([&](auto j) { z[int(j)] = slot < slots ? z[int(j)] : -INFINITY; });
            add(own, sum, z);
        }
        if (wave == 0) {
            float z[1] = {rest < vocab ? S::one(row + uint64_t(rest) * S::kBytes) : -INFINITY};
            add(own, sum, z);
        }
        base = own;
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) base = fmaxf(base, __shfl_xor(base, d));
        sum = moved(sum, own, base);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) {
            bases[wave] = base;
            sums[wave] = sum;
        }
        __syncthreads();
        base = bases[0];
        for (int i = 1; i < kWaves; i++) base = fmaxf(base, bases[i]);
        for (int i = 0; i < kWaves; i++) total += moved(sums[i], bases[i], base);
        empty = base == -INFINITY && total == 0;
        base = base_of(base);
    }
    if (empty) {
        if (threadIdx.x == 0) {
            logp_out[t] = loss_out[t] = 0.f;
            parts[t] = PolicyPart{0, 0, wanted ? kTokenInvalid : 0u, 0u};
        }
        if (dlogits) {
            for (uint32_t i = threadIdx.x; i < slots; i += THREADS) store16_unaligned<true>(out + 16ull * i, u32x4{0, 0, 0, 0});
            if (rest < vocab) S::put(out + uint64_t(rest) * S::kBytes, 0.f);
        }
        return;
    }
    if (wave == 0) {
        double logp, loss, kl, factor;
        bool clipped;
        token(b, k, base, total, lane, logp, loss, kl, clipped, factor);
        if (lane == 0) {
            logp_out[t] = static_cast<float>(logp);
            loss_out[t] = static_cast<float>(loss);
            parts[t] = PolicyPart{k.weight * loss, k.weight * kl, kTokenCounts | (clipped ? kTokenClipped : 0u), 0u};
            S::set_factors(factors, factor, total);
            factors[2] = static_cast<float>(factor * -expm1(logp));
        }
    }
    if (!dlogits) return;
    __syncthreads();
    const float f0 = factors[0], f1 = factors[1], target_grad = factors[2];
    const uint32_t y32 = static_cast<uint32_t>(y);
    auto gradient = [&](const u32x4 in, const uint32_t slot) {
        float z[N];
        S::read(in, z);
        static_for<N>([&](auto j) { z[int(j)] = S::gradient(z[int(j)] - base, f0); });
        u32x4 g = S::write(z, f1);
        if (slot == y32 / N) g = S::with(g, y32 % N, target_grad);
        return g;
    };
    static_for<K>([&](auto i) {
        const uint32_t slot = i * THREADS + threadIdx.x;
        if (i * THREADS + wave_first < slots && slot < slots)
            store16_unaligned<true>(out + 16ull * slot, gradient(held[int(i)], slot));
    });
    for (uint32_t slot = K * THREADS + threadIdx.x; slot < slots; slot += THREADS)
        store16_unaligned<true>(out + 16ull * slot, gradient(load16_unaligned<false>(row + 16ull * slot), slot));
    if (rest < vocab) {
        const float z = S::one(row + uint64_t(rest) * S::kBytes);
        S::put(out + uint64_t(rest) * S::kBytes, rest == y32 ? target_grad : S::signed_by(S::gradient(z - base, f0), f1));
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

using Kernel = void (*)(const ff_policy_batch, float*, float*, uint8_t*, uint64_t, PolicyPart*);
struct Choice {
    Kernel kernel;
    int threads;
};
// By the slots of a row: whole rows in registers up to 16384.
template <uint32_t DTYPE>
Choice choose(uint64_t slots)
{
    if (slots <= 1024) return {policy_kernel<DTYPE, 256, 4>, 256};
    if (slots <= 4096) return {policy_kernel<DTYPE, 512, 8>, 512};
    if (slots <= 8192) return {policy_kernel<DTYPE, 1024, 8>, 1024};
    return {policy_kernel<DTYPE, 1024, 16>, 1024};
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
        const Choice c = b.dtype == FF_F32 ? choose<FF_F32>(b.vocab / 4) : b.dtype == FF_BF16 ? choose<FF_BF16>(b.vocab / 8) : choose<FF_F16>(b.vocab / 8);
        hipLaunchKernelGGL(c.kernel, dim3(static_cast<uint32_t>(b.n_tokens)), dim3(c.threads), 0, stream, b, logp, token_loss,
                           static_cast<uint8_t*>(dlogits), grad_stride, parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(policy_finish_kernel, dim3(1), dim3(kFinishThreads), 0, stream, parts, b.n_tokens, stats);
    return hipGetLastError();
}

}  // namespace ffsnap
