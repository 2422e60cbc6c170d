// Clipped policy loss with a KL term, and its gradient, for gfx950.
//
// One workgroup takes the row of one token.  Every thread keeps the running maximum of its logits and the sum
// of their exponentials against it while they arrive, and holds the logits themselves in registers; the workgroup
// joins those, and what hangs on the token's log-probability alone -- ratio, clipping, KL term, the slope of the loss in it
// -- is a handful of operations in 64 bits of one wavefront.  The gradient is the slope times ([j is the target] -
// softmax), from the logits in registers: they are read once.  What tokens add to the sums goes to memory and is
// joined, always in the same order, by the last workgroups to be done (count_and_finish).
//
// What bounds it: memory, or for few tokens the launch and the chain from a row's load to its store.  A workgroup's loads do not overlap its
// stores, so what counts is how many rows a compute unit has at once (choose).  The arithmetic of a row, two exponentials and some ten
// other operations a logit, would fill half of the longest rows' time by itself.  Rows kept over in a loop of workgroups, the next one's loads
// under way while the gradient is stored, took a third more.  Us, gradient and all, 4096 tokens on 1000 / 4000 / 8000 / 16,000 / 32,000 /
// 64,000 / 128,256 bf16 logits 13.5 / 23.7 / 31.9 / 54.1 / 94.7 / 191 / 371 (all tokens count; a copy of the last one's bytes takes 330), fp16
// 13.2 / 22.9 / 31.7 / 54.7 / 95.0 / 192 / 372, fp32 13.2 / 28.3 / 49.7 / 89.6 / 186 / 370 / 829; 1.05 GB of bf16 logits without gradient 170 (6.2 TB/s).
// Machines differ by 5 %: of figures elsewhere in this file, those that stand beside each other are of one.
#include "policy.hpp"

#include <hip/hip_fp16.h>

#include "fold.h"
#include "xcd_order.h"

namespace ffsnap {

namespace {

constexpr uint64_t kComputeUnits = 256;
constexpr int kPartThreads = 256;  // of a workgroup that takes a part of a row

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// exp in 64 bits: x = n log(2) + r, |r| <= log(2) / 2, and the series of exp(r), whose first term left out is 6e-15.  (With
// coefficients in scalar registers: as constants they are put into vector registers, which the held logits need.)
__device__ const double kSeries[] = {1.0 / 39916800, 1.0 / 3628800, 1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720,
                                     1.0 / 120,      1.0 / 24,      1.0 / 6,      1.0 / 2,     1.0,        1.0,
                                     0x1.71547652b82fep+0, 0x1.62e42fefa39efp-1, 0x1.abc9e3b39803fp-56};  // log2(e), log(2) in two parts
__device__ __forceinline__ double exp64(double x)
{
    const double* series = kSeries;
    asm volatile("" : "+s"(series));  // or they would be constants again
    auto c = [&](int i) { return table_entry(series, i); };
    x = x > 710.0 ? INFINITY : x < -750.0 ? -750.0 : x;  // (neither for a NaN)
    const double n = rint(x * c(12));
    const double r = fma(-n, c(14), fma(-n, c(13), x));
    double p = c(0);
    static_for<11>([&](auto k) { p = fma(p, r, c(k + 1)); });
    return x == INFINITY ? x : ldexp(p, static_cast<int>(n));
}
// log in 64 bits of a sum that is at least about 1: what a logarithm in 32 bits leaves is a few 1e-7.
__device__ __forceinline__ double log64(double x)
{
    const double l = static_cast<double>(logf(static_cast<float>(x)));
    const double e = fma(x, exp64(-l), -1.0);
    return l + (e - 0.5 * e * e);
}

// The running maximum m of some logits, and the sum of their exponentials against it.  m is -inf as long as all are, and the sum
// 0; or NaN, as ever after a NaN or +inf.
//
// A term is 2^(z log2(e) - c), c = m log2(e) in 24 bits, in one rounded operation in front of the exponential: c's rounding is
// the same for all terms, and known.  What log2(e) loses in 24 bits is taken as that of m, which is out by 1.3e-8 (m - z)
// of a term; a thread's own maximum is not far above what counts in its sum: log-probabilities of long rows are out by 1-2e-8.  (log2(e) to 48 bits, (z - m)
// first, is three operations for no better: 5 % slower on long rows.)  Where m is so large that c would be out by
// more than a few, z - m takes the place of z.
struct Running {
    float m = -INFINITY, c = 0.f, b0 = 0.f;
    double sum = 0;
};
constexpr float kLog2E = 0x1.715476p+0f, kLog2ELow = 0x1.4ae0bep-26f;  // log2(e) to 48 bits
constexpr float kLarge = 0x1p28f;

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(fmaf(d, kLog2E, d * kLog2ELow)); }
// exp(x) with what the exponent loses in 24 bits: in a factor of a whole sum this is not one error of many.  (Next to 0, where the sum
// is that of the largest logit, without the rounding of the result either.)
__device__ __forceinline__ double factor_of(double x)
{
    if (fabs(x) < 0x1p-8) return 1.0 + x * (1.0 + x * (1.0 / 2 + x * (1.0 / 6 + x * (1.0 / 24))));
    const double t = fmax(x, -1000.0) * 0x1.71547652b82fep+0;
    const float high = static_cast<float>(t), low = static_cast<float>(t - static_cast<double>(high));
    return static_cast<double>(__builtin_amdgcn_exp2f(high)) * (1.0 + 0x1.62e42fefa39efp-1 * static_cast<double>(low));
}
// The logarithm of what a sum of 1 stands for.
__device__ __forceinline__ double against(const Running& r)
{
    const double above = static_cast<double>(r.m) - static_cast<double>(r.b0);
    return static_cast<double>(r.b0) + 0x1.62e42fefa39efp-1 * (static_cast<double>(r.c) + above * static_cast<double>(kLog2ELow));
}

// What rounding the largest logit's own term has left out of the sum, for one such logit: where one stands out it decides.  (Of 1000 logits with
// a likely target among them, log-probabilities are out by 6e-9 with this, with 64-bit sums of the terms and 64-bit factors of few threads'
// sums; by 4e-8 without.)
__device__ __forceinline__ double left_out(const Running& r)
{
    const float t = fmaf(r.m - r.b0, kLog2E, -r.c);  // c's rounding
    return fabsf(t) < 0x1p-12f ? (1.0 + 0x1.62e42fefa39efp-1 * static_cast<double>(t)) - static_cast<double>(__builtin_amdgcn_exp2f(t)) : 0.0;
}

// FEW: terms are added in 64 bits.
template <bool FEW, int N>
__device__ __forceinline__ void add(Running& r, float (&z)[N])
{
    float m = z[0];
    static_for<N - 1>([&](auto k) { m = fmaxf(m, z[k + 1]); });
    if (__any(m > r.m)) {
        if (m > r.m) {
            const double was = against(r);
            const bool first = r.m == -INFINITY;
            r.m = m;
            r.b0 = fabsf(m) > kLarge ? m : 0.f;
            r.c = (m - r.b0) * kLog2E;
            if (!first) r.sum *= factor_of(was - against(r));
        }
    }
    if (__any(r.b0 != 0.f)) static_for<N>([&](auto k) { z[int(k)] -= r.b0; });
    static_for<N>([&](auto k) { z[int(k)] = __builtin_amdgcn_exp2f(fmaf(z[int(k)], kLog2E, -r.c)); });
    if constexpr (FEW) {
        double s[2] = {r.sum, 0};
        static_for<N>([&](auto k) { s[k % 2] += static_cast<double>(z[int(k)]); });
        r.sum = s[0] + s[1];
    } else {
        for (int d = 1; d < N; d *= 2)
            for (int k = 0; k + d < N; k += 2 * d) z[k] += z[k + d];
        r.sum += static_cast<double>(z[0]);
    }
}

// A wavefront-uniform address, as such: a lane's 32-bit offset is added to it by the access itself.
typedef FF_GLOBAL uint8_t* Bytes;
__device__ __forceinline__ Bytes uniform(const uint8_t* p)
{
    uint64_t a = reinterpret_cast<uint64_t>(p);
    asm volatile("" : "+s"(a));
    return (Bytes)a;
}
template <bool NT>
__device__ __forceinline__ u32x4 load16(Bytes p, uint32_t lane_bytes)
{
    const auto* const q = (const FF_GLOBAL u32x4_a2*)(p + lane_bytes);
    return NT ? __builtin_nontemporal_load(q) : *q;
}
__device__ __forceinline__ void store16(Bytes p, uint32_t lane_bytes, u32x4 w)
{
    __builtin_nontemporal_store(w, (FF_GLOBAL u32x4_a2*)(p + lane_bytes));
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
    static __device__ __forceinline__ float one(Bytes p, uint32_t i) { return ((FF_GLOBAL float*)p)[i]; }
    static __device__ __forceinline__ void put(Bytes p, uint32_t i, float v) { ((FF_GLOBAL float*)p)[i] = v; }
    // A large factor's products with probabilities below 2^-126, or above 2^128 the factor itself, would be lost in 32 bits: there a lower
    // maximum takes its exponent, and what rounding makes of that is in the factor.
    static __device__ __forceinline__ bool set_factors(float* f, double factor, double total, float& m)
    {
        double both = -factor / total;
        if (fabs(both) > 0x1p64 && fabs(both) != INFINITY) {
            int e;
            const double part = 2.0 * frexp(fabs(both), &e);  // 1 to 2
            const double wanted = static_cast<double>(m) - (log64(part) + 0x1.62e42fefa39efp-1 * (e - 1));
            float lower = static_cast<float>(wanted);
            if (static_cast<double>(lower) > wanted) lower = nextafterf(lower, -INFINITY);
            both *= exp64(static_cast<double>(lower) - static_cast<double>(m));
            both = copysign(fmax(fabs(both), 0x1p-126), both);  // (about 1, unless the maximum is beyond 2^20)
            m = lower;
        }
        f[0] = static_cast<float>(both);
        f[1] = 0.f;
        return true;
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
    static __device__ __forceinline__ float one(Bytes p, uint32_t i) { return low(((FF_GLOBAL uint16_t*)p)[i]); }
    static __device__ __forceinline__ void put(Bytes p, uint32_t i, float v)
    {
        ((FF_GLOBAL uint16_t*)p)[i] = static_cast<uint16_t>(pair(v, 0.f));
    }
    // (the maximum as well joins the exponent, unless it is large)
    static __device__ __forceinline__ bool set_factors(float* f, double factor, double total, float& m)
    {
        const bool large = fabsf(m) > 64.f;
        int e = 0;
        const bool over = fabs(factor) > 0x1.fffffep+127 && fabs(factor) != INFINITY;  // (its products with small probabilities are not)
        const double part = over ? frexp(factor, &e) : factor;
        f[0] = log2f(fabsf(static_cast<float>(part))) + static_cast<float>(e) - log2f(static_cast<float>(total));
        if (!large) f[0] = fmaf(-m, kLog2E, f[0]);
        f[1] = __uint_as_float(factor > 0 ? 0x80008000u : 0u);
        return large;
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

// What hangs on a token's log-probability.  By a whole wavefront: three exponentials in three lanes.  total: of exp(z - base) over
// the row, z_y: the target's logit.
struct Token {
    double logp, loss, kl;
    double factor;  // the gradient is factor * ([j is the target] - softmax),
    double target;  // and at the target this
    bool clipped;
};
struct Given {  // of a token, by scalar loads with the row's first
    float weight, gain, old_logp, ref_logp;
};
__device__ __forceinline__ Given given(const ff_policy_batch& b, const uint32_t t)
{
    const float* const ref = b.ref_logp ? b.ref_logp : b.old_logp;  // (a load either way)
    Given g = {table_entry(b.weights, t), table_entry(b.advantages, t), table_entry(b.old_logp, t), table_entry(ref, t)};
    const double* series = kSeries;
    asm volatile("" : "+s"(series));
    const double first = table_entry(series, 0), last = table_entry(series, 14);  // exp64's lines, for later
    asm volatile("" : "+s"(g.weight), "+s"(g.gain), "+s"(g.old_logp), "+s"(g.ref_logp) : "s"(first), "s"(last));
    return g;
}
__device__ __forceinline__ Token token(const ff_policy_batch& b, const Given& given, const float z_y, const float base, const double total,
                                       const int lane)
{
    Token k;
    k.logp = (static_cast<double>(z_y) - static_cast<double>(base)) - log64(total);
    const double gain = given.gain;
    const double lo = 1.0 - static_cast<double>(b.clip_low), hi = 1.0 + static_cast<double>(b.clip_high);
    const double beta = b.beta;
    const double change = k.logp - static_cast<double>(given.old_logp);
    const double d = b.ref_logp ? static_cast<double>(given.ref_logp) - k.logp : 0.0;
    const double all = exp64(lane == 0 ? change : lane == 1 ? d : k.logp);
    const double r = __shfl(all, 0), kept = r * gain, cut = (r < lo ? lo : r > hi ? hi : r) * gain;
    k.clipped = cut < kept;
    k.loss = k.clipped ? -cut : -kept;
    double slope = k.clipped ? 0.0 : -kept;
    // exp(d) - 1 - d, whose beginnings cancel where d is small
    const double e = __shfl(all, 1) - 1.0;
    k.kl = d == INFINITY            ? d
           : fabs(d) < 0x1p-6 ? d * d * (1.0 / 2 + d * (1.0 / 6 + d * (1.0 / 24 + d * (1.0 / 120 + d * (1.0 / 720)))))
                                    : e - d;
    if (beta > 0) {
        k.loss += beta * k.kl;
        slope -= beta * e;
    }
    k.factor = static_cast<double>(given.weight) * slope * static_cast<double>(b.loss_scale);
    k.target = k.factor * (1.0 - __shfl(all, 2));
    return k;
}

// What is known of a part of a row whose parts go to several workgroups.
struct RowPart {
    double total;  // of exp(z - m)
    float m, z_y;  // z_y: the target's logit, in a row's first part
};

struct PolicyArgs {
    ff_policy_batch b;
    float *logp, *token_loss;
    uint8_t* dlogits;
    uint64_t grad_stride;
    PolicyPart* parts;    // what every token adds to the sums
    RowPart* row_parts;   // of split rows
    struct Counters* counters;
    ff_policy_stats* stats;
};

// A token's part on its way to whichever workgroup joins them: past the caches of this one's XCD, and that one's.
__device__ __forceinline__ void send(PolicyPart* to, const PolicyPart& p)
{
    static_assert(sizeof(PolicyPart) == 24, "three words");
    uint64_t w[3];
    __builtin_memcpy(w, &p, sizeof(w));
    static_for<3>([&](auto i) {
        __hip_atomic_store(reinterpret_cast<uint64_t*>(to) + i, w[int(i)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
}
__device__ __forceinline__ PolicyPart receive(const PolicyPart* from)
{
    uint64_t w[3];
    static_for<3>([&](auto i) {
        w[int(i)] = __hip_atomic_load(reinterpret_cast<const uint64_t*>(from) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    PolicyPart p;
    __builtin_memcpy(&p, w, sizeof(w));
    return p;
}

// Sums over tokens.
struct Sums {
    double loss, kl;
    uint32_t counts[3];
    __device__ __forceinline__ void add(const PolicyPart& p)
    {
        loss += p.loss;
        kl += p.kl;
        static_for<3>([&](auto k) { counts[int(k)] += p.what >> k & 1u; });
    }
    __device__ __forceinline__ void add(const Sums& s)
    {
        loss += s.loss;
        kl += s.kl;
        static_for<3>([&](auto k) { counts[int(k)] += s.counts[int(k)]; });
    }
    // of a wavefront's lanes, in all of them
    __device__ __forceinline__ void join()
    {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
            loss += __shfl_xor(loss, d);
            kl += __shfl_xor(kl, d);
            static_for<3>([&](auto k) { counts[int(k)] += __shfl_xor(counts[int(k)], d); });
        }
    }
    __device__ __forceinline__ ff_policy_stats stats() const
    {
        return {static_cast<float>(loss), static_cast<float>(kl), counts[0], counts[1], counts[2]};
    }
};

// Tokens in groups: token t is in group t % kGroups, whose last token adds the group's up, and the last group of all
// adds those; one counter for all of more than kCountedTokens would queue up, 50 ns each.  Whoever is last,
// the sums are in the same order.  (A kernel of one workgroup behind the others instead: 4096 tokens on 1000 / 8000 / 32,000 15.6 / 33.9 / 89.6 us
// where this takes 12.5 / 31.3 / 86.9, 777 on 50,021 without gradient 36.0 and 34.2.)
constexpr uint32_t kCountedTokens = 64, kGroups = 64;
struct Counters {
    struct {
        uint32_t done, unused[15];
    } all, group[kGroups];  // zero before and after
    struct {
        uint64_t loss, kl, counts[3], unused[3];
    } sums[kGroups];
};

__device__ __forceinline__ bool is_last(uint32_t* count, const uint32_t n)
{
    // What this thread has sent has arrived when its stores are done.  (A release fence would
    // write the L2's other lines back as well, the gradient's among them: 64 tokens on 32,000 13.3 us with one.)
    asm volatile("" ::: "memory");
    wait_loads<0>();
    if (__hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 != n) return false;
    __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

// Token t is done, and its part on its way.  By the wavefront that has sent it.
__device__ __forceinline__ void count_and_finish(const PolicyArgs& A, const uint32_t t, const int lane)
{
    const uint32_t n = static_cast<uint32_t>(A.b.n_tokens);
    if (n == 1) return;  // (deliver)
    const bool few = n <= kCountedTokens;
    const uint32_t group = few ? 0 : t % kGroups, step = few ? 1 : kGroups;
    int last = 0;
    if (lane == 0) last = is_last(few ? &A.counters->all.done : &A.counters->group[group].done, (n - group + step - 1) / step);
    if (!__shfl(last, 0)) return;
    asm volatile("" ::: "memory");
    Sums s = {};
    constexpr int kAtOnce = 4;  // on their way
    for (uint64_t i0 = group + uint64_t(lane) * step; i0 < n; i0 += kAtOnce * kWaveSize * step) {
        PolicyPart p[kAtOnce];
        static_for<kAtOnce>([&](auto k) {
            const uint64_t i = i0 + k * kWaveSize * step;
            p[int(k)] = receive(A.parts + (i < n ? i : i0));
        });
        static_for<kAtOnce>([&](auto k) {
            if (i0 + k * kWaveSize * step < n) s.add(p[int(k)]);
        });
    }
    s.join();
    if (!few) {
        last = 0;
        auto& mine = A.counters->sums[group];
        auto put = [&](uint64_t* to, uint64_t v) { __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        if (lane == 0) {
            put(&mine.loss, __builtin_bit_cast(uint64_t, s.loss));
            put(&mine.kl, __builtin_bit_cast(uint64_t, s.kl));
            static_for<3>([&](auto k) { put(&mine.counts[int(k)], s.counts[int(k)]); });
            last = is_last(&A.counters->all.done, kGroups);
        }
        if (!__shfl(last, 0)) return;
        asm volatile("" ::: "memory");
        auto get = [&](const uint64_t* from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        const auto& other = A.counters->sums[lane];
        s.loss = __builtin_bit_cast(double, get(&other.loss));
        s.kl = __builtin_bit_cast(double, get(&other.kl));
        static_for<3>([&](auto k) { s.counts[int(k)] = static_cast<uint32_t>(get(&other.counts[int(k)])); });
        s.join();
    }
    if (lane == 0) *A.stats = s.stats();
}

// What a token adds, from the thread that knows it: to those that join the tokens, or at once, if it is the only one.
__device__ __forceinline__ void deliver(const PolicyArgs& A, const uint32_t t, const PolicyPart& p)
{
    if (A.b.n_tokens != 1) {
        send(A.parts + t, p);
        return;
    }
    Sums s = {};
    s.add(p);
    *A.stats = s.stats();
}

// What a workgroup does with the slots it has: all of a row, the sum of a part of one, or, behind that, the part's gradient.
enum Mode { kWhole, kSumOfPart, kGradOfPart };

// A thread holds L slots of 16 bytes in LDS and K in registers (slot i * THREADS + thread), which is all of a row's or part's unless LONG: what is
// behind them is then read again for the gradient.  WAVES: wavefronts on a SIMD that the registers leave room for.
template <uint32_t DTYPE, int THREADS, int K, int WAVES, bool GRAD, bool LONG, Mode MODE, int L = 0>
__device__ __forceinline__ void policy_row(const PolicyArgs& A, const uint32_t t, const uint32_t part, const uint32_t n_parts)
{
    using S = typename SlotOf<DTYPE>::Type;
    constexpr int N = S::kItems, kWaves = THREADS / kWaveSize;
    constexpr bool kFew = THREADS <= kPartThreads;  // few terms decide: their sums to more than 24 bits
    __shared__ float maxima[kWaves];
    __shared__ double sums[kWaves];
    __shared__ struct {
        float m, f0, f1, target_grad;
        int empty, apart;
    } shared;
    const ff_policy_batch& b = A.b;
    const int lane = threadIdx.x & (kWaveSize - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const uint32_t wave_first = wave * kWaveSize;  // a wavefront's first slot of a round
    const uint32_t vocab = static_cast<uint32_t>(b.vocab), row_slots = vocab / N;
    // the workgroup's slots, and the elements behind a row's last whole slot, one to a thread of its last workgroup
    const uint32_t first_slot = MODE == kWhole ? 0 : part * (THREADS * K);
    const uint32_t slots = MODE == kWhole ? row_slots : row_slots - first_slot < THREADS * K ? row_slots - first_slot : THREADS * K;
    const uint32_t n_rest = MODE == kWhole || part + 1 == n_parts ? vocab - row_slots * N : 0;
    const uint8_t* const row = static_cast<const uint8_t*>(b.logits) + t * b.row_stride * S::kBytes;
    const uint8_t* const in = row + 16ull * first_slot;
    uint8_t* const out = GRAD ? A.dlogits + t * A.grad_stride * S::kBytes + 16ull * first_slot : nullptr;
    const int64_t target = table_entry(b.targets, t);
    const Given have = given(b, t);
    const bool wanted = have.weight != 0.f;
    auto leave_out = [&] {
        if (MODE == kSumOfPart) return;
        if (threadIdx.x == 0 && part == 0) {
            A.logp[t] = A.token_loss[t] = 0.f;
            deliver(A, t, PolicyPart{0, 0, wanted ? kTokenInvalid : 0u, 0u});
        }
        if (!GRAD) return;
        for (uint32_t first = wave_first; first < slots; first += THREADS)
            if (first + lane < slots) store16(uniform(out + 16ull * first), 16 * lane, u32x4{0, 0, 0, 0});
        if (threadIdx.x < n_rest) S::put(uniform(out + 16ull * slots), threadIdx.x, 0.f);
    };
    if (!wanted || target < 0 || target >= static_cast<int64_t>(vocab)) {
        leave_out();
        return;
    }
    // Does the wavefront have slots in round i, and where is a lane's?  Lanes behind the last slot take that one again.
    auto has = [&](auto i) { return i * THREADS + wave_first < slots; };
    auto at = [&](auto i) {
        const uint32_t last = slots - 1 - i * THREADS;
        return threadIdx.x < last ? threadIdx.x : last;
    };
    const uint32_t y = static_cast<uint32_t>(target) - first_slot * N;  // among the workgroup's elements, if it is
    float z_y = 0.f, end = -INFINITY;
    if (wave == 0) {
        if (MODE != kGradOfPart) z_y = S::one(uniform(row), static_cast<uint32_t>(target));
        if (threadIdx.x < n_rest) end = S::one(uniform(in + 16ull * slots), threadIdx.x);
    }
    u32x4 held[K], early[L ? L : 1];
    __shared__ u32x4 in_lds[L ? L * THREADS : 1];
    auto fetch = [&](u32x4& to, auto round) {
        if (has(round)) to = load16<true>(uniform(in + 16ull * THREADS * round), 16 * at(round));
    };
    if (MODE != kGradOfPart || GRAD) {
        static_for<L>([&](auto i) { fetch(early[int(i)], i); });
        static_for<K - L>([&](auto i) { fetch(held[L + i], std::integral_constant<int, 2 * L + i>{}); });
    }
    constexpr int kAhead = L ? 2 : 4;  // slots under way of those that are not held
    if constexpr (MODE != kGradOfPart) {
        Running r;
        // Two slots, of which a wavefront has the first.  (first: of the wavefront's in either)
        auto take = [&](const u32x4 w0, const u32x4 w1, const uint32_t first0, const uint32_t first1) {
            float z[2 * N], x[N];
            S::read(w0, x);
            static_for<N>([&](auto j) { z[int(j)] = x[int(j)]; });
            S::read(w1, x);
            static_for<N>([&](auto j) { z[N + j] = x[int(j)]; });
            if (first1 + kWaveSize > slots) {  // the end
                const bool mine0 = first0 + lane < slots, mine1 = first1 + lane < slots;
                static_for<N>([&](auto j) {
                    z[int(j)] = mine0 ? z[int(j)] : -INFINITY;
                    z[N + j] = mine1 ? z[N + j] : -INFINITY;
                });
            }
            add<kFew>(r, z);
        };
        static_for<L / 2>([&](auto i) {
            if (has(std::integral_constant<int, 2 * i>{}))
                take(early[2 * i], early[2 * i + 1], 2 * i * THREADS + wave_first, (2 * i + 1) * THREADS + wave_first);
            in_lds[2 * i * THREADS + threadIdx.x] = early[2 * i];
            in_lds[(2 * i + 1) * THREADS + threadIdx.x] = early[2 * i + 1];
            fetch(held[2 * i], std::integral_constant<int, L + 2 * i>{});
            fetch(held[2 * i + 1], std::integral_constant<int, L + 2 * i + 1>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        static_for<K / 2>([&](auto i) {
            constexpr int h = (2 * i + L) % K;  // those that were asked for first
            if (has(std::integral_constant<int, L + h>{}))
                take(held[h], held[h + 1], (L + h) * THREADS + wave_first, (L + h + 1) * THREADS + wave_first);
            if constexpr (L) __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (LONG)
            for (uint32_t first = (L + K) * THREADS + wave_first; first < slots; first += kAhead * THREADS) {
                u32x4 w[kAhead];
                static_for<kAhead>([&](auto i) {
                    const uint32_t f = first + i * THREADS;
                    if (f < slots) w[int(i)] = load16<false>(uniform(in + 16ull * f), 16 * (f + lane < slots ? lane : 0));
                });
                static_for<kAhead / 2>([&](auto i) {
                    const uint32_t f = first + 2 * i * THREADS;
                    if (f < slots) take(w[2 * i], w[2 * i + 1], f, f + THREADS);
                });
            }
        if (wave == 0) {
            float z[1] = {end};
            add<kFew>(r, z);
        }
        float m = r.m;
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
        double sum = r.sum;
        const double by = against(r) - static_cast<double>(m);
        if (r.m != -INFINITY) sum = (sum + left_out(r)) * (kFew ? exp64(by) : factor_of(by));
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) {
            maxima[wave] = m;
            sums[wave] = sum;
        }
        __syncthreads();
    }
    if (wave == 0) {
        // the sums of the workgroup's wavefronts, or of the row's parts, in a lane each
        float from = -INFINITY;
        double total = 0;
        if (MODE == kGradOfPart) {
            const RowPart* const p = A.row_parts + t * n_parts;
            if (lane < static_cast<int>(n_parts)) {
                from = p[lane].m;
                total = p[lane].total;
            }
            z_y = p->z_y;
        } else {
            from = maxima[lane % kWaves];
            total = lane < kWaves ? sums[lane] : 0.0;
        }
        float m = from;
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
        if (from != -INFINITY) total *= exp64(static_cast<double>(from) - static_cast<double>(m));
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) total += __shfl_xor(total, d);
        if (MODE == kSumOfPart) {
            if (lane == 0) A.row_parts[t * n_parts + part] = RowPart{total, m, z_y};
        } else {
            const bool empty = m == -INFINITY && total == 0;
            if (m == -INFINITY) m = 0.f;
            const Token k = token(b, have, z_y, m, total, lane);
            if (lane == 0) {
                if (!empty && part == 0) {
                    const double w = have.weight;
                    A.logp[t] = static_cast<float>(k.logp);
                    A.token_loss[t] = static_cast<float>(k.loss);
                    deliver(A, t, PolicyPart{w * k.loss, w * k.kl, kTokenCounts | (k.clipped ? kTokenClipped : 0u), 0u});
                }
                float f[2];
                const bool apart = S::set_factors(f, k.factor, total, m);
                shared = {m, f[0], f[1], static_cast<float>(k.target), empty, apart};
            }
        }
    }
    if (MODE == kSumOfPart) return;
    __syncthreads();
    if (shared.empty) {
        leave_out();
        return;
    }
    if constexpr (GRAD) {
        const float m = shared.m, f0 = shared.f0, f1 = shared.f1, target_grad = shared.target_grad;
        const bool apart = __builtin_amdgcn_readfirstlane(shared.apart) != 0;
        auto gradient = [&](const u32x4 w, const bool has_target) {
            float z[N];
            S::read(w, z);
            if (apart) static_for<N>([&](auto j) { z[int(j)] -= m; });
            static_for<N>([&](auto j) { z[int(j)] = S::gradient(z[int(j)], f0); });
            u32x4 g = S::write(z, f1);
            if (has_target) g = S::with(g, y % N, target_grad);
            return g;
        };
        auto put_round = [&](const u32x4 w, auto i) {
            const uint32_t mine = at(i);
            store16(uniform(out + 16ull * THREADS * i), 16 * mine, gradient(w, y / N - i * THREADS == mine));
        };
        static_for<L>([&](auto i) {
            if (has(i)) put_round(in_lds[i * THREADS + threadIdx.x], i);
        });
        static_for<K>([&](auto i) {
            constexpr std::integral_constant<int, L + i> round;
            if (has(round)) put_round(held[int(i)], round);
        });
        if constexpr (LONG)
            for (uint32_t first = (L + K) * THREADS + wave_first; first < slots; first += kAhead * THREADS) {
                u32x4 w[kAhead];
                static_for<kAhead>([&](auto i) {
                    const uint32_t f = first + i * THREADS;
                    if (f + lane < slots) w[int(i)] = load16<false>(uniform(in + 16ull * f), 16 * lane);
                });
                static_for<kAhead>([&](auto i) {
                    const uint32_t f = first + i * THREADS;
                    if (f + lane < slots) store16(uniform(out + 16ull * f), 16 * lane, gradient(w[int(i)], f + lane == y / N));
                });
            }
        if (threadIdx.x < n_rest) {
            const float z = S::one(uniform(in + 16ull * slots), threadIdx.x);
            S::put(uniform(out + 16ull * slots), threadIdx.x,
                   slots * N + threadIdx.x == y ? target_grad : S::signed_by(S::gradient(apart ? z - m : z, f0), f1));
        }
    }
}

// Rows that follow each other go to one XCD, four at a time (xcd_order.h), unless they are among the longest.  us, 4096 rows of 4000 / 8000 /
// 16,000 / 32,000 / 64,000 / 128,256 bf16 logits in launch order 22.4 / 31.3 / 54.4 / 97.0 / 194 / 382, by two 22.5 / 31.4 / 52.9 / 94.8 / 191 / 385, by
// eight 22.4 / 31.1 / 52.8 / 94.8 / 192 / 386, by 64 - / 31.6 / 53.5 / 95.0 / 195 / 388 (the last with a tenth masked).  Plain loads and stores instead of
// non-temporal ones: stores 3-6 % slower; loads 2-3 % slower from 128 MB of logits on, and below 80 MB 10 % faster if the same logits are read
// again and again, but 4-10 us slower where they are not in the caches.
constexpr uint32_t kXcdRows = 4;
template <uint32_t DTYPE, int THREADS, int K, int WAVES, bool GRAD, bool LONG, int L = 0>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(WAVES))) void policy_kernel(const PolicyArgs A, const uint32_t first)
{
    const uint32_t t = first + xcd_order(blockIdx.x, gridDim.x, THREADS * (K + L) <= 8192 ? kXcdRows : 0);
    policy_row<DTYPE, THREADS, K, WAVES, GRAD, LONG, kWhole, L>(A, t, 0, 1);
    if (threadIdx.x < kWaveSize) count_and_finish(A, t, threadIdx.x);
}

// So many rows of more than 4096 slots are split into parts of 1024: the parts' sums in one launch, and in another, once more for
// each of them, what is left of policy_kernel, on logits that are in the caches.  Whole / split, us: 1 / 4 / 16 / 32 / 60 / 100 rows of
// 128,256 bf16 logits 21.6 / 22.0 / 22.8 / 22.5 / 22.5 / 25 and 10.8 / 11.1 / 12.0 / 12.9 / 15.3 / 22.4, 200 28.6 and 37.8; 16 / 64 / 120 rows of
// 50,000 13.8 / 13.8 / 15.1 and 11.2 / 12.5 / 16.7; 16 / 64 / 128 of 130,000 fp32 ones 29.8 / 31.2 / 41.2 and 12.0 / 21.4 / 43.0.  Without a gradient 100 / 300 / 777 / 2000 rows of 50,021 fp32 ones
// 12.9 / 20.4 / 34.2 / 70.6 and 13.9 / 19.9 / 33.4 / 75, of 128,256 21.0 / 43.5 / 82 / 176 and 18.1 / 32.7 / 74 / 176, bf16 777 / 2000 47 / 90 and 48 / 111.
constexpr int kPartSlots = 4 * kPartThreads;
constexpr uint32_t kSplitFrom = 4096, kSplitRows = 64, kMostParts = 64;
template <uint32_t DTYPE>
__global__ __launch_bounds__(kPartThreads) void policy_sum_kernel(const PolicyArgs A, const uint32_t n_parts)
{
    policy_row<DTYPE, kPartThreads, 4, 4, false, false, kSumOfPart>(A, blockIdx.x / n_parts, blockIdx.x % n_parts, n_parts);
}
template <uint32_t DTYPE, bool GRAD>
__global__ __launch_bounds__(kPartThreads) void policy_grad_kernel(const PolicyArgs A, const uint32_t n_parts)
{
    const uint32_t per = GRAD ? n_parts : 1, part = blockIdx.x % per;
    policy_row<DTYPE, kPartThreads, 4, 4, GRAD, false, kGradOfPart>(A, blockIdx.x / per, part, n_parts);
    if (part == 0 && threadIdx.x < kWaveSize) count_and_finish(A, blockIdx.x / per, threadIdx.x);
}

__global__ void policy_of_nothing_kernel(ff_policy_stats* stats) { *stats = {}; }

struct Choice {
    void (*kernel)(const PolicyArgs, uint32_t first);
    int threads;
};
// By the slots of a row and the number of rows, so that as many rows as possible are on a compute unit at once, and are held there whole.
// Threads hold four slots each in registers where that leaves room for 2048 on a compute unit, sixteen where two rows of 1024 threads no
// longer fit.  LDS holds more of them:
// - Rows of 2049-4096 slots: four on a unit, half of each in LDS (512 threads), or two, in registers (1024).  Many short rounds beat few
//   long ones where the rows then end in one round, or are far from 4096 slots.  us, four / two, 600 / 1000 / 1500 / 2000 / 3000 bf16 rows of
//   20,000 16.3 / 20.4 / 29.6 / 37.0 / 51.0 and 18.1 / 23.6 / 31.3 / 38.8 / 53.2, of 24,000 16.8 / 21.5 / 32.0 / 40.5 / 56.9 and 19.8 / 26.3 /
//   35.2 / 43.3 / 60.0, of 28,000 20.0 / 25.0 / 38.1 / 48.8 / 69.9 and 21.4 / 29.0 / 38.8 / 48.7 / 68.0, of 32,000 21.3 / 26.0 / 42.1 / 52.2 /
//   75.2 and 22.1 / 30.6 / 42.0 / 53.0 / 74.6; 4096 of 32,000 99.7 and 97.4, a quarter of them masked 93.0 and 87.3.
// - Rows of 8193-20,480: two on a unit, one's loads under the other's stores, 20 slots of a thread in registers and 8 in LDS (14,336 in all;
//   what is behind them is read again), or one, 16 of its 1024 threads each.  us, two / one, 4096 rows of 80,000 / 100,000 / 128,256 bf16 logits
//   244 / 322 / 393 and 281 / 352 / 427, 300 / 500 / 1000 of 128,256 41.7 / 47.7 / 97.0 and 47.8 / 57.7 / 113, 2000 of 147,000 / 164,000 /
//   180,000 256 / 280 / 315 and 271 / 280 / 313, of 50,000 / 65,000 fp32 ones 159 / 216 and 167 / 227, 1024 of 130,000 301 and 245.
//   (18 slots in registers 399 where 20 take 393, with no LDS 436; 22 need scratch memory; what is read again four rounds at a time instead of
//   two, or in front of what is held, 395 and 396.)
// Three rows of 4097-8192 slots on a unit, 10 slots of a thread in registers and 6 in LDS (some scratch memory): 600 / 777 / 2000 / 4096 rows of
// 50,000 30.7 / 40.7 / 82.7 / 162 where two take 34.8 / 42.2 / 86 / 164, of 64,000 34.8 / 49.0 / 103 / 198 and 39.9 / 49.0 / 100 / 193; 1000 fp32
// rows of 32,000 58 and 50: not kept.
// Other splits, us: 4096 rows of 2000 slots by 256 / 512 / 1024 threads 63 / 56 / 60; of 8000 by 512 threads with 16, by 1024 with 8, with 4 of 8
// slots held 195 / 222 / 217; 1024 fp32 rows of 32,500 by 1024 threads with 16 / 8 / 4 held 247 / 281 / 278.  Few rows take 1024 threads where
// many would take 512.  Without a gradient nothing is held, and four slots are on their way.
// As a row is one workgroup's, 65 / 100 / 150 / 200 / 300 rows fill part of the chip, or two rows some units: of 32,000 bf16 logits 11.5 / 11.9 / 12.0 /
// 12.5 / 15.5 us, of 50,021 16.6 / 16.9 / 17.2 / 17.2 / 24.7, of 128,256 22.5 / 23.1 / 23.5 / 26.8 / 40.6 (fp16 within 3 %; fp32 31 / 35 / 39 / 47 / 82,
// half of a row read twice); without a gradient, of 128,256, 16.8 / 16.8 / 17.2 / 18.0 / 26.9.
template <uint32_t DTYPE>
Choice choose(uint64_t slots, uint64_t rows, bool grad)
{
    const bool many = rows > kComputeUnits;
    if (slots <= 256) return {grad ? policy_kernel<DTYPE, 64, 4, 8, true, false> : policy_kernel<DTYPE, 64, 4, 8, false, false>, 64};
    if (slots <= 1024) return {grad ? policy_kernel<DTYPE, 256, 4, 8, true, false> : policy_kernel<DTYPE, 256, 4, 8, false, false>, 256};
    if (slots <= 2048 && many) return {grad ? policy_kernel<DTYPE, 512, 4, 8, true, false> : policy_kernel<DTYPE, 512, 4, 8, false, true>, 512};
    if (slots <= 4096 && grad && rows > 2 * kComputeUnits && (rows <= 4 * kComputeUnits || slots <= 3072))
        return {policy_kernel<DTYPE, 512, 4, 8, true, false, 4>, 512};
    if (slots <= 4096) return {grad ? policy_kernel<DTYPE, 1024, 4, 8, true, false> : policy_kernel<DTYPE, 1024, 4, 8, false, true>, 1024};
    if (slots <= 8192 && many) return {grad ? policy_kernel<DTYPE, 512, 16, 4, true, false> : policy_kernel<DTYPE, 512, 4, 8, false, true>, 512};
    if (slots <= 20480 && many && grad) return {policy_kernel<DTYPE, 512, 20, 4, true, true, 8>, 512};
    return {grad ? policy_kernel<DTYPE, 1024, 16, 4, true, true> : policy_kernel<DTYPE, 1024, 4, 8, false, true>, 1024};
}

template <uint32_t DTYPE>
hipError_t launch(const PolicyArgs& A, hipStream_t stream)
{
    const uint32_t rows = static_cast<uint32_t>(A.b.n_tokens);
    const uint64_t slots = A.b.vocab / SlotOf<DTYPE>::Type::kItems;
    const uint64_t n_parts = (slots + kPartSlots - 1) / kPartSlots;
    const bool grad = A.dlogits != nullptr;
    if (slots > kSplitFrom && n_parts <= kMostParts && rows <= kSplitRows) {
        const uint32_t parts = static_cast<uint32_t>(n_parts);
        hipLaunchKernelGGL(policy_sum_kernel<DTYPE>, dim3(rows * parts), dim3(kPartThreads), 0, stream, A, parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (grad)
            hipLaunchKernelGGL((policy_grad_kernel<DTYPE, true>), dim3(rows * parts), dim3(kPartThreads), 0, stream, A, parts);
        else
            hipLaunchKernelGGL((policy_grad_kernel<DTYPE, false>), dim3(rows), dim3(kPartThreads), 0, stream, A, parts);
        return hipGetLastError();
    }
    const Choice c = choose<DTYPE>(slots, rows, grad);
    // in one launch, up to 4 million rows and more; tokens are counted over all
    const uint32_t most = most_groups(c.threads);
    for (uint64_t first = 0; first < rows; first += most) {
        const uint32_t left = rows - static_cast<uint32_t>(first);
        hipLaunchKernelGGL(c.kernel, dim3(left < most ? left : most), dim3(c.threads), 0, stream, A, static_cast<uint32_t>(first));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// The workspace: the counters; what tokens add to the sums; the parts of split rows.
uint64_t parts_bytes(uint64_t n_tokens) { return (n_tokens * sizeof(PolicyPart) + 15) / 16 * 16; }

}  // namespace

// (With room for the parts of split rows however many tokens there are: a workspace serves smaller calls as well.)
uint64_t policy_workspace(uint64_t n_tokens, uint64_t vocab)
{
    const uint64_t rows = n_tokens < kSplitRows ? n_tokens : kSplitRows;
    const uint64_t most = vocab / (4 * kPartSlots) + 1;  // of 32-bit logits
    return sizeof(Counters) + parts_bytes(n_tokens) + rows * (most < kMostParts ? most : kMostParts) * sizeof(RowPart);
}

hipError_t launch_policy(const ff_policy_batch& b, float* logp, float* token_loss, void* dlogits, uint64_t grad_stride,
                         ff_policy_stats* stats, void* workspace, hipStream_t stream)
{
    uint8_t* const w = static_cast<uint8_t*>(workspace);
    const PolicyArgs A = {b,
                          logp,
                          token_loss,
                          static_cast<uint8_t*>(dlogits),
                          grad_stride,
                          reinterpret_cast<PolicyPart*>(w + sizeof(Counters)),
                          reinterpret_cast<RowPart*>(w + sizeof(Counters) + parts_bytes(b.n_tokens)),
                          reinterpret_cast<Counters*>(w),
                          stats};
    if (b.n_tokens)
        return b.dtype == FF_F32 ? launch<FF_F32>(A, stream) : b.dtype == FF_BF16 ? launch<FF_BF16>(A, stream) : launch<FF_F16>(A, stream);
    hipLaunchKernelGGL(policy_of_nothing_kernel, dim3(1), dim3(1), 0, stream, stats);
    return hipGetLastError();
}

}  // namespace ffsnap
