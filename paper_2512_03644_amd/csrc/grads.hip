// Gradient norm and clipping for gfx950.
//
// The norm is one pass over all gradients, which bounds it: 6.8 and 7.0 TB/s on 1.7 and 3.2 GB (247 and 461 us; the pass of a restore that only
// reads reaches 7.0 on 12 GB).  A wavefront takes items of 8 KiB of one tensor (grads.hpp), lane l of a row of 1 KiB taking 16 bytes.
// Every element is squared and summed in 64 bits: squares of 16- and 32-bit floats are exact there and cannot overflow, so
// no finite gradient needs a second look.  An item's sum that is not finite tells that the item holds an infinity or NaN; only then are
// those counted.  Sums go from lanes to the wavefront to the workgroup to memory in an order that depends on the list alone,
// and the last workgroup to be done joins them: the same bits every time.  Short lists are bound by the launch and that chain (64
// tensors, 4 MB: 5.3 us; 8.4 where a second kernel joined the parts).
// An item's rows asked for while the one before is added up take 1-5 % longer, 1024 workgroups 2 % (10,000 tensors in 20 MB: 10 % less).
//
// Clipping reads and writes every gradient once.
#include "grads.hpp"

#include <hip/hip_fp16.h>

#include "fold.h"
#include "xcd_order.h"

namespace ffsnap {

namespace {

constexpr int kThreads = kGradWaves * kWaveSize;
constexpr int kRows = kGradItemBytes / 1024;

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

__device__ __forceinline__ float f16_to_f32(uint32_t bits) { return __half2float(__ushort_as_half(static_cast<unsigned short>(bits))); }

// The two elements of a dword (a 32-bit one: itself and zero).
template <uint32_t FORMAT>
__device__ __forceinline__ void elements(uint32_t w, float& a, float& b)
{
    if constexpr (FORMAT == kGradF32) {
        a = __uint_as_float(w);
        b = 0.f;
    } else if constexpr (FORMAT == kGradBf16) {
        a = __uint_as_float(w << 16);
        b = __uint_as_float(w & 0xFFFF0000u);
    } else {
        a = f16_to_f32(w & 0xFFFFu);
        b = f16_to_f32(w >> 16);
    }
}

template <uint32_t FORMAT>
__device__ __forceinline__ void add_squares(double (&sum)[4], const u32x4 w)
{
    static_for<4>([&](auto k) {
        float a, b;
        elements<FORMAT>(w[int(k)], a, b);
        sum[int(k)] = fma(static_cast<double>(a), static_cast<double>(a), sum[int(k)]);
        if constexpr (FORMAT != kGradF32)
            sum[(k + 2) % 4] = fma(static_cast<double>(b), static_cast<double>(b), sum[(k + 2) % 4]);
    });
}

// Of the whole wavefront.  (By scalar additions: this is hardly ever looked at, and should not cost the sums their registers.)
template <uint32_t FORMAT>
__device__ __forceinline__ uint32_t count_nonfinite(const u32x4 w)
{
    uint32_t n = 0;
    static_for<4>([&](auto k) {
        float a, b;
        elements<FORMAT>(w[int(k)], a, b);
        n += __popcll(__ballot(!__builtin_isfinite(a)));
        if constexpr (FORMAT != kGradF32) n += __popcll(__ballot(!__builtin_isfinite(b)));
    });
    return n;
}

// The wavefront's part of an item: whole slots of 16 bytes, and what is left behind the last of them, an
// element for each of the first lanes.  What is not the item's is zero.
struct Rows {
    u32x4 slot[kRows];
    uint32_t rest;
};

__device__ __forceinline__ GradItem item_at(const GradItem* items, const uint32_t i)
{
    const u32x4 w = table_entry(reinterpret_cast<const u32x4*>(items), i);
    return GradItem{w.x | uint64_t(w.y) << 32, w.z, w.w};
}
__device__ __forceinline__ uint32_t item_bytes(const GradItem& it) { return it.what & 0x3FFFFFFFu; }
__device__ __forceinline__ uint32_t item_format(const GradItem& it) { return it.what >> 30; }

template <bool NT>
__device__ __forceinline__ void load_rows(Rows& q, const GradItem& it, const uint8_t* at, const int lane)
{
    const uint32_t bytes = item_bytes(it);
    q.rest = 0;
    if (bytes == kGradItemBytes) {
        static_for<kRows>([&](auto r) { q.slot[int(r)] = load16_unaligned<NT>(at + 1024 * r + 16 * lane); });
        return;
    }
    static_for<kRows>([&](auto r) {
        q.slot[int(r)] = u32x4{0, 0, 0, 0};
        if (1024 * r + 16u * lane + 16 <= bytes) q.slot[int(r)] = load16_unaligned<NT>(at + 1024 * r + 16 * lane);
    });
    const uint32_t whole = bytes & ~15u;
    if (item_format(it) == kGradF32) {
        const uint32_t o = whole + 4 * lane;
        if (o < bytes) q.rest = *as_global(reinterpret_cast<const uint32_t*>(at + o));
    } else {
        const uint32_t o = whole + 2 * lane;
        if (o < bytes) q.rest = *as_global(reinterpret_cast<const uint16_t*>(at + o));
    }
}

template <uint32_t FORMAT>
__device__ __forceinline__ void sum_item(const Rows& q, double& total, uint64_t& bad)
{
    double s[4] = {0, 0, 0, 0};
    static_for<kRows>([&](auto r) {
        add_squares<FORMAT>(s, q.slot[int(r)]);
        __builtin_amdgcn_sched_barrier(0);  // (a row at a time, not 64 elements in 64 bits before the first is added)
    });
    add_squares<FORMAT>(s, u32x4{q.rest, 0, 0, 0});
    const double sum = (s[0] + s[1]) + (s[2] + s[3]);
    if (__any(!__builtin_isfinite(sum))) {
        uint32_t n = count_nonfinite<FORMAT>(u32x4{q.rest, 0, 0, 0});
        static_for<kRows>([&](auto r) { n += count_nonfinite<FORMAT>(q.slot[int(r)]); });
        bad += n;
    }
    total += sum;
}

// What follows from the sum of the squares.  By one thread.
__device__ __forceinline__ void write_stats(ff_grad_stats* out, double sumsq, uint64_t bad, double inv_scale,
                                            double max_norm)
{
    const double norm = sqrt(sumsq) * inv_scale;
    const double factor = norm > max_norm ? max_norm / norm : 1.0;
    out->sumsq = sumsq;
    out->n_nonfinite = bad;
    out->norm = norm;
    out->scale = bad ? 0.f : static_cast<float>(factor * inv_scale);
    out->skip = bad ? 1u : 0u;
}

// Sums over a workgroup of THREADS, in thread 0.  bad: of a whole wavefront.
template <int THREADS>
__device__ __forceinline__ void group_sum(double& sum, uint64_t& bad)
{
    constexpr int kWaves = THREADS / kWaveSize;
    __shared__ double sums[kWaves];
    __shared__ uint64_t bads[kWaves];
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x / kWaveSize;
    sum = wave_sum(sum);
    if (lane == 0) {
        sums[wave] = sum;
        bads[wave] = bad;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; w++) {
            sum += sums[w];
            bad += bads[w];
        }
    }
}

// How the parts of all workgroups are joined in the same launch: workgroups count at one of 32 places, the last one at each
// of them at the root, and the last of those joins the parts, in their order whoever it is.  (On one counter workgroups that end together would queue up, 50 ns each.)
// Counters, on lines of their own, are zero before and after.
struct Joining {
    uint64_t* counts;  // kLeaves, and the root
    GradPart* parts;
    uint32_t n;  // workgroups
    double inv_scale, max_norm;
    ff_grad_stats* stats;
};
constexpr uint32_t kLeaves = 32, kLineWords = 8;
constexpr uint64_t kCountBytes = (kLeaves + 1) * kLineWords * 8;

__device__ __forceinline__ bool is_last(uint64_t* count, uint64_t n)
{
    if (__hip_atomic_fetch_add(count, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 != n) return false;
    __hip_atomic_store(count, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

// By the whole workgroup, whose sums thread 0 has.
__device__ __forceinline__ void join_parts(const Joining& J, double sum, uint64_t bad)
{
    __shared__ int last;
    if (threadIdx.x == 0) {
        const uint32_t at = blockIdx.x;
        // past the caches of this workgroup's XCD, and of the one that joins
        __hip_atomic_store(reinterpret_cast<uint64_t*>(&J.parts[at].sumsq), __builtin_bit_cast(uint64_t, sum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&J.parts[at].n_nonfinite, bad, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("" ::: "memory");
        wait_loads<0>();  // (and stores: they have arrived)
        const uint32_t leaf = at % kLeaves, leaves = J.n < kLeaves ? J.n : kLeaves;
        last = is_last(J.counts + leaf * kLineWords, (J.n - leaf + kLeaves - 1) / kLeaves) &&
               is_last(J.counts + kLeaves * kLineWords, leaves);
    }
    __syncthreads();
    if (!last) return;
    asm volatile("" ::: "memory");
    sum = 0;
    bad = 0;
    constexpr int kAtOnce = 8;  // on their way
    for (uint32_t i0 = threadIdx.x; i0 < J.n; i0 += kAtOnce * kThreads) {
        uint64_t part[kAtOnce][2];
        static_for<kAtOnce>([&](auto k) {
            const uint32_t i = i0 + k * kThreads;
            const auto* const p = reinterpret_cast<const uint64_t*>(J.parts + (i < J.n ? i : i0));
            static_for<2>([&](auto w) { part[int(k)][int(w)] = __hip_atomic_load(p + w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); });
        });
        static_for<kAtOnce>([&](auto k) {
            if (i0 + k * kThreads < J.n) {
                sum += __builtin_bit_cast(double, part[int(k)][0]);
                bad += part[int(k)][1];
            }
        });
    }
    if (__any(bad != 0)) {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) bad += __shfl_xor(static_cast<unsigned long long>(bad), d);
    }
    group_sum<kThreads>(sum, bad);
    if (threadIdx.x == 0) write_stats(J.stats, sum, bad, J.inv_scale, J.max_norm);
}

// Addresses of the tensors: the list's, in memory, or the call's, in the arguments.
struct ListAddresses {
    const uint64_t* p;
    __device__ __forceinline__ uint64_t of(uint32_t tensor) const { return table_entry(p, tensor); }
};
struct CallAddresses {
    uint32_t base;
    GradPtrs grads;
    __device__ __forceinline__ uint64_t of(uint32_t tensor) const { return grads.p[tensor - base]; }
};

template <class Addresses>
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const GradItem* __restrict__ items, uint32_t n_items,
                                                             const Joining J, Addresses addresses)
{
    const int lane = threadIdx.x & (kWaveSize - 1);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const uint32_t stride = gridDim.x * kGradWaves;
    double sum = 0;
    uint64_t bad = 0;
    for (uint32_t i = blockIdx.x * kGradWaves + wave; i < n_items; i += stride) {
        const GradItem it = item_at(items, i);
        Rows q;
        load_rows<true>(q, it, reinterpret_cast<const uint8_t*>(addresses.of(it.tensor)) + it.begin, lane);
        switch (item_format(it)) {
        case kGradF32: sum_item<kGradF32>(q, sum, bad); break;
        case kGradBf16: sum_item<kGradBf16>(q, sum, bad); break;
        default: sum_item<kGradF16>(q, sum, bad);
        }
    }
    group_sum<kThreads>(sum, bad);
    join_parts(J, sum, bad);
}

// The addresses of a call into its workspace, for lists of more tensors than a launch's arguments hold: the norm is one launch, over the same
// parts in the same order, wherever addresses come from.
__global__ __launch_bounds__(kThreads) void grad_addresses_kernel(const CallAddresses addresses, const uint32_t n, uint64_t* table)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i < n) table[addresses.base + i] = addresses.grads.p[i];
}

// One wavefront: it loads the parts side by side, and adds them one after the other.
__global__ __launch_bounds__(kWaveSize) void grad_join_kernel(const ff_grad_stats* parts, uint64_t n, double inv_scale,
                                                              double max_norm, ff_grad_stats* stats)
{
    double sum = 0;
    uint64_t bad = 0;
    for (uint64_t i0 = 0; i0 < n; i0 += kWaveSize) {
        const uint64_t i = i0 + threadIdx.x;
        const double s = i < n ? parts[i].sumsq : 0.0;
        const unsigned long long b = i < n ? parts[i].n_nonfinite : 0;
        for (int k = 0; k < kWaveSize; k++) {
            sum += __shfl(s, k);
            bad += __shfl(b, k);
        }
    }
    if (threadIdx.x == 0) write_stats(stats, sum, bad, inv_scale, max_norm);
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The elements of a dword, multiplied in fp32 and rounded to nearest even.
template <uint32_t FORMAT>
__device__ __forceinline__ uint32_t scaled(uint32_t w, const float scale)
{
    float a, b;
    elements<FORMAT>(w, a, b);
    if constexpr (FORMAT == kGradF32) return __float_as_uint(a * scale);
    if constexpr (FORMAT == kGradBf16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a * scale, b * scale}, bf16x2));
    return __half_as_ushort(__float2half_rn(a * scale)) | uint32_t(__half_as_ushort(__float2half_rn(b * scale))) << 16;
}

template <uint32_t FORMAT>
__device__ __forceinline__ void clip_item(const Rows& q, const uint32_t bytes, uint8_t* at, const float scale, const int lane)
{
    static_for<kRows>([&](auto r) {
        u32x4 w = q.slot[int(r)];
        static_for<4>([&](auto k) { w[int(k)] = scaled<FORMAT>(w[int(k)], scale); });
        if (1024 * r + 16u * lane + 16 <= bytes) store16_unaligned<true>(at + 1024 * r + 16 * lane, w);
    });
    constexpr uint32_t kItem = FORMAT == kGradF32 ? 4 : 2;
    const uint32_t o = (bytes & ~15u) + kItem * lane;
    if (o < bytes) {
        const uint32_t w = scaled<FORMAT>(q.rest, scale);
        if constexpr (FORMAT == kGradF32)
            *as_global(reinterpret_cast<uint32_t*>(at + o)) = w;
        else
            *as_global(reinterpret_cast<uint16_t*>(at + o)) = static_cast<uint16_t>(w);
    }
}

// Workgroups to a run of an XCD (xcd_order.h), us, 1.7 GB of bf16 in place, in launch order / 2 / 4 / 8 / 16 / 32 / 64 / 2048 615 / 600 / 559 /
// 561 / 560 / 588 / 575 / 586 (a copy of as many bytes: 529); plain loads or stores instead of non-temporal ones, in launch order, 670 and
// 636; two or four items to a wavefront, one after the other, 591 and 589.
constexpr uint32_t kClipXcdGroup = 8;
template <class Addresses>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(const GradItem* __restrict__ items, uint32_t n_items,
                                                             const ff_grad_stats* __restrict__ stats, Addresses addresses)
{
    const float scale = stats->scale;
    if (stats->skip || scale == 1.f) return;
    const int lane = threadIdx.x & (kWaveSize - 1);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const uint32_t i = xcd_order(blockIdx.x, gridDim.x, kClipXcdGroup) * kGradWaves + wave;
    if (i >= n_items) return;
    const GradItem it = item_at(items, i);
    uint8_t* const at = reinterpret_cast<uint8_t*>(addresses.of(it.tensor)) + it.begin;
    const uint32_t bytes = item_bytes(it);
    Rows q;
    load_rows<true>(q, it, at, lane);
    switch (item_format(it)) {
    case kGradF32: clip_item<kGradF32>(q, bytes, at, scale, lane); break;
    case kGradBf16: clip_item<kGradBf16>(q, bytes, at, scale, lane); break;
    default: clip_item<kGradF16>(q, bytes, at, scale, lane);
    }
}

CallAddresses call_addresses(const GradWork& work, const void* const* grads, uint64_t k)
{
    CallAddresses a;
    a.base = static_cast<uint32_t>(k * kGradsPerLaunch);
    for (uint32_t i = 0; i < kGradsPerLaunch; i++)
        a.grads.p[i] = a.base + i < work.n ? reinterpret_cast<uint64_t>(grads[a.base + i]) : 0;
    return a;
}

}  // namespace

bool build_grad_items(const ff_segment* segs, uint64_t n, std::vector<GradItem>& items, std::vector<uint32_t>& begin)
{
    uint64_t count = 0;  // before any of them is stored
    for (uint64_t k = 0; k < n; k++) {
        count += segs[k].nbytes / kGradItemBytes + (segs[k].nbytes % kGradItemBytes != 0);
        if (count > (1ull << 31)) return false;
    }
    items.reserve(count);
    begin.push_back(0);
    for (uint64_t k = 0; k < n; k++) {
        if (k && k % kGradsPerLaunch == 0) begin.push_back(static_cast<uint32_t>(items.size()));
        const uint32_t format = segs[k].dtype == FF_F32 ? kGradF32 : segs[k].dtype == FF_BF16 ? kGradBf16 : kGradF16;
        for (uint64_t b = 0; b < segs[k].nbytes; b += kGradItemBytes) {
            const uint64_t left = segs[k].nbytes - b;
            items.push_back({b, static_cast<uint32_t>(k),
                             static_cast<uint32_t>(left < kGradItemBytes ? left : kGradItemBytes) | format << 30});
        }
    }
    begin.push_back(static_cast<uint32_t>(items.size()));
    return true;
}

// The workspace: counters, parts, and the addresses of a call on a long list.
hipError_t launch_grad_norm(const GradWork& work, const void* const* grads, double inv_scale, double max_norm,
                            void* workspace, ff_grad_stats* stats, hipStream_t stream)
{
    uint8_t* const w = static_cast<uint8_t*>(workspace);
    const uint32_t n_items = work.launch.back(), groups = grad_groups(n_items);
    const Joining J = {reinterpret_cast<uint64_t*>(w), reinterpret_cast<GradPart*>(w + kCountBytes), groups, inv_scale, max_norm, stats};
    auto norm = [&](const auto& addresses) {
        hipLaunchKernelGGL(grad_norm_kernel<std::decay_t<decltype(addresses)>>, dim3(groups), dim3(kThreads), 0, stream, work.items, n_items, J,
                           addresses);
        return hipGetLastError();
    };
    if (!grads) return norm(ListAddresses{work.address});
    if (work.n <= kGradsPerLaunch) return norm(call_addresses(work, grads, 0));
    uint64_t* const table = reinterpret_cast<uint64_t*>(w + kCountBytes + groups * sizeof(GradPart));
    for (uint64_t k = 0; k * kGradsPerLaunch < work.n; k++) {
        const uint64_t left = work.n - k * kGradsPerLaunch;
        const uint32_t n = static_cast<uint32_t>(left < kGradsPerLaunch ? left : kGradsPerLaunch);
        hipLaunchKernelGGL(grad_addresses_kernel, dim3((n + kThreads - 1) / kThreads), dim3(kThreads), 0, stream,
                           call_addresses(work, grads, k), n, table);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return norm(ListAddresses{table});
}

uint64_t grad_workspace(const GradWork& work)
{
    return kCountBytes + grad_groups(work.launch.back()) * sizeof(GradPart) + (work.n > kGradsPerLaunch ? work.n * sizeof(uint64_t) : 0);
}

hipError_t launch_grad_join(const ff_grad_stats* parts, uint64_t n, double inv_scale, double max_norm,
                            ff_grad_stats* stats, hipStream_t stream)
{
    hipLaunchKernelGGL(grad_join_kernel, dim3(1), dim3(kWaveSize), 0, stream, parts, n, inv_scale, max_norm, stats);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const GradWork& work, const void* const* grads, const ff_grad_stats* stats, hipStream_t stream)
{
    auto clip = [&](uint32_t begin, const uint32_t end, const auto& addresses) {
        constexpr uint32_t kMost = most_groups(kThreads) * kGradWaves;
        while (begin < end) {
            const uint32_t n = end - begin < kMost ? end - begin : kMost;
            hipLaunchKernelGGL(grad_clip_kernel<std::decay_t<decltype(addresses)>>, dim3((n + kGradWaves - 1) / kGradWaves), dim3(kThreads), 0,
                               stream, work.items + begin, n, stats, addresses);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            begin += n;
        }
        return hipSuccess;
    };
    if (!grads) return clip(0, work.launch.back(), ListAddresses{work.address});
    for (size_t k = 0; k + 1 < work.launch.size(); k++) {
        const hipError_t e = clip(work.launch[k], work.launch[k + 1], call_addresses(work, grads, k));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ffsnap
