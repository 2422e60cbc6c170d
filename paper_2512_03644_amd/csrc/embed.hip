// Embedding of tokens with scaling, and its gradient by sorted tokens, for gfx950.
//
// Lookup: out[t] = scale * table[id[t]], a wavefront to eight times 64 elements of a token's row.
//
// Gradient: dtable[v] (+)= scale * (sum of dout[t] over the tokens t with id v).  Tokens are sorted by id, and among equal ids
// by their position, so that a row's sum has one order.  The table's ids are dealt out to workgroups in ranges; each reads all ids,
// keeps its own in order, and knows from how many it has seen below its range where its part of the sorted list begins: one launch, with
// no workgroup waiting for another.  Then a wavefront makes 512 elements of a row of the table: the sum of its tokens' rows.  Rows of more than
// kPart tokens -- frequent words -- are summed in parts first, a wavefront to kPart entries of the sorted list, in 32 bits, and joined in
// their order.
//
// What bounds it: memory; few tokens: the launches.
#include "embed.hpp"

#include <algorithm>

#include "rows.h"
#include "xcd_order.h"

namespace ffsnap {

namespace {

constexpr uint32_t kWaves = 4, kSlab = kWaveSize * kLaneItems;  // elements of a row that a wavefront makes

__device__ __forceinline__ uint32_t wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize); }

// ---- lookup -----------------------------------------------------------------------------------------

template <uint32_t DTYPE>
__global__ __launch_bounds__(kWaveSize * kWaves) void embed_kernel(const EmbedArgs a, const uint32_t slabs)
{
    using I = Items<DTYPE>;
    const uint32_t width = static_cast<uint32_t>(a.width);
    const uint64_t total = a.n_tokens * slabs, step = static_cast<uint64_t>(gridDim.x) * kWaves;
    for (uint64_t w = static_cast<uint64_t>(blockIdx.x) * kWaves + wave_of(); w < total; w += step) {
        const uint64_t t = w / slabs;
        const uint32_t at = static_cast<uint32_t>(w - t * slabs) * kSlab + threadIdx.x % kWaveSize * kLaneItems;
        if (at >= width) continue;
        const int64_t id = a.ids[t];
        f32x8 v = {};
        if (id >= 0 && static_cast<uint64_t>(id) < a.vocab)
            v = I::wide(I::load(a.rows + static_cast<uint64_t>(id) * a.rows_stride * I::kBytes, at, width)) * a.scale;
        I::store(a.out + t * a.out_stride * I::kBytes, at, width, I::narrow(v));
    }
}

// ---- order of the tokens ------------------------------------------------------------------------------

constexpr uint32_t kSortThreads = 1024, kSortWaves = kSortThreads / kWaveSize, kSortRounds = 8;
constexpr uint32_t kSortIds = kSortThreads * kSortRounds;  // that a workgroup looks at at once
constexpr uint32_t kRange = 512;                           // ids of a workgroup
constexpr uint32_t kPart = 32;                             // entries of the sorted list that are summed by themselves at most

struct Sorted {
    uint32_t* begin;  // [vocab + 1] of every id's tokens in the list
    uint32_t* order;  // the list: positions of tokens
    uint32_t* ids;    // and their ids
    float* parts;     // [2 * parts of the list][width]: sums of long rows' parts
};

__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const EmbedArgs a, const Sorted s)
{
    __shared__ uint32_t bins[kRange], mine_at[kSortIds], sums[kSortWaves], below_of[kSortWaves];
    __shared__ uint16_t mine_bin[kSortIds], wave_bins[kSortWaves][kRange];
    const uint32_t n = static_cast<uint32_t>(a.n_tokens), wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    const uint32_t first = blockIdx.x * kRange, vocab = static_cast<uint32_t>(a.vocab);
    const uint32_t range = vocab - first < kRange ? vocab - first : kRange;
    const uint64_t lower = (1ull << lane) - 1;
    // an id's place in the range; above it: an id of another workgroup, or none.  `below`: those of the workgroups before this one
    auto place = [&](uint64_t t, uint32_t& below) {
        if (t >= n) return kRange;
        const int64_t id = a.ids[t];
        below += id >= 0 && id < static_cast<int64_t>(first);
        const uint64_t in = static_cast<uint64_t>(id) - first;
        return id >= 0 && in < range ? static_cast<uint32_t>(in) : kRange;
    };
    for (uint32_t i = threadIdx.x; i < kRange; i += kSortThreads) bins[i] = 0;
    __syncthreads();
    uint32_t below = 0, unused = 0;
    for (uint64_t t = threadIdx.x; t < n; t += kSortThreads) {
        const uint32_t b = place(t, below);
        if (b < kRange) atomicAdd(&bins[b], 1u);
    }
    for (int d = 32; d; d /= 2) below += __shfl_xor(below, d);
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    // where each id's tokens begin
    below = 0;
    for (uint32_t k = 0; k < kSortWaves; k++) below += below_of[k];
    {
        uint32_t x = threadIdx.x < kRange ? bins[threadIdx.x] : 0;
        const uint32_t own = x;
        for (int d = 1; d < kWaveSize; d *= 2) {
            const uint32_t y = __shfl_up(x, d);
            if (lane >= static_cast<uint32_t>(d)) x += y;
        }
        if (lane == kWaveSize - 1) sums[wave] = x;
        __syncthreads();
        for (uint32_t k = 0; k < wave; k++) x += sums[k];
        if (threadIdx.x < kRange) bins[threadIdx.x] = below + x - own;
        if (threadIdx.x < range) s.begin[first + threadIdx.x] = below + x - own;
        if (first + range == vocab && threadIdx.x == range - 1) s.begin[vocab] = below + x;
    }
    __syncthreads();
    // the range's tokens, kSortIds ids at a time: in their order into LDS, and from there each behind the last one of its id
    for (uint64_t from = 0; from < n; from += kSortIds) {
        uint32_t b[kSortRounds], count = 0;
        const uint64_t t0 = from + wave * (kWaveSize * kSortRounds) + lane;
        for (uint32_t i = 0; i < kSortRounds; i++) {
            b[i] = place(t0 + i * kWaveSize, unused);
            count += __popcll(__ballot(b[i] < kRange));
        }
        if (lane == 0) sums[wave] = count;
        __syncthreads();
        uint32_t at = 0, all = 0;
        for (uint32_t k = 0; k < kSortWaves; k++) {
            if (k < wave) at += sums[k];
            all += sums[k];
        }
        for (uint32_t i = 0; i < kSortRounds; i++) {
            const uint64_t who = __ballot(b[i] < kRange);
            if (b[i] < kRange) {
                const uint32_t k = at + __popcll(who & lower);
                mine_at[k] = static_cast<uint32_t>(t0 + i * kWaveSize);
                mine_bin[k] = static_cast<uint16_t>(b[i]);
            }
            at += __popcll(who);
        }
        for (uint32_t first_k = 0; first_k < all; first_k += kSortThreads) {
            for (uint32_t i = threadIdx.x; i < kSortWaves * kRange / 2; i += kSortThreads) reinterpret_cast<uint32_t*>(wave_bins)[i] = 0;
            __syncthreads();  // (and what has been put into LDS is there)
            const uint32_t k = first_k + threadIdx.x;
            const bool on = k < all;
            const uint32_t bin = on ? mine_bin[k] : 0;
            uint64_t same = __ballot(on);
            for (uint32_t bit = 1; bit < kRange; bit *= 2) {
                const uint64_t set = __ballot(bin & bit);
                same &= bin & bit ? set : ~set;
            }
            if (on && (same & lower) == 0) wave_bins[wave][bin] = static_cast<uint16_t>(__popcll(same));
            __syncthreads();
            uint32_t to = 0;
            if (on) {
                to = bins[bin] + __popcll(same & lower);
                for (uint32_t w = 0; w < wave; w++) to += wave_bins[w][bin];
            }
            __syncthreads();
            if (threadIdx.x < kRange) {
                uint32_t more = 0;
                for (uint32_t w = 0; w < kSortWaves; w++) more += wave_bins[w][threadIdx.x];
                bins[threadIdx.x] += more;
            }
            if (on) {
                s.order[to] = mine_at[k];
                s.ids[to] = first + bin;
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

// ---- sums -------------------------------------------------------------------------------------------

// The rows of tokens order[from .. to), elements [at, at + 8).
template <uint32_t DTYPE>
__device__ __forceinline__ f32x8 sum_of(const EmbedArgs& a, const uint32_t* order, uint32_t from, uint32_t to, uint32_t at)
{
    using I = Items<DTYPE>;
    constexpr uint32_t kAhead = 4;
    const uint32_t width = static_cast<uint32_t>(a.width);
    f32x8 sum = {};
    auto row = [&](uint32_t k) { return a.rows + static_cast<uint64_t>(order[k]) * a.rows_stride * I::kBytes; };
    uint32_t k = from;
    for (; k + kAhead <= to; k += kAhead) {
        typename I::Held h[kAhead];
        static_for<kAhead>([&](auto i) { h[int(i)] = I::load(row(k + i), at, width); });
        static_for<kAhead>([&](auto i) { sum += I::wide(h[int(i)]); });
    }
    for (; k < to; k++) sum += I::wide(I::load(row(k), at, width));
    return sum;
}

// Entries [kPart * c, kPart * (c + 1)) of the list: what they add to the long rows, of which two at most reach in.
template <uint32_t DTYPE>
__global__ __launch_bounds__(kWaveSize* kWaves) void embed_parts_kernel(const EmbedArgs a, const Sorted s, const uint32_t slabs)
{
    const uint32_t vocab = static_cast<uint32_t>(a.vocab), width = static_cast<uint32_t>(a.width);
    const uint32_t n = s.begin[vocab], n_parts = (n + kPart - 1) / kPart;
    const uint64_t total = static_cast<uint64_t>(n_parts) * slabs, step = static_cast<uint64_t>(gridDim.x) * kWaves;
    for (uint64_t w = static_cast<uint64_t>(blockIdx.x) * kWaves + wave_of(); w < total; w += step) {
        const uint32_t c = static_cast<uint32_t>(w / slabs), begin = c * kPart, end = begin + kPart < n ? begin + kPart : n;
        const uint32_t at = static_cast<uint32_t>(w - static_cast<uint64_t>(c) * slabs) * kSlab + threadIdx.x % kWaveSize * kLaneItems;
        if (at >= width) continue;
        const uint32_t ids[2] = {s.ids[begin], s.ids[end - 1]};
        for (int i = 0; i < 2; i++) {
            if (i && ids[1] == ids[0]) break;
            const uint32_t from = s.begin[ids[i]], to = s.begin[ids[i] + 1];
            if (to - from <= kPart) continue;
            const f32x8 sum = sum_of<DTYPE>(a, s.order, from > begin ? from : begin, to < end ? to : end, at);
            Items<FF_F32>::store(reinterpret_cast<uint8_t*>(s.parts + (2ull * c + (from >= begin)) * width), at, width, Items<FF_F32>::narrow(sum));
        }
    }
}

// Rows of the table: all of them, or (ADD) those that tokens have, found at their first entry in the list.
template <uint32_t DTYPE, bool ADD>
__global__ __launch_bounds__(kWaveSize* kWaves) void embed_grad_kernel(const EmbedArgs a, const Sorted s, const uint32_t slabs)
{
    using I = Items<DTYPE>;
    using F = Items<FF_F32>;
    const uint32_t vocab = static_cast<uint32_t>(a.vocab), width = static_cast<uint32_t>(a.width);
    const uint64_t total = static_cast<uint64_t>(ADD ? s.begin[vocab] : vocab) * slabs, step = static_cast<uint64_t>(gridDim.x) * kWaves;
    for (uint64_t w = static_cast<uint64_t>(blockIdx.x) * kWaves + wave_of(); w < total; w += step) {
        const uint32_t which = static_cast<uint32_t>(w / slabs);
        const uint32_t at = static_cast<uint32_t>(w - static_cast<uint64_t>(which) * slabs) * kSlab + threadIdx.x % kWaveSize * kLaneItems;
        const uint32_t id = ADD ? s.ids[which] : which, from = s.begin[id], to = s.begin[id + 1];
        if (at >= width || (ADD && which != from)) continue;
        f32x8 sum = {};
        if (to - from <= kPart) {
            sum = sum_of<DTYPE>(a, s.order, from, to, at);
        } else {
            for (uint32_t c = from / kPart; c * kPart < to; c++)
                sum += F::wide(F::load(reinterpret_cast<const uint8_t*>(s.parts + (2ull * c + (from >= c * kPart)) * width), at, width));
        }
        sum *= a.scale;
        uint8_t* const out = a.out + static_cast<uint64_t>(id) * a.out_stride * I::kBytes;
        if (ADD) sum += I::wide(I::load(out, at, width));
        I::store(out, at, width, I::narrow(sum));
    }
}

uint64_t up(uint64_t x) { return (x + 255) / 256 * 256; }

struct Places {
    uint64_t begin, order, ids, parts, bytes;
};
Places place(uint64_t n, uint64_t vocab, uint64_t width)
{
    Places p = {};
    p.order = up((vocab + 1) * 4);
    p.ids = p.order + up(n * 4);
    p.parts = p.ids + up(n * 4);
    p.bytes = p.parts + (n / kPart + 1) * 2 * width * 4;
    return p;
}

// Workgroups for so many wavefronts' work, several rounds for each where there is much.
uint32_t groups(uint64_t waves) { return static_cast<uint32_t>(std::max<uint64_t>(1, std::min<uint64_t>((waves + kWaves - 1) / kWaves, 1u << 20))); }

template <uint32_t DTYPE>
hipError_t launch_grad(const EmbedArgs& a, bool add, const Sorted& s, hipStream_t stream)
{
    const uint32_t slabs = static_cast<uint32_t>((a.width + kSlab - 1) / kSlab);
    hipLaunchKernelGGL(embed_sort_kernel, dim3(static_cast<uint32_t>((a.vocab + kRange - 1) / kRange)), dim3(kSortThreads), 0, stream, a, s);
    const dim3 threads(kWaveSize * kWaves);
    if (a.n_tokens > kPart)
        hipLaunchKernelGGL(embed_parts_kernel<DTYPE>, dim3(groups((a.n_tokens / kPart + 1) * slabs)), threads, 0, stream, a, s, slabs);
    if (add)
        hipLaunchKernelGGL((embed_grad_kernel<DTYPE, true>), dim3(groups(a.n_tokens * slabs)), threads, 0, stream, a, s, slabs);
    else
        hipLaunchKernelGGL((embed_grad_kernel<DTYPE, false>), dim3(groups(a.vocab * slabs)), threads, 0, stream, a, s, slabs);
    return hipGetLastError();
}

}  // namespace

uint64_t embed_workspace(uint64_t n_tokens, uint64_t vocab, uint64_t width) { return place(n_tokens, vocab, width).bytes; }

hipError_t launch_embed(const EmbedArgs& a, uint32_t dtype, hipStream_t stream)
{
    if (!a.n_tokens) return hipSuccess;
    const uint32_t slabs = static_cast<uint32_t>((a.width + kSlab - 1) / kSlab);
    const dim3 grid(groups(a.n_tokens * slabs)), threads(kWaveSize * kWaves);
    if (dtype == FF_BF16) hipLaunchKernelGGL(embed_kernel<FF_BF16>, grid, threads, 0, stream, a, slabs);
    else if (dtype == FF_F16) hipLaunchKernelGGL(embed_kernel<FF_F16>, grid, threads, 0, stream, a, slabs);
    else hipLaunchKernelGGL(embed_kernel<FF_F32>, grid, threads, 0, stream, a, slabs);
    return hipGetLastError();
}

hipError_t launch_embed_grad(const EmbedArgs& a, uint32_t dtype, bool add, void* workspace, hipStream_t stream)
{
    if (add && !a.n_tokens) return hipSuccess;
    const Places p = place(a.n_tokens, a.vocab, a.width);
    uint8_t* const w = static_cast<uint8_t*>(workspace);
    const Sorted s = {reinterpret_cast<uint32_t*>(w + p.begin), reinterpret_cast<uint32_t*>(w + p.order), reinterpret_cast<uint32_t*>(w + p.ids),
                      reinterpret_cast<float*>(w + p.parts)};
    if (dtype == FF_BF16) return launch_grad<FF_BF16>(a, add, s, stream);
    if (dtype == FF_F16) return launch_grad<FF_F16>(a, add, s, stream);
    return launch_grad<FF_F32>(a, add, s, stream);
}

}  // namespace ffsnap
