// Embedding of tokens with scaling, and its gradient by sorted tokens, for gfx950.
//
// Lookup: out[t] = scale * table[id[t]], a wavefront to eight times 64 elements of a token's row.
//
// Gradient: dtable[v] (+)= scale * (sum of dout[t] over the tokens t with id v).  Tokens are sorted by id, and among equal ids
// by their position, so that a row's sum has one order.  The table's ids are dealt out to workgroups in ranges; each reads all ids,
// keeps its own in order, and knows from how many it has seen below its range where its part of the sorted list begins: one launch, with
// no workgroup waiting for another.  Then the list is cut into parts of equal length, frequent words or not: a wavefront takes 512 elements
// of the rows of a part's tokens, and writes every sum that begins and ends there.  What reaches over a part's ends is left
// in the workspace, in 32 bits, and a last launch joins it in its order.
//
// What bounds it: memory; few tokens: the steps of a workgroup, which hang on one another.  Lookup of 16,384 tokens of 8192 bf16 elements 84 us; gradient of 16,384 tokens of 4096 added to 32,000 rows 75 us: the
// list 14, sums 36 (of 134 MB and 89 MB of rows read and written, 6.0 TB/s), joins 7.
#include "embed.hpp"

#include <algorithm>

#include "rows.h"
#include "xcd_order.h"

namespace ffsnap {

namespace {

constexpr uint32_t kWaves = 4, kSlab = kWaveSize * kLaneItems;  // elements of a row that a wavefront makes

__device__ __forceinline__ uint32_t wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize); }

// ---- lookup -----------------------------------------------------------------------------------------

template <class I, bool PAST>
__global__ __launch_bounds__(kWaveSize * kWaves) void embed_kernel(const EmbedArgs a, const uint32_t slabs)
{
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
        I::template store<PAST>(a.out + t * a.out_stride * I::kBytes, at, width, I::narrow(v));
    }
}

// Rows [0, n) of the table's gradient from `out` on, elements [from, to): zeros in those that `which(row)` names.  `waves` wavefronts, of which this
// is number `wave`; as many rows at a time as a wavefront has lanes for.
template <class I, bool PAST, class Which>
__device__ __forceinline__ void clear_rows(uint8_t* out, uint64_t stride, uint64_t n, uint32_t from, uint32_t to, uint64_t wave, uint64_t waves, Which&& which)
{
    const uint32_t lane = threadIdx.x % kWaveSize;
    uint32_t lanes = 1;  // of a row
    while (lanes < kWaveSize && lanes * kLaneItems < to - from) lanes *= 2;
    const uint32_t rows = kWaveSize / lanes;
    for (uint64_t r = wave * rows + lane / lanes; r < n; r += waves * rows)
        if (which(r))
            for (uint32_t at = from + lane % lanes * kLaneItems; at < to; at += lanes * kLaneItems)
                I::template store<PAST>(out + r * stride * I::kBytes, at, to, I::narrow(f32x8{}));
}

// The sum over a wavefront's lanes that have the same elements, every `lanes`-th, in the first of them.
__device__ __forceinline__ f32x8 join_turns(f32x8 sum, uint32_t lanes)
{
    for (uint32_t d = kWaveSize / 2; d >= lanes; d /= 2)
        static_for<8>([&](auto i) { sum[int(i)] += __shfl_down(sum[int(i)], d); });
    return sum;
}

// ---- order of the tokens ------------------------------------------------------------------------------

constexpr uint32_t kSortThreads = 1024, kSortWaves = kSortThreads / kWaveSize, kSortRounds = 16;
constexpr uint32_t kSortIds = kSortThreads * kSortRounds;  // that a workgroup looks at at once
constexpr uint32_t kRange = 256;                           // ids of a workgroup

struct Sorted {
    uint32_t* begin;  // [vocab + 1] of every id's tokens in the list
    uint32_t* order;  // the list: positions of tokens
    uint32_t* ids;    // and their ids
    float* ends;      // [part of the list][its beginning, its end][width]: sums that reach over it
    uint32_t part;    // entries of a part
    uint32_t* counts; // of runs that reach over parts' ends: over few parts, over many
    uint2* runs[2];   // the part that each begins in, and its last one, in any order
};
constexpr uint32_t kManyParts = 8;  // more than these

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
    if (blockIdx.x == 0 && threadIdx.x < 2) s.counts[threadIdx.x] = 0;
    __syncthreads();
    // ids of one round: a wavefront's follow each other.  Those of the last round are kept: up to kSortIds tokens are read once
    uint32_t below = 0, unused = 0, b[kSortRounds];
    auto look = [&](uint64_t from, uint32_t& low) {
        const uint64_t t0 = from + wave * (kWaveSize * kSortRounds) + lane;
        static_for<kSortRounds>([&](auto i) { b[int(i)] = place(t0 + i * kWaveSize, low); });
    };
    for (uint64_t from = 0; from < n; from += kSortIds) {
        look(from, below);
        static_for<kSortRounds>([&](auto i) {
            if (b[int(i)] < kRange) atomicAdd(&bins[b[int(i)]], 1u);
        });
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
        uint32_t count = 0;
        const uint64_t t0 = from + wave * (kWaveSize * kSortRounds) + lane;
        if (n > kSortIds) look(from, unused);
        static_for<kSortRounds>([&](auto i) { count += __popcll(__ballot(b[int(i)] < kRange)); });
        if (lane == 0) sums[wave] = count;
        __syncthreads();
        uint32_t at = 0, all = 0;
        for (uint32_t k = 0; k < kSortWaves; k++) {
            if (k < wave) at += sums[k];
            all += sums[k];
        }
        static_for<kSortRounds>([&](auto i) {
            const uint64_t who = __ballot(b[int(i)] < kRange);
            if (b[int(i)] < kRange) {
                const uint32_t k = at + __popcll(who & lower);
                mine_at[k] = static_cast<uint32_t>(t0 + i * kWaveSize);
                mine_bin[k] = static_cast<uint16_t>(b[int(i)]);
            }
            at += __popcll(who);
        });
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

// Part c of the list, for a whole wavefront.
struct Part {
    const uint32_t *ids, *order;  // of its first entry
    uint32_t count;
    bool joins_before, joins_behind;  // its first run begins in front of it, its last one ends behind it
    __device__ __forceinline__ Part(const Sorted& s, uint32_t c, uint32_t n)
    {
        const uint32_t begin = c * s.part;
        count = n - begin < s.part ? n - begin : s.part;
        ids = s.ids + begin;
        order = s.order + begin;
        joins_before = c && table_entry(s.ids, begin - 1) == id_of(0);
        joins_behind = begin + count < n && table_entry(s.ids, begin + count) == id_of(count - 1);
    }
    __device__ __forceinline__ uint32_t id_of(uint32_t i) const { return table_entry(ids, i); }
    __device__ __forceinline__ uint32_t token_of(uint32_t i) const { return table_entry(order, i); }
    // does the run of the last entry begin in the part?
    __device__ __forceinline__ bool last_begins() const { return !joins_before || id_of(count - 1) != id_of(0); }
};

// Elements [at, at + 8) of a part's tokens' rows; ADD: sums are added to what is there.
template <class I, bool ADD, bool PAST>
__device__ __forceinline__ void sum_part(const EmbedArgs& a, const Sorted& s, uint32_t c, uint32_t n, uint32_t at)
{
    constexpr uint32_t kAhead = 4;
    const uint32_t width = static_cast<uint32_t>(a.width);
    const Part p(s, c, n);
    if (p.joins_behind && p.last_begins() && at < kLaneItems) {  // (one lane, of one wavefront to a part)
        const uint32_t last = (s.begin[p.id_of(p.count - 1) + 1] - 1) / s.part;
        const uint32_t many = last - c >= kManyParts;
        s.runs[many][atomicAdd(s.counts + many, 1u)] = uint2{c, last};
    }
    if (at >= width) return;
    bool begins = !p.joins_before;  // does the run at work begin in this part?
    f32x8 sum = {};
    for (uint32_t k = 0; k < p.count; k += kAhead) {
        typename I::Held h[kAhead], old[kAhead];
        bool ends[kAhead], whole[kAhead];
        bool first = begins;
        static_for<kAhead>([&](auto i) {
            ends[int(i)] = whole[int(i)] = false;
            if (k + i >= p.count) return;
            const uint32_t id = p.id_of(k + i);
            h[int(i)] = I::load(a.rows + static_cast<uint64_t>(p.token_of(k + i)) * a.rows_stride * I::kBytes, at, width);
            ends[int(i)] = k + i + 1 == p.count || p.id_of(k + i + 1) != id;
            whole[int(i)] = ends[int(i)] && first && !(k + i + 1 == p.count && p.joins_behind);
            if (ADD && whole[int(i)]) old[int(i)] = I::load(a.out + static_cast<uint64_t>(id) * a.out_stride * I::kBytes, at, width);
            if (ends[int(i)]) first = true;
        });
        static_for<kAhead>([&](auto i) {
            if (k + i >= p.count) return;
            sum += I::wide(h[int(i)]);
            if (!ends[int(i)]) return;
            if (whole[int(i)]) {
                sum *= a.scale;
                if (ADD) sum += I::wide(old[int(i)]);
                I::template store<PAST>(a.out + static_cast<uint64_t>(p.id_of(k + i)) * a.out_stride * I::kBytes, at, width, I::narrow(sum));
            } else {
                I::Wide::store(reinterpret_cast<uint8_t*>(s.ends + (2ull * c + begins) * width), at, width, I::Wide::narrow(sum));
            }
            begins = true;
            sum = f32x8{};
        });
    }
}

// The first `sum_blocks` workgroups: the parts of the list.  The others, unless it is added: zeros into rows without tokens.
template <class I, bool ADD, bool PAST>
__global__ __launch_bounds__(kWaveSize* kWaves) void embed_sum_kernel(const EmbedArgs a, const Sorted s, const uint32_t slabs, const uint32_t sum_blocks)
{
    const uint32_t vocab = static_cast<uint32_t>(a.vocab), width = static_cast<uint32_t>(a.width), n = s.begin[vocab];
    const uint32_t lane_at = threadIdx.x % kWaveSize * kLaneItems;
    if (blockIdx.x < sum_blocks) {
        const uint64_t total = static_cast<uint64_t>((n + s.part - 1) / s.part) * slabs, step = static_cast<uint64_t>(sum_blocks) * kWaves;
        for (uint64_t w = static_cast<uint64_t>(blockIdx.x) * kWaves + wave_of(); w < total; w += step) {
            const uint32_t c = static_cast<uint32_t>(w / slabs), at = static_cast<uint32_t>(w - static_cast<uint64_t>(c) * slabs) * kSlab + lane_at;
            sum_part<I, ADD, PAST>(a, s, c, n, at);
        }
    } else if (!ADD) {
        clear_rows<I, PAST>(a.out, a.out_stride, vocab, 0, width, static_cast<uint64_t>(blockIdx.x - sum_blocks) * kWaves + wave_of(),
                          static_cast<uint64_t>(gridDim.x - sum_blocks) * kWaves, [&](uint64_t v) { return s.begin[v] == s.begin[v + 1]; });
    }
}

// Sums that reach over the ends of parts.  Over few parts: a wavefront to 512 elements of one; over many: a workgroup, whose wavefronts take its parts in
// turn.  `few_blocks` workgroups take the former.
constexpr uint32_t kJoinWaves = 8, kJoinFewBlocks = 1024, kJoinManyBlocks = 512;
template <class I, bool ADD>
__global__ __launch_bounds__(kWaveSize* kJoinWaves) void embed_join_kernel(const EmbedArgs a, const Sorted s, const uint32_t slabs, const uint32_t few_blocks)
{
    using F = typename I::Wide;
    __shared__ u32x4 joined[kJoinWaves][2][kWaveSize];
    const uint32_t width = static_cast<uint32_t>(a.width), wave = wave_of(), lane = threadIdx.x % kWaveSize;
    auto end_of = [&](uint32_t k, uint32_t which, uint32_t at) {
        return F::wide(F::load(reinterpret_cast<const uint8_t*>(s.ends + (2ull * k + which) * width), at, width));
    };
    // parts from, from + step, ... up to last: their beginnings
    auto sum_of = [&](f32x8 sum, uint32_t from, uint32_t last, uint32_t step, uint32_t at) {
        constexpr uint32_t kAhead = 8;
        for (uint32_t k = from; k <= last; k += kAhead * step) {
            f32x8 x[kAhead];
            static_for<kAhead>([&](auto i) {
                if (k + i * step <= last) x[int(i)] = end_of(k + i * step, 0, at);
            });
            static_for<kAhead>([&](auto i) {
                if (k + i * step <= last) sum += x[int(i)];
            });
        }
        return sum;
    };
    auto put = [&](uint32_t part, f32x8 sum, uint32_t at) {
        const uint32_t id = s.ids[(part + 1) * s.part - 1];
        uint8_t* const out = a.out + static_cast<uint64_t>(id) * a.out_stride * I::kBytes;
        sum *= a.scale;
        if (ADD) sum += I::wide(I::load(out, at, width));
        I::store(out, at, width, I::narrow(sum));
    };
    if (blockIdx.x < few_blocks) {
        const uint64_t total = static_cast<uint64_t>(s.counts[0]) * slabs;
        for (uint64_t w = static_cast<uint64_t>(blockIdx.x) * kJoinWaves + wave; w < total; w += static_cast<uint64_t>(few_blocks) * kJoinWaves) {
            const uint32_t k = static_cast<uint32_t>(w / slabs), at = static_cast<uint32_t>(w - static_cast<uint64_t>(k) * slabs) * kSlab + lane * kLaneItems;
            const uint2 run = s.runs[0][k];
            if (at < width) put(run.x, sum_of(end_of(run.x, 1, at), run.x + 1, run.y, 1, at), at);
        }
        return;
    }
    // (narrow rows: several parts to a wavefront at a time)
    uint32_t lanes = 1;
    while (lanes < kWaveSize && lanes * kLaneItems < width) lanes *= 2;
    const uint32_t turn = lane / lanes, turns = kWaveSize / lanes;
    const uint64_t total = static_cast<uint64_t>(s.counts[1]) * slabs;
    for (uint64_t w = blockIdx.x - few_blocks; w < total; w += gridDim.x - few_blocks) {
        const uint32_t k = static_cast<uint32_t>(w / slabs), at = static_cast<uint32_t>(w - static_cast<uint64_t>(k) * slabs) * kSlab + lane % lanes * kLaneItems;
        const uint2 run = s.runs[1][k];
        f32x8 sum = {};
        if (at < width) sum = sum_of(wave == 0 && turn == 0 ? end_of(run.x, 1, at) : sum, run.x + 1 + wave * turns + turn, run.y, kJoinWaves * turns, at);
        sum = join_turns(sum, lanes);
        const typename F::Held h = F::narrow(sum);
        joined[wave][0][lane] = h.w[0];
        joined[wave][1][lane] = h.w[1];
        __syncthreads();
        if (wave == 0 && turn == 0 && at < width) {
            for (uint32_t i = 1; i < kJoinWaves; i++) sum += F::wide(typename F::Held{{joined[i][0][lane], joined[i][1][lane]}});
            put(run.x, sum, at);
        }
        __syncthreads();
    }
}

// ---- few tokens ---------------------------------------------------------------------------------------

// All of it in one launch: a workgroup takes 512 elements of the rows of a range of ids, and finds and sorts the tokens that ask for
// them in LDS.  A wavefront sums a row's tokens, several at a time where its lanes are more than a row takes; rows of more than kLong are
// summed by all wavefronts together.  Of the range's ids only those that have any are looked at again: 128 tokens added to 32,000 x 4096
// bf16 elements 13.1 us where wavefronts go through all, 7.0 so.
//
// For up to kFewTokens, unless the table is so large that kMostFewBlocks workgroups are too few for it.  (Us, this / sort, sums, join; bf16, words as
// frequent as in text, added: 1000 tokens on 32,000 x 4096 11 / 19, 4096 20 / 29, 4000 on 128,256 x 4096 (2008 workgroups) 26 / 36, x 6144 (3012) 36 / 42, 500
// on 128,256 x 8192 (4016) 32 / 23.  All of 4096 tokens the same word: 80 / 44, what one compute unit reads.)
constexpr uint32_t kFewThreads = 512, kFewWaves = kFewThreads / kWaveSize, kFewTokens = 4096, kFewRounds = kFewTokens / kFewThreads;
constexpr uint32_t kLong = 16, kFewBlocks = 768, kMostFewBlocks = 3200;

// Rows of tokens list[from], list[from + step], ... in front of `to`.
template <class I>
__device__ __forceinline__ f32x8 sum_list(const EmbedArgs& a, const uint16_t* list, uint32_t from, uint32_t to, uint32_t step, uint32_t at)
{
    constexpr uint32_t kAhead = 8;
    f32x8 sum = {};
    for (uint32_t k = from; k < to; k += kAhead * step) {
        typename I::Held h[kAhead];
        static_for<kAhead>([&](auto i) {
            if (k + i * step < to) h[int(i)] = I::load(a.rows + list[k + i * step] * a.rows_stride * I::kBytes, at, static_cast<uint32_t>(a.width));
        });
        static_for<kAhead>([&](auto i) {
            if (k + i * step < to) sum += I::wide(h[int(i)]);
        });
    }
    return sum;
}

template <class I, bool ADD>
__global__ __launch_bounds__(kFewThreads) void embed_few_kernel(const EmbedArgs a, const uint32_t slabs, const uint32_t range_ids)
{
    using F = typename I::Wide;
    __shared__ uint32_t begin[kFewThreads + 1], sums[kFewWaves];
    __shared__ uint16_t token[kFewTokens], bin_of[kFewTokens], order[kFewTokens], wave_bins[kFewWaves][kFewThreads];
    __shared__ u32x4 joined[kFewWaves][2][kWaveSize];
    const uint32_t n = static_cast<uint32_t>(a.n_tokens), vocab = static_cast<uint32_t>(a.vocab), width = static_cast<uint32_t>(a.width);
    const uint32_t wave = wave_of(), lane = threadIdx.x % kWaveSize, block = blockIdx.x / slabs;
    const uint32_t first = block * range_ids, range = vocab - first < range_ids ? vocab - first : range_ids;
    const uint32_t slab = (blockIdx.x - block * slabs) * kSlab, slab_end = width - slab < kSlab ? width : slab + kSlab;
    uint32_t lanes = 1;  // that a row takes
    while (lanes < kWaveSize && lanes * kLaneItems < slab_end - slab) lanes *= 2;
    const uint32_t at = slab + lane % lanes * kLaneItems, turn = lane / lanes, turns = kWaveSize / lanes;
    const bool mine = at < width, puts = mine && turn == 0;
    const uint64_t lower = (1ull << lane) - 1;
    // The whole range is cleared first, while the ids are on their way; sums overwrite it, behind the barriers.
    if (!ADD) {
        clear_rows<I, false>(a.out + static_cast<uint64_t>(first) * a.out_stride * I::kBytes, a.out_stride, range, slab, slab_end, wave, kFewWaves,
                          [](uint64_t) { return true; });
    }
    // the range's tokens in their order
    uint32_t b[kFewRounds], count = 0;
    const uint32_t t0 = wave * (kWaveSize * kFewRounds) + lane;
    static_for<kFewRounds>([&](auto i) {
        const uint32_t t = t0 + i * kWaveSize;
        const uint64_t in = t < n ? static_cast<uint64_t>(a.ids[t]) - first : ~0ull;  // (a negative id is beyond all)
        b[int(i)] = in < range ? static_cast<uint32_t>(in) : kFewThreads;
    });
    static_for<kFewRounds>([&](auto i) { count += __popcll(__ballot(b[int(i)] < kFewThreads)); });
    if (lane == 0) sums[wave] = count;
    begin[threadIdx.x] = 0;
    if (threadIdx.x == 0) begin[kFewThreads] = 0;
    __syncthreads();
    uint32_t place = 0, all = 0;
    for (uint32_t k = 0; k < kFewWaves; k++) {
        if (k < wave) place += sums[k];
        all += sums[k];
    }
    static_for<kFewRounds>([&](auto i) {
        const uint64_t who = __ballot(b[int(i)] < kFewThreads);
        if (b[int(i)] < kFewThreads) {
            const uint32_t k = place + __popcll(who & lower);
            token[k] = static_cast<uint16_t>(t0 + i * kWaveSize);
            bin_of[k] = static_cast<uint16_t>(b[int(i)]);
            atomicAdd(&begin[b[int(i)]], 1u);
        }
        place += __popcll(who);
    });
    __syncthreads();
    // where each id's begin
    {
        uint32_t x = begin[threadIdx.x];
        const uint32_t own = x;
        for (int d = 1; d < kWaveSize; d *= 2) {
            const uint32_t y = __shfl_up(x, d);
            if (lane >= static_cast<uint32_t>(d)) x += y;
        }
        if (lane == kWaveSize - 1) sums[wave] = x;
        __syncthreads();
        for (uint32_t k = 0; k < wave; k++) x += sums[k];
        begin[threadIdx.x] = x - own;
        if (threadIdx.x == kFewThreads - 1) begin[kFewThreads] = x;
    }
    // each behind the last one of its id.  (`begin` moves on to the next id's as the list grows)
    for (uint32_t first_k = 0; first_k < all; first_k += kFewThreads) {
        for (uint32_t i = threadIdx.x; i < kFewWaves * kFewThreads / 2; i += kFewThreads) reinterpret_cast<uint32_t*>(wave_bins)[i] = 0;
        __syncthreads();
        const uint32_t k = first_k + threadIdx.x;
        const bool on = k < all;
        const uint32_t bin = on ? bin_of[k] : 0;
        uint64_t same = __ballot(on);
        for (uint32_t bit = 1; bit < kFewThreads; bit *= 2) {
            const uint64_t set = __ballot(bin & bit);
            same &= bin & bit ? set : ~set;
        }
        if (on && (same & lower) == 0) wave_bins[wave][bin] = static_cast<uint16_t>(__popcll(same));
        __syncthreads();
        if (on) {
            uint32_t to = begin[bin] + __popcll(same & lower);
            for (uint32_t w = 0; w < wave; w++) to += wave_bins[w][bin];
            order[to] = token[k];
        }
        __syncthreads();
        uint32_t more = 0;
        for (uint32_t w = 0; w < kFewWaves; w++) more += wave_bins[w][threadIdx.x];
        begin[threadIdx.x] += more;
        __syncthreads();  // the next round clears what the others read here
    }
    __syncthreads();
    // an id's tokens lie between the end of the one before it and its own
    auto put = [&](uint32_t id, f32x8 sum, const typename I::Held& old) {
        sum *= a.scale;
        if (ADD) sum += I::wide(old);
        I::store(a.out + static_cast<uint64_t>(first + id) * a.out_stride * I::kBytes, at, width, I::narrow(sum));
    };
    auto there = [&](uint32_t id) { return I::load(a.out + static_cast<uint64_t>(first + id) * a.out_stride * I::kBytes, at, width); };
    // ids that have any, and behind kFewThreads those that have more than kLong
    uint32_t some = 0, many = 0;
    {
        const uint32_t of = begin[threadIdx.x] - (threadIdx.x ? begin[threadIdx.x - 1] : 0);
        const uint64_t few = __ballot(of && of <= kLong), more = __ballot(of > kLong);
        if (lane == 0) sums[wave] = __popcll(few) | __popcll(more) << 16;
        __syncthreads();
        uint32_t before = 0;
        for (uint32_t k = 0; k < kFewWaves; k++) {
            if (k < wave) before += sums[k];
            some += sums[k];
        }
        if (of && of <= kLong) bin_of[(before & 0xFFFF) + __popcll(few & lower)] = static_cast<uint16_t>(threadIdx.x);
        if (of > kLong) bin_of[kFewThreads + (before >> 16) + __popcll(more & lower)] = static_cast<uint16_t>(threadIdx.x);
        many = some >> 16;
        some &= 0xFFFF;
        __syncthreads();
    }
    for (uint32_t k = wave; k < some; k += kFewWaves) {
        const uint32_t id = bin_of[k], from = id ? begin[id - 1] : 0, to = begin[id];
        typename I::Held old;
        if (ADD && puts) old = there(id);
        f32x8 sum = {};
        if (mine) sum = sum_list<I>(a, order, from + turn, to, turns, at);
        sum = join_turns(sum, lanes);
        if (puts) put(id, sum, old);
    }
    for (uint32_t k = 0; k < many; k++) {
        const uint32_t id = bin_of[kFewThreads + k], from = id ? begin[id - 1] : 0, to = begin[id];
        f32x8 sum = {};
        if (mine) sum = sum_list<I>(a, order, from + wave * turns + turn, to, kFewWaves * turns, at);
        sum = join_turns(sum, lanes);
        const typename F::Held h = F::narrow(sum);
        joined[wave][0][lane] = h.w[0];
        joined[wave][1][lane] = h.w[1];
        __syncthreads();
        if (wave == 0 && puts) {
            typename I::Held old;
            if (ADD) old = there(id);
            for (uint32_t k = 1; k < kFewWaves; k++) sum += F::wide(typename F::Held{{joined[k][0][lane], joined[k][1][lane]}});
            put(id, sum, old);
        }
        __syncthreads();
    }
}

uint64_t up(uint64_t x) { return (x + 255) / 256 * 256; }

// A new gradient goes past the caches where it and the tokens' rows together are beyond the 256 MiB that lie in front of memory: zeros would drive those
// out.  (Us, through the caches / past them: tables of 32,000 x 4096 bf16 elements, 4096 tokens 60 and 65, 16,384 115 and 83; of 128,256 x 8192, 16,384 tokens
// 475 and 447.)
constexpr uint64_t kPastGradBytes = 320ull << 20;
// Entries of a part: as many as leave work for kPartWaves wavefronts, within limits.
constexpr uint32_t kPartWaves = 8192, kLeastPart = 8, kMostPart = 32;
uint32_t part_of(uint64_t n, uint64_t slabs)
{
    return static_cast<uint32_t>(std::min<uint64_t>(std::max<uint64_t>(n * slabs / kPartWaves, kLeastPart), kMostPart));
}

struct Places {
    uint64_t begin, order, ids, counts, runs, ends, bytes;
};
Places place(uint64_t n, uint64_t vocab, uint64_t width)
{
    Places p = {};
    p.order = up((vocab + 1) * 4);
    p.ids = p.order + up(n * 4);
    p.counts = p.ids + up(n * 4);
    p.runs = p.counts + 256;
    p.ends = p.runs + 2 * up((n / kLeastPart + 1) * sizeof(uint2));
    // (both ends of every part; never less for more tokens or elements, whatever the parts come to)
    const uint64_t parts = (n / kMostPart + 1) * width + std::min<uint64_t>((n / kLeastPart + 1) * width, 2ull * kPartWaves * kSlab);
    p.bytes = p.ends + parts * 2 * 4;
    return p;
}

// Workgroups for so many wavefronts' work, several rounds for each where there is much.
uint32_t groups(uint64_t waves) { return static_cast<uint32_t>(std::max<uint64_t>(1, std::min<uint64_t>((waves + kWaves - 1) / kWaves, 1u << 20))); }

template <class I, bool ADD>
hipError_t launch_grad(const EmbedArgs& a, Sorted s, hipStream_t stream)
{
    const uint32_t slabs = static_cast<uint32_t>((a.width + kSlab - 1) / kSlab);
    if (a.n_tokens <= kFewTokens && (a.vocab + kFewThreads - 1) / kFewThreads * slabs <= kMostFewBlocks) {
        // ranges of 8 to 512 ids, for about kFewBlocks workgroups
        uint32_t range = 8;
        while (range < kFewThreads && (a.vocab + range - 1) / range * slabs > kFewBlocks) range *= 2;
        hipLaunchKernelGGL((embed_few_kernel<I, ADD>), dim3(static_cast<uint32_t>((a.vocab + range - 1) / range * slabs)), dim3(kFewThreads), 0, stream, a,
                           slabs, range);
        return hipGetLastError();
    }
    s.part = part_of(a.n_tokens, slabs);
    const uint64_t n_parts = (a.n_tokens + s.part - 1) / s.part;
    hipLaunchKernelGGL(embed_sort_kernel, dim3(static_cast<uint32_t>((a.vocab + kRange - 1) / kRange)), dim3(kSortThreads), 0, stream, a, s);
    const dim3 threads(kWaveSize * kWaves);
    const uint32_t sum_blocks = groups(n_parts * slabs), rows_at_once = static_cast<uint32_t>(std::max<uint64_t>(kSlab / a.width, 1));
    const bool past = !ADD && (a.n_tokens + a.vocab) * a.width * I::kBytes >= kPastGradBytes;
    const auto sums = past ? embed_sum_kernel<I, ADD, !ADD> : embed_sum_kernel<I, ADD, false>;
    hipLaunchKernelGGL(sums, dim3(sum_blocks + (ADD ? 0 : groups((a.vocab + rows_at_once - 1) / rows_at_once))), threads, 0, stream, a, s, slabs, sum_blocks);
    if (n_parts > 1) {
        const uint32_t few_blocks = static_cast<uint32_t>(std::min<uint64_t>((n_parts * slabs + kJoinWaves - 1) / kJoinWaves, kJoinFewBlocks));
        const uint32_t many_blocks = static_cast<uint32_t>(std::min<uint64_t>(n_parts / kManyParts * slabs, kJoinManyBlocks));
        hipLaunchKernelGGL((embed_join_kernel<I, ADD>), dim3(few_blocks + many_blocks), dim3(kWaveSize * kJoinWaves), 0, stream, a, s, slabs, few_blocks);
    }
    return hipGetLastError();
}

}  // namespace

uint64_t embed_workspace(uint64_t n_tokens, uint64_t vocab, uint64_t width) { return place(n_tokens, vocab, width).bytes; }

hipError_t launch_embed(const EmbedArgs& a, uint32_t dtype, hipStream_t stream)
{
    if (!a.n_tokens) return hipSuccess;
    const uint32_t slabs = static_cast<uint32_t>((a.width + kSlab - 1) / kSlab);
    const dim3 grid(groups(a.n_tokens * slabs)), threads(kWaveSize * kWaves);
    with_items(dtype, a.width, [&](auto items) {
        using I = decltype(items);
        const auto kernel = a.n_tokens * a.width * I::kBytes >= kPastBytes ? embed_kernel<I, true> : embed_kernel<I, false>;
        hipLaunchKernelGGL(kernel, grid, threads, 0, stream, a, slabs);
    });
    return hipGetLastError();
}

hipError_t launch_embed_grad(const EmbedArgs& a, uint32_t dtype, bool add, void* workspace, hipStream_t stream)
{
    if (add && !a.n_tokens) return hipSuccess;
    const Places p = place(a.n_tokens, a.vocab, a.width);
    uint8_t* const w = static_cast<uint8_t*>(workspace);
    const Sorted s = {reinterpret_cast<uint32_t*>(w + p.begin), reinterpret_cast<uint32_t*>(w + p.order), reinterpret_cast<uint32_t*>(w + p.ids),
                      reinterpret_cast<float*>(w + p.ends), 0, reinterpret_cast<uint32_t*>(w + p.counts),
                      {reinterpret_cast<uint2*>(w + p.runs), reinterpret_cast<uint2*>(w + p.runs) + (a.n_tokens / kLeastPart + 1)}};
    hipError_t err = hipSuccess;
    with_items(dtype, a.width, [&](auto items) {
        using I = decltype(items);
        err = add ? launch_grad<I, true>(a, s, stream) : launch_grad<I, false>(a, s, stream);
    });
    return err;
}

}  // namespace ffsnap
