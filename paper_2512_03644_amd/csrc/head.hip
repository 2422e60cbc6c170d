// Cross entropy over a large vocabulary from hidden states, and its gradients, for gfx950.
//
// z = H W^T is made in tiles of 256 vocabulary entries: a tile leaves, for each token, its largest logit and the sum of
// exponentials against it, and the target's logit.  Joined over the tiles these give the log-probability.  For the
// gradients the vocabulary is taken in pieces, of up to 2^29 logits.  A piece's logits become G = (softmax - [target]) * weight in
// 16 bits, and two products take G: dH += G W, in 32 bits over the pieces, and dW = G^T H.  The last piece, with which they
// begin, is still there from the first time (kKeep); the others' logits are made once more: three products of 2 * tokens * vocab *
// width operations for the last piece, four for the others.  What is kept goes by the card's 288 GB, of which 3 GiB are one hundredth.  (Pieces
// of 2^25 / 2^26 / 2^27 / 2^28 / 2^29 / 2^30 logits: 4096 tokens, a tenth of them masked, 8192 x 128,256 25.2 / 24.7 / 23.3 / 21.7 /
// 18.7 / 18.8 ms, 4096 x 32,000, which lies in one from 2^27 on, 3.20 / 3.10 / 2.70 / 2.70 / 2.62 / 2.64.)
//
// G is rounded to 16 bits, for the matrix instructions; nothing else is, in front of the outputs.  Weights are divided
// by the largest one first, so that tokens of equal weight have exact factors of 1 (a factor rounded with G would
// be the same error in every token); it comes back, with the loss scale, on 32-bit sums.  For fp16, G is 2^14 times that: a
// softmax of 2^-28 is still a normal number.
//
// What bounds it: many tokens, the matrix instructions (product.h); few, reading W once for the logits and once for dH, and writing dW: 64 tokens and
// fewer take kernels of their own for the logits (head_stream_kernel) and dW (head_few_dweight_kernel); small heads, five
// kernels one behind the other on few compute units.  Us, scoring / with both gradients, width 4096, 1 / 16 / 64 / 128 / 256 tokens on 32,000 (which lie in the caches from the call before, in part) 52 / 71 /
// 70 / 84 / 109 and 158 / 177 / 202 / 240 / 322, on 128,256 216 / 266 / 249 / 276 / 286 and 661 / 723 / 721 / 888 / 1053.
#include "head.hpp"

#include <algorithm>

#include "product.h"
#include "xcd_order.h"

namespace ffsnap {

namespace {

constexpr uint32_t kTile = 256;        // vocabulary entries of a tile
constexpr uint32_t kFewTokens = 64;    // up to so many, G is made of the whole vocabulary at once
constexpr uint32_t kComputeUnits = 256;
constexpr float kLog2E = 0x1.715476p+0f;

constexpr uint64_t up(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

// A token that counts, by its place among those.
struct Row {
    float lse2;    // log2(sum of exp(logits))
    float factor;  // of its gradient
    float target;  // gradient at the target
    int32_t y;     // the target
};

// Known on the device alone.
struct State {
    uint32_t used, invalid;  // tokens that count; tokens with a weight but no target
    float largest;           // weight of those that count
    float scale;             // of the gradients: what G has been divided by
    uint32_t done;           // rows whose loss is known, of few
};

struct HeadArgs {
    ff_head_batch b;
    float* logp;
    uint8_t *dhidden, *dweight;
    uint64_t dhidden_stride, dweight_stride;
    ff_head_stats* stats;
    // the workspace
    State* state;
    uint32_t* index;    // of the tokens that count, in their order
    float* weights;     // theirs
    int32_t* targets;
    Row* rows;
    double* losses;     // of each of them, times its weight
    float* picked;      // logit of the target
    float2* parts;      // [token][tile]: largest logit times log2(e), sum of exponentials against it
    uint8_t* hidden;    // packed rows of those tokens: `stride` bytes, zeros behind the width and behind the last up to 64 rows
    uint8_t* weight;    // packed rows of a piece, if W's own do not lie as the loads want them; or null
    uint8_t* grad;      // G of a piece: [tokens up to a tile][piece]
    float* logits;      // [token][piece]: of the last piece, if they are kept
    float* dh;          // [slice][token][width up to 64]: dH so far
    uint32_t tokens_up; // tokens, up to a whole tile
    uint32_t tiles;     // of the vocabulary: parts of a token's sums
    uint32_t stride;    // bytes of a packed row
    uint32_t piece;     // vocabulary entries that G has, a multiple of 256
    uint32_t step;      // and that the gradients' products take at once
    uint32_t slices;    // of dH's sum over a piece
    uint32_t splits;    // of the logits' sums, of few tiles
    float* dw;          // [slice][piece][width up to 64]: dW so far, of few tiles
    uint32_t dw_slices; // of dW's sum over the tokens
    float grad_scale;   // loss scale, and what G is too large by
    uint32_t past;      // dW's rows are whole pieces of 16 bytes
};

__device__ __forceinline__ OperandTile hidden_tile(const HeadArgs& A, uint32_t m0, uint32_t used)
{
    return {A.hidden + static_cast<uint64_t>(m0) * A.stride, A.stride, used - m0, A.stride / 2};
}
// Rows [v0, ...) of W; `first` is the piece's.
__device__ __forceinline__ const uint8_t* weight_row(const HeadArgs& A, uint32_t first, uint32_t v0, uint64_t* stride)
{
    if (A.weight) {
        *stride = A.stride;
        return A.weight + static_cast<uint64_t>(v0 - first) * A.stride;
    }
    *stride = A.b.weight_stride * 2;
    return static_cast<const uint8_t*>(A.b.weight) + v0 * *stride;
}

// ---- which tokens count ---------------------------------------------------------------------------

// In their order, by a whole workgroup: index[k] of the k-th; the workgroup that writes leaves what is known of them in the workspace.
template <int THREADS>
__device__ __forceinline__ uint32_t select(const HeadArgs& A, uint32_t* index, bool writes)
{
    __shared__ uint32_t count[THREADS / kWaveSize];
    __shared__ float largest[THREADS / kWaveSize];
    const uint32_t n = static_cast<uint32_t>(A.b.n_tokens), wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    uint32_t used = 0, invalid = 0;
    float most = 0.f;
    for (uint64_t first = 0; first < n; first += THREADS) {
        const uint64_t t = first + threadIdx.x;
        const float w = t < n ? A.b.weights[t] : 0.f;
        const int64_t y = t < n ? A.b.targets[t] : -1;
        const bool wanted = !(w == 0.f), inside = y >= 0 && static_cast<uint64_t>(y) < A.b.vocab, mine = wanted && inside;
        const uint64_t who = __ballot(mine);
        if (lane == 0) count[wave] = __popcll(who);
        __syncthreads();
        uint32_t at = used + __popcll(who & ((1ull << lane) - 1)), all = 0;
        for (uint32_t k = 0; k < THREADS / kWaveSize; k++) {
            if (k < wave) at += count[k];
            all += count[k];
        }
        if (mine) index[at] = static_cast<uint32_t>(t);
        if (mine && writes) {
            A.index[at] = static_cast<uint32_t>(t);
            A.weights[at] = w;
            A.targets[at] = static_cast<int32_t>(y);
            if (__builtin_isfinite(w)) most = fmaxf(most, fabsf(w));
        }
        if (!mine && writes && t < n) A.logp[t] = 0.f;
        used += all;
        invalid += __syncthreads_count(wanted && !inside);
    }
    if (writes) {
        for (int d = 32; d; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
        if (lane == 0) largest[wave] = most;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (uint32_t k = 0; k < THREADS / kWaveSize; k++) most = fmaxf(most, largest[k]);
            *A.state = {used, invalid, most, most * A.grad_scale, 0};
        }
    }
    return used;
}

// One workgroup: a few thousand tokens are a few rounds.
constexpr int kSelectThreads = 1024;
__global__ __launch_bounds__(kSelectThreads) void head_select_kernel(const HeadArgs A) { select<kSelectThreads>(A, A.index, true); }

// Elements [at, at + 8) of a row of `width`, zeros behind it.
__device__ __forceinline__ u32x4 load8(const uint8_t* row, uint32_t at, uint32_t width)
{
    if (at + 8 <= width) return *(const FF_GLOBAL u32x4_a2*)(row + 2ull * at);
    uint32_t x[8] = {};
    for (uint32_t k = 0; k < 8; k++)
        if (at + k < width) x[k] = as_global(reinterpret_cast<const uint16_t*>(row))[at + k];
    return u32x4{x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
}

// `width` elements of a row to a packed one of `bytes`; elements behind them are zeros.
__device__ __forceinline__ void copy_row(uint8_t* to, uint32_t bytes, const uint8_t* from, uint32_t width)
{
    for (uint32_t i = threadIdx.x; i < bytes / 16; i += blockDim.x) *(FF_GLOBAL u32x4*)(to + 16ull * i) = load8(from, i * 8, width);
}

// Hidden states of the tokens that count, one behind the other, and zeros up to 64 rows; gradients of the other tokens.
__device__ __forceinline__ void gather(const HeadArgs& A, const uint32_t used, const uint32_t* index, const uint32_t blocks)
{
    const uint32_t until = (used + 63) / 64 * 64, n = static_cast<uint32_t>(A.b.n_tokens);
    for (uint32_t r = blockIdx.x; r < until; r += blocks) {
        const uint64_t t = r < used ? index[r] : 0;
        copy_row(A.hidden + static_cast<uint64_t>(r) * A.stride, A.stride,
                 static_cast<const uint8_t*>(A.b.hidden) + t * A.b.hidden_stride * 2, r < used ? static_cast<uint32_t>(A.b.width) : 0);
    }
    if (!A.dhidden) return;
    for (uint64_t t = blockIdx.x; t < n; t += blocks) {
        const float w = A.b.weights[t];
        const int64_t y = A.b.targets[t];
        if (!(w == 0.f) && y >= 0 && static_cast<uint64_t>(y) < A.b.vocab) continue;
        uint16_t* const to = reinterpret_cast<uint16_t*>(A.dhidden + t * A.dhidden_stride * 2);
        for (uint32_t i = threadIdx.x; i < A.b.width; i += blockDim.x) as_global(to)[i] = 0;
    }
}
__global__ __launch_bounds__(256) void head_gather_kernel(const HeadArgs A) { gather(A, A.state->used, A.index, gridDim.x); }

// Rows [first, first + n) of W, packed, by `blocks` workgroups.
__device__ __forceinline__ void pack(const HeadArgs& A, const uint32_t first, const uint32_t n, const uint32_t block, const uint32_t blocks)
{
    for (uint32_t r = block; r < n; r += blocks)
        copy_row(A.weight + static_cast<uint64_t>(r) * A.stride, A.stride,
                 static_cast<const uint8_t*>(A.b.weight) + (static_cast<uint64_t>(first) + r) * A.b.weight_stride * 2, static_cast<uint32_t>(A.b.width));
}
constexpr uint32_t kPackBlocks = 8192;
__global__ __launch_bounds__(256) void head_pack_kernel(const HeadArgs A, const uint32_t first, const uint32_t n) { pack(A, first, n, blockIdx.x, gridDim.x); }

// Tokens and hidden states in one launch, where every workgroup can look at all tokens by itself; the workgroups behind the first `blocks` pack the
// first n rows of W.
constexpr uint32_t kSelectFew = 1024;
__global__ __launch_bounds__(256) void head_few_kernel(const HeadArgs A, const uint32_t blocks, const uint32_t n)
{
    if (blockIdx.x >= blocks) {
        pack(A, 0, n, blockIdx.x - blocks, gridDim.x - blocks);
        return;
    }
    __shared__ uint32_t index[kSelectFew];
    const uint32_t used = select<256>(A, index, blockIdx.x == 0);
    __syncthreads();
    gather(A, used, index, blocks);
}

// An element of G.
__device__ __forceinline__ float gradient(float z, uint32_t v, uint32_t vocab, const Row& r)
{
    const float p = __builtin_amdgcn_exp2f(fmaf(z, kLog2E, -r.lse2)) * r.factor;
    return v >= vocab ? 0.f : static_cast<int32_t>(v) == r.y ? r.target : p;
}

// ---- logits ---------------------------------------------------------------------------------------

// For a token's N logits of each of the four lanes that have its row, entries of the vocabulary v + 16 j + e: the target's logit is put down,
// those behind the vocabulary are left out, and the largest, times log2(e), and the sum of exponentials against it come back to all four.
template <int N>
__device__ __forceinline__ float2 join_lanes(const HeadArgs& A, f32x4 (&z)[N], const uint32_t t, const uint32_t v, const int32_t y)
{
    const uint32_t vocab = static_cast<uint32_t>(A.b.vocab), in = static_cast<uint32_t>(y) - v;
    if (__any(in < 16 * N)) {  // (the target is in few of the tiles)
#pragma unroll
        for (int j = 0; j < N; j++)
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (in == 16u * j + e) A.picked[t] = z[j][e];
    }
    if (__any(v + 16 * N > vocab)) {
#pragma unroll
        for (int j = 0; j < N; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) z[j][e] = v + 16 * j + e < vocab ? z[j][e] : -INFINITY;
    }
    // (a NaN or +inf stays in the sum, as exp(NaN - top) or exp(inf - inf))
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int j = 0; j < N; j++) top = fmaxf(fmaxf(top, fmaxf(z[j][0], z[j][1])), fmaxf(z[j][2], z[j][3]));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    // Terms are 2^(z log2(e) - c), c = top log2(e) in 24 bits: one operation in front of the exponential, and c stands for the part from here on.
    const float c = top * kLog2E, against = top == -INFINITY ? 0.f : c;
#pragma unroll
    for (int j = 0; j < N; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) total += __builtin_amdgcn_exp2f(fmaf(z[j][e], kLog2E, -against));
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    return {c, total};
}
// Parts of several wavefronts.
template <int N>
__device__ __forceinline__ float2 join_parts(const float2 (&p)[N])
{
    float c = -INFINITY, total = 0.f;
#pragma unroll
    for (int k = 0; k < N; k++) c = fmaxf(c, p[k].x);
    const float against = c == -INFINITY ? 0.f : c;
#pragma unroll
    for (int k = 0; k < N; k++) total += p[k].y * __builtin_amdgcn_exp2f(p[k].x - against);
    return {c, total};
}

// The tiles of vocabulary entries [first, first + n): their parts of the sums, with kKeep the logits as well; or G.
// kSplit: nothing but a slice of their sums.
enum Mode { kSums, kKeep, kGrad, kSplit };
template <bool BF16, int BM, Mode MODE>
__global__ __launch_bounds__(kProductThreads) __attribute__((amdgpu_waves_per_eu(2))) void head_logits_kernel(const HeadArgs A, const uint32_t first,
                                                                                                             const uint32_t n)
{
    using S = Share<BM>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kProductLds<BM, kAlongK, kAlongK>];
    const uint32_t used = A.state->used;
    uint32_t m0, n0;
    const uint32_t tiles = gridDim.x / (MODE == kSplit ? A.splits : 1), slice = MODE == kSplit ? blockIdx.x / tiles : 0;
    tile_at(xcd_order(blockIdx.x - slice * tiles, tiles, kXcdTiles), A.tokens_up / BM, (n + kTile - 1) / kTile, &m0, &n0);
    m0 *= BM;
    n0 *= kTile;
    if (m0 >= used) return;
    const uint32_t v0 = first + n0, vocab = static_cast<uint32_t>(A.b.vocab);
    OperandTile b;
    b.base = weight_row(A, first, v0, &b.stride);
    b.valid = n - n0;
    b.k_valid = A.weight ? A.stride / 2 : static_cast<uint32_t>(A.b.width);
    const uint32_t steps = A.stride / (2 * kStepK), from = MODE == kSplit ? steps * slice / A.splits : 0;
    f32x4 z[S::kM][S::kN];
    product<BF16, BM, kAlongK, kAlongK>(hidden_tile(A, m0, used), b, from, MODE == kSplit ? steps * (slice + 1) / A.splits : steps, b.k_valid % kStepK ? steps - 1 : ~0u, (FF_LDS uint8_t*)lds, z);
    const int wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    const uint32_t m = m0 + (wave / S::kAcross) * (16 * S::kM) + lane % 16;                    // + 16 i
    const uint32_t v = v0 + (wave % S::kAcross) * (16 * S::kN) + 4 * (lane / 16);              // + 16 j + e
    if constexpr (MODE == kSplit) {
        static_for<S::kM>([&](auto i) {
            const uint32_t t = m + 16 * i;
            float* const out = A.logits + (static_cast<uint64_t>(slice) * A.tokens_up + t) * A.piece + v;
            static_for<S::kN>([&](auto j) {
                if (t < used) *(FF_GLOBAL f32x4*)(out + 16 * j) = z[int(i)][int(j)];
            });
        });
    } else if constexpr (MODE == kGrad) {
        const uint32_t row0 = m - lane % 16, at = v - 4 * (lane / 16) - first;
        Row rows[S::kM];
        static_for<S::kM>([&](auto i) {
            rows[int(i)] = {0.f, 0.f, 0.f, -1};
            if (m + 16 * i < used) rows[int(i)] = A.rows[m + 16 * i];
        });
        RowsByLds<S::kM, S::kN>::pass(
            (FF_LDS uint8_t*)lds,
            [&](auto i, auto j) {
                f32x4 g;
                static_for<4>([&](auto e) {
                    const float x = gradient(z[int(i)][int(j)][int(e)], v + 16 * j + e, vocab, rows[int(i)]);
                    g[int(e)] = m + 16 * i < used ? x : 0.f;
                });
                return to_half<BF16>(g);
            },
            [&](uint32_t row, uint32_t column, u32x4 x) {
                *(FF_GLOBAL u32x4*)(A.grad + (static_cast<uint64_t>(row0 + row) * A.piece + at + column) * 2) = x;
            });
    } else {
        __shared__ float2 part[BM][S::kAcross];
        const uint32_t kept_from = A.piece < vocab ? first : 0;  // of few tokens all are kept
        static_for<S::kM>([&](auto i) {
            const uint32_t t = m + 16 * i;
            const int32_t y = t < used ? A.targets[t] : -1;
            if constexpr (MODE == kKeep) {
                float* const out = A.logits + static_cast<uint64_t>(t) * A.piece + (v - kept_from);
                static_for<S::kN>([&](auto j) {
                    if (t < used) *(FF_GLOBAL f32x4*)(out + 16 * j) = z[int(i)][int(j)];
                });
            }
            const float2 p = join_lanes(A, z[int(i)], t, v, y);
            if (lane < 16) part[(wave / S::kAcross) * (16 * S::kM) + 16 * i + lane][wave % S::kAcross] = p;
        });
        __syncthreads();
        for (uint32_t r = threadIdx.x; r < BM && m0 + r < used; r += kProductThreads)
            A.parts[static_cast<uint64_t>(m0 + r) * A.tiles + v0 / kTile] = join_parts(part[r]);
    }
}

// The logits of few tokens, all of the vocabulary: W passes once from memory through registers, rows of any alignment where they lie.  A
// wavefront takes 16 V rows of it and 16 T tokens, whose hidden states come from the caches; the products of a chunk of K times 32 elements
// are made while the next one is on its way.  What bounds it: reading W; of 17 tokens and more hidden states as well, and 64 x 256
// tiles are better, also where rows have to be copied for them, but for up to 32 tokens that are only scored.  (Us, scoring, this / tiles: 1
// token on 32,000 x 4096 64 / 89, 17 80 / 92, 32 88 / 93, 64 114 / 102, on 128,256 x 4096 17 266 / 242; copied for tiles, 22 tokens on 67,725 x 1491 108 / 154, 51 on
// 10,863 x 2651 87 / 61; with both gradients, which have rows copied anyway, 2 tokens on 49,835 x 2189 360 / 307.)
constexpr int kStreamThreads = 256, kStreamWaves = kStreamThreads / kWaveSize;
template <int T>
struct Stream {
    static constexpr int V = T, K = 8 / T;
    static constexpr uint32_t kEntries = 16 * V * kStreamWaves;  // of a workgroup
};
template <bool BF16, int T, Mode MODE>
__global__ __launch_bounds__(kStreamThreads) void head_stream_kernel(const HeadArgs A)
{
    using S = Stream<T>;
    const uint32_t used = A.state->used, width = static_cast<uint32_t>(A.b.width), vocab = static_cast<uint32_t>(A.b.vocab);
    const uint32_t wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    const uint32_t v0 = blockIdx.x * S::kEntries + wave * (16 * S::V);
    if (used == 0) return;
    const uint8_t *w[S::V], *h[T];
    static_for<S::V>([&](auto j) {
        const uint32_t v = v0 + 16 * j + lane % 16;
        w[int(j)] = static_cast<const uint8_t*>(A.b.weight) + (v < vocab ? v : vocab - 1) * A.b.weight_stride * 2;
    });
    static_for<T>([&](auto i) {
        const uint32_t t = 16 * i + lane % 16;
        h[int(i)] = A.hidden + static_cast<uint64_t>(t < used ? t : used - 1) * A.stride;
    });
    struct Chunk {
        s16x8 w[S::K][S::V], h[S::K][T];
    };
    const uint32_t steps = (width + 31) / 32, chunks = (steps + S::K - 1) / S::K, whole = width / (32 * S::K);
    auto fetch = [&](Chunk& c, uint32_t k) {
        static_for<S::K>([&](auto s) {
            const uint32_t at = (k * S::K + s) * 32 + lane / 16 * 8;
            static_for<S::V>([&](auto j) {
                if (k < whole) c.w[int(s)][int(j)] = __builtin_bit_cast(s16x8, *(const FF_GLOBAL u32x4_a2*)(w[int(j)] + 2 * at));
                else c.w[int(s)][int(j)] = __builtin_bit_cast(s16x8, load8(w[int(j)], at, width));
            });
            static_for<T>([&](auto i) {  // (zeros up to 64 elements)
                const s16x8 none = {};
                c.h[int(s)][int(i)] = at < A.stride / 2 ? *(const FF_GLOBAL s16x8*)(h[int(i)] + 2 * at) : none;
            });
        });
    };
    f32x4 z[T][S::V];
    static_for<T>([&](auto i) { static_for<S::V>([&](auto j) { z[int(i)][int(j)] = f32x4{0, 0, 0, 0}; }); });
    auto multiply_all = [&](const Chunk& c) {
        static_for<S::K>([&](auto s) {
            static_for<T>([&](auto i) {
                static_for<S::V>([&](auto j) { z[int(i)][int(j)] = multiply<BF16>(c.w[int(s)][int(j)], c.h[int(s)][int(i)], z[int(i)][int(j)]); });
            });
        });
    };
    Chunk one, other;
    fetch(one, 0);
    for (uint32_t k = 0; k < chunks; k += 2) {
        if (k + 1 < chunks) fetch(other, k + 1);
        multiply_all(one);
        if (k + 2 < chunks) fetch(one, k + 2);
        if (k + 1 < chunks) multiply_all(other);
    }
    __shared__ float2 part[16 * T][kStreamWaves];
    const uint32_t v = v0 + 4 * (lane / 16);
    static_for<T>([&](auto i) {
        const uint32_t t = 16 * i + lane % 16;
        if constexpr (MODE == kKeep) {
            static_for<S::V>([&](auto j) {
                if (t < used && v + 16 * j < A.piece) *(FF_GLOBAL f32x4*)(A.logits + static_cast<uint64_t>(t) * A.piece + v + 16 * j) = z[int(i)][int(j)];
            });
        }
        const float2 p = join_lanes(A, z[int(i)], t, v, t < used ? A.targets[t] : -1);
        if (lane < 16) part[16 * i + lane][wave] = p;
    });
    __syncthreads();
    if (threadIdx.x < used) A.parts[static_cast<uint64_t>(threadIdx.x) * A.tiles + blockIdx.x] = join_parts(part[threadIdx.x]);
}

// ---- log-probabilities, G of kept logits ------------------------------------------------------------

// The loss, from every row's in an order that their number gives, by a wavefront.
__device__ __forceinline__ void put_stats(const HeadArgs& A, double loss, const uint32_t used)
{
    A.stats->loss = static_cast<float>(loss);
    A.stats->reserved = 0;
    A.stats->n_tokens = used;
    A.stats->n_invalid = A.state->invalid;
}

constexpr uint32_t kCountFew = 256;
// What is known of row r from its sum of exponentials `total` against c and its target's logit.  The wavefront that writes leaves the results; of few rows
// (kCountFew: they count one another at one address, 10 ns each) the last one to do so adds their losses up, of others a launch.
template <bool BF16>
__device__ __forceinline__ Row outcome(const HeadArgs& A, const uint32_t r, const uint32_t used, const float c, const double total, const float picked, const bool writes)
{
    const uint32_t lane = threadIdx.x % kWaveSize;
    const double against = static_cast<double>(c) / static_cast<double>(kLog2E), rest = log(total);
    const double logp = (static_cast<double>(picked) - against) - rest;
    const float w = A.weights[r], f = w / A.state->largest * (BF16 ? 1.f : 0x1p14f);
    const Row row = {static_cast<float>((against + rest) * 1.4426950408889634), f, f * static_cast<float>(expm1(logp)), A.targets[r]};
    if (writes && lane == 0) {
        A.logp[A.index[r]] = static_cast<float>(logp);
        A.rows[r] = row;
        __hip_atomic_store(A.losses + r, -static_cast<double>(w) * logp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (writes && A.b.n_tokens <= kCountFew) {
        bool last = false;
        if (lane == 0) {
            // (the loss has arrived when the store is done; a release would write the caches back)
            asm volatile("" ::: "memory");
            wait_loads<0>();
            last = __hip_atomic_fetch_add(&A.state->done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == used;
        }
        if (__any(last)) {
            double s = 0;
            for (uint32_t k = lane; k < used; k += kWaveSize) s += __hip_atomic_load(A.losses + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            for (int d = 32; d; d /= 2) s += __shfl_xor(s, d);
            if (lane == 0) put_stats(A, s, used);
        }
    }
    return row;
}

// A wavefront joins the tiles' parts of row r, in 64 bits from the exponentials on.
template <bool BF16>
__device__ __forceinline__ Row finish(const HeadArgs& A, const uint32_t r, const uint32_t used, const bool writes)
{
    const uint32_t lane = threadIdx.x % kWaveSize;
    const float2* const parts = A.parts + static_cast<uint64_t>(r) * A.tiles;
    // fn(part), several on their way at once
    auto each_part = [&](auto&& fn) {
        constexpr uint32_t kAhead = 8;
        for (uint32_t k = lane; k < A.tiles; k += kAhead * kWaveSize) {
            float2 p[kAhead];
            static_for<kAhead>([&](auto i) { p[int(i)] = k + i * kWaveSize < A.tiles ? parts[k + i * kWaveSize] : float2{-INFINITY, 0.f}; });
            static_for<kAhead>([&](auto i) { fn(p[int(i)]); });
        }
    };
    float c = -INFINITY;
    each_part([&](float2 p) { c = fmaxf(c, p.x); });
    for (int d = 32; d; d /= 2) c = fmaxf(c, __shfl_xor(c, d));
    if (c == -INFINITY) c = 0.f;
    double total = 0;
    each_part([&](float2 p) {
        if (p.y != 0.f) total += static_cast<double>(p.y) * exp2(static_cast<double>(p.x) - static_cast<double>(c));
    });
    for (int d = 32; d; d /= 2) total += __shfl_xor(total, d);
    return outcome<BF16>(A, r, used, c, total, A.picked[r], writes);
}

// A wavefront to a row.
template <bool BF16>
__global__ __launch_bounds__(256) void head_finish_kernel(const HeadArgs A)
{
    const uint32_t used = A.state->used, r = blockIdx.x * (256 / kWaveSize) + threadIdx.x / kWaveSize;
    if (r < used) finish<BF16>(A, r, used, true);
    if (used == 0 && r == 0 && threadIdx.x == 0) put_stats(A, 0.0, 0);
}

// The same, and G of vocabulary entries [first, first + n), whose logits were kept; rows of zeros up to 64.
template <bool BF16>
__global__ __launch_bounds__(256) void head_kept_kernel(const HeadArgs A, const uint32_t first, const uint32_t n, const uint32_t wide)
{
    const uint32_t used = A.state->used, vocab = static_cast<uint32_t>(A.b.vocab), until = (used + 63) / 64 * 64;
    const uint32_t t = blockIdx.x / wide, part = blockIdx.x - t * wide;  // of `wide` parts of a row
    if (used == 0 && blockIdx.x == 0 && threadIdx.x == 0) put_stats(A, 0.0, 0);
    if (t >= until) return;
    __shared__ Row row;
    if (t < used && threadIdx.x < kWaveSize) {
        const Row known = finish<BF16>(A, t, used, part == 0);
        if (threadIdx.x == 0) row = known;
    }
    __syncthreads();
    const Row r = row;
    const uint32_t end = (n + kTile - 1) / kTile * kTile;
    for (uint32_t at = (part * 256 + threadIdx.x) * 8; at < end; at += wide * 2048) {
        u32x4 out = {0, 0, 0, 0};
        if (t < used) {
            const FF_GLOBAL f32x4* const z = (const FF_GLOBAL f32x4*)(A.logits + static_cast<uint64_t>(t) * A.piece + at);
            f32x4 g[2] = {z[0], z[1]};
            for (int k = 0; k < 2; k++)
                for (int e = 0; e < 4; e++) g[k][e] = gradient(g[k][e], first + at + 4 * k + e, vocab, r);
            const u32x2 a = to_half<BF16>(g[0]), b = to_half<BF16>(g[1]);
            out = u32x4{a.x, a.y, b.x, b.y};
        }
        *(FF_GLOBAL u32x4*)(A.grad + (static_cast<uint64_t>(t) * A.piece + at) * 2) = out;
    }
}

// Both, and the sums of the logits' slices before, for a row of few tiles: a workgroup.  A thread's elements are its own from one pass to the next.  What bounds
// it: three passes over the caches, one behind the other.
template <bool BF16>
__global__ __launch_bounds__(256) void head_row_kernel(const HeadArgs A, const bool grad)
{
    __shared__ float top[256 / kWaveSize], target;
    __shared__ double sum[256 / kWaveSize];
    __shared__ Row row;
    const uint32_t used = A.state->used, vocab = static_cast<uint32_t>(A.b.vocab), t = blockIdx.x, wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    if (used == 0 && t == 0 && threadIdx.x == 0) put_stats(A, 0.0, 0);
    if (t >= (grad ? (used + 63) / 64 * 64 : used)) return;
    float* const z = A.logits + static_cast<uint64_t>(t) * A.piece;
    auto each = [&](auto&& fn) {
        for (uint32_t v = threadIdx.x * 4; v < A.piece; v += 256 * 4) fn(v);
    };
    if (t < used) {
        const uint64_t step = static_cast<uint64_t>(A.tokens_up) * A.piece;
        const uint32_t y = static_cast<uint32_t>(A.targets[t]);
        float most = -INFINITY;
        each([&](uint32_t v) {
            constexpr uint32_t kAhead = 8;
            f32x4 s = {0, 0, 0, 0};
            for (uint32_t k = 0; k < A.splits; k += kAhead) {
                f32x4 x[kAhead];
                static_for<kAhead>([&](auto i) { x[int(i)] = *(const FF_GLOBAL f32x4*)(z + v + (k + i < A.splits ? k + i : k) * step); });
                static_for<kAhead>([&](auto i) {
                    if (k + i < A.splits) s += x[int(i)];
                });
            }
            for (int e = 0; e < 4; e++) {
                if (v + e == y) target = s[e];
                s[e] = v + e < vocab ? s[e] : -INFINITY;
                most = fmaxf(most, s[e]);
            }
            *(FF_GLOBAL f32x4*)(z + v) = s;
        });
        for (int d = 32; d; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
        if (lane == 0) top[wave] = most;
        __syncthreads();
        most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        const float c = most == -INFINITY ? 0.f : most * kLog2E;
        double total = 0;
        each([&](uint32_t v) {
            const f32x4 x = *(const FF_GLOBAL f32x4*)(z + v);
            float s = 0;
            for (int e = 0; e < 4; e++) s += __builtin_amdgcn_exp2f(fmaf(x[e], kLog2E, -c));
            total += static_cast<double>(s);
        });
        for (int d = 32; d; d /= 2) total += __shfl_xor(total, d);
        if (lane == 0) sum[wave] = total;
        __syncthreads();
        if (wave == 0) {
            const Row known = outcome<BF16>(A, t, used, c, (sum[0] + sum[1]) + (sum[2] + sum[3]), target, true);
            if (lane == 0) row = known;
        }
        if (!grad) return;
        __syncthreads();
    }
    const Row r = row;
    each([&](uint32_t v) {
        f32x4 g = {0, 0, 0, 0};
        if (t < used) {
            g = *(const FF_GLOBAL f32x4*)(z + v);
            for (int e = 0; e < 4; e++) g[e] = gradient(g[e], v + e, vocab, r);
        }
        *(FF_GLOBAL u32x2*)(A.grad + (static_cast<uint64_t>(t) * A.piece + v) * 2) = to_half<BF16>(g);
    });
}

// The loss of many rows.
__global__ __launch_bounds__(kSelectThreads) void head_sum_kernel(const HeadArgs A)
{
    __shared__ double sum[kSelectThreads];
    const uint32_t used = A.state->used;
    double s = 0;
    for (uint64_t r = threadIdx.x; r < used; r += kSelectThreads) s += A.losses[r];
    sum[threadIdx.x] = s;
    __syncthreads();
    for (int d = kSelectThreads / 2; d; d /= 2) {
        if (static_cast<int>(threadIdx.x) < d) sum[threadIdx.x] += sum[threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x == 0) put_stats(A, sum[0], used);
}

// ---- gradients ------------------------------------------------------------------------------------

// Elements [at, at + 8) of a row of `width`, at < width.
__device__ __forceinline__ void put8(uint8_t* row, uint32_t at, uint32_t width, u32x4 v)
{
    uint8_t* const p = row + 2ull * at;
    if (at + 8 <= width) {
        *(FF_GLOBAL u32x4_a2*)p = v;
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 7; e++)
            if (at + e < width) as_global(reinterpret_cast<uint16_t*>(p))[e] = static_cast<uint16_t>(v[e / 2] >> e % 2 * 16);
    }
}

// The same, past the caches: a gradient of W is far larger than they are.  (Us, plain / so: dW of 1, 64, 128 tokens on 128,256 x 4096, with all in front of
// it, 505, 565, 699 and 483, 527, 590.)  Not where rows begin between 16-byte steps: pieces of lines would go to memory one by one (2 tokens on 49,835 x 2189,
// dW 168 us past the caches, 60 through them).
__device__ __forceinline__ void put8_past(bool past, uint8_t* row, uint32_t at, uint32_t width, u32x4 v)
{
    if (past && at + 8 <= width) __builtin_nontemporal_store(v, (FF_GLOBAL u32x4_a2*)(row + 2ull * at));
    else put8(row, at, width, v);
}

// dH (+)= G W over a slice of vocabulary entries [first, first + n), which begin at a column of G; where that is all of it, in its place.
enum Sum { kOnly, kFirst, kNext };
template <bool BF16, int BM>
__device__ __forceinline__ void dhidden(const HeadArgs& A, const uint32_t first, const uint32_t n, const uint32_t column, const Sum which,
                                        const uint32_t block, const uint32_t blocks, FF_LDS uint8_t* lds)
{
    using S = Share<BM>;
    const uint32_t used = A.state->used, width_up = A.stride / 2;
    const uint32_t tiles_m = A.tokens_up / BM, tiles_n = (width_up + kTile - 1) / kTile;
    const uint32_t tile = xcd_order(block, blocks, kXcdTiles), slice = tile / (tiles_m * tiles_n);
    uint32_t m0, n0;
    tile_at(tile - slice * (tiles_m * tiles_n), tiles_m, tiles_n, &m0, &n0);
    m0 *= BM;
    n0 *= kTile;
    if (m0 >= used) return;
    const uint32_t steps = (n + kStepK - 1) / kStepK, each = (steps + A.slices - 1) / A.slices;
    const uint32_t from = slice * each, to = from + each < steps ? from + each : steps;
    if (which == kNext && from >= to) return;
    const OperandTile a = {A.grad + (static_cast<uint64_t>(m0) * A.piece + column) * 2, static_cast<uint64_t>(A.piece) * 2, A.tokens_up - m0, A.piece};
    OperandTile b;
    b.base = weight_row(A, first, first, &b.stride) + n0 * 2;
    b.valid = (A.weight ? width_up : static_cast<uint32_t>(A.b.width)) - n0;
    b.k_valid = n;
    f32x4 sum[S::kM][S::kN];
    product<BF16, BM, kAlongK, kAcrossK>(a, b, from, to, n % kStepK ? steps - 1 : ~0u, lds, sum);
    const int wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    const uint32_t m = m0 + (wave / S::kAcross) * (16 * S::kM) + lane % 16;
    const uint32_t d = n0 + (wave % S::kAcross) * (16 * S::kN) + 4 * (lane / 16);
    if (which == kOnly) {
        const float scale = A.state->scale;
        const uint32_t row0 = m - lane % 16, d0 = d - 4 * (lane / 16), width = static_cast<uint32_t>(A.b.width);
        RowsByLds<S::kM, S::kN>::pass(
            lds, [&](auto i, auto j) { return to_half<BF16>(sum[int(i)][int(j)] * scale); },
            [&](uint32_t row, uint32_t column, u32x4 v) {
                if (row0 + row < used && d0 + column < width)
                    put8(A.dhidden + A.index[row0 + row] * A.dhidden_stride * 2, d0 + column, width, v);
            });
        return;
    }
    static_for<S::kM>([&](auto i) {
        const uint32_t t = m + 16 * i;
        if (t >= used) return;
        float* const out = A.dh + (static_cast<uint64_t>(slice) * A.tokens_up + t) * width_up + d;
        static_for<S::kN>([&](auto j) {
            FF_GLOBAL f32x4* const p = (FF_GLOBAL f32x4*)(out + 16 * j);
            if (d + 16 * j < width_up) *p = which == kNext ? *p + sum[int(i)][int(j)] : sum[int(i)][int(j)];
        });
    });
}

// Sums of slices, rounded, in their place: four elements of a row to a thread; of narrow rows the threads that are left over take slices in turn
// (85 of them, dH of 189 tokens, 120 wide: 13.5 us one behind the other, 5 so).
constexpr uint32_t kPutThreads = 256, kPutRows = 1 << 16;
struct Slices {
    const float* from;
    uint64_t step;  // elements from one slice to the next
    uint32_t count, rows;
    uint8_t* out;
    uint64_t stride;  // elements
    const uint32_t* index;  // of the rows in their place, or null
};
template <bool BF16>
__device__ __forceinline__ void put_rows(const HeadArgs& A, const Slices& s, const uint32_t block, const uint32_t blocks)
{
    __shared__ f32x4 joined[kPutThreads];
    const uint32_t width_up = A.stride / 2, width = static_cast<uint32_t>(A.b.width);
    uint32_t across = kPutThreads;  // threads of a row
    while (across > kWaveSize / 4 && across * 2 >= width_up) across /= 2;
    const uint32_t turn = threadIdx.x / across, turns = kPutThreads / across;
    const uint32_t d = (blockIdx.y * across + threadIdx.x % across) * 4;
    constexpr uint32_t kAhead = 8;
    const float scale = A.state->scale;
    for (uint32_t r = block; r < s.rows; r += blocks) {
        const float* const from = s.from + static_cast<uint64_t>(r) * width_up + d;
        f32x4 sum = {0, 0, 0, 0};
        if (d < width)
            for (uint32_t k = turn; k < s.count; k += kAhead * turns) {
                f32x4 x[kAhead];
                static_for<kAhead>([&](auto i) { x[int(i)] = *(const FF_GLOBAL f32x4*)(from + (k + i * turns < s.count ? k + i * turns : k) * s.step); });
                static_for<kAhead>([&](auto i) {
                    if (k + i * turns < s.count) sum += x[int(i)];
                });
            }
        if (turns > 1) {
            __syncthreads();
            joined[threadIdx.x] = sum;
            __syncthreads();
            if (turn) continue;
            for (uint32_t k = 1; k < turns; k++) sum += joined[k * across + threadIdx.x];
        }
        if (d >= width) continue;
        uint8_t* const out = s.out + ((s.index ? s.index[r] : r) * s.stride + d) * 2;
        const u32x2 h = to_half<BF16>(sum * scale);
        if (d + 4 <= width) {
            *(FF_GLOBAL u32x2_a2*)out = h;
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 3; e++)
                if (d + e < width) as_global(reinterpret_cast<uint16_t*>(out))[e] = static_cast<uint16_t>(h[e / 2] >> e % 2 * 16);
        }
    }
}
// dH of all pieces and slices by the first `dh_blocks` workgroups, dW by the others.
template <bool BF16>
__global__ __launch_bounds__(kPutThreads) void head_put_kernel(const HeadArgs A, const uint32_t dh_blocks)
{
    const uint32_t width_up = A.stride / 2;
    const bool dh = blockIdx.x < dh_blocks;
    const Slices s = dh ? Slices{A.dh, static_cast<uint64_t>(A.tokens_up) * width_up, A.slices, A.state->used, A.dhidden, A.dhidden_stride, A.index}
                        : Slices{A.dw, static_cast<uint64_t>(A.piece) * width_up, A.dw_slices, static_cast<uint32_t>(A.b.vocab), A.dweight, A.dweight_stride, nullptr};
    put_rows<BF16>(A, s, dh ? blockIdx.x : blockIdx.x - dh_blocks, dh ? dh_blocks : gridDim.x - dh_blocks);
}

// dW = G^T H of vocabulary entries [first, first + n).
template <bool BF16>
__device__ __forceinline__ void dweight(const HeadArgs& A, const uint32_t first, const uint32_t n, const uint32_t column, const uint32_t block, const uint32_t blocks,
                                        FF_LDS uint8_t* lds)
{
    using S = Share<256>;
    const uint32_t used = A.state->used, width = static_cast<uint32_t>(A.b.width), width_up = A.stride / 2;
    const uint32_t tiles = blocks / A.dw_slices, slice = block / tiles;
    uint32_t m0, n0;
    tile_at(xcd_order(block - slice * tiles, tiles, kXcdTiles), (n + kTile - 1) / kTile, (width_up + kTile - 1) / kTile, &m0, &n0);
    m0 *= kTile;
    n0 *= kTile;
    const uint32_t steps = (used + kStepK - 1) / kStepK;
    const OperandTile a = {A.grad + (static_cast<uint64_t>(column) + m0) * 2, static_cast<uint64_t>(A.piece) * 2, A.piece - column - m0, A.tokens_up};
    const OperandTile b = {A.hidden + n0 * 2, A.stride, A.stride / 2 - n0, A.tokens_up};
    f32x4 sum[S::kM][S::kN];
    product<BF16, 256, kAcrossK, kAcrossK>(a, b, steps * slice / A.dw_slices, steps * (slice + 1) / A.dw_slices, ~0u, lds, sum);
    const float scale = A.state->scale;
    const int wave = threadIdx.x / kWaveSize;
    const uint32_t row0 = m0 + (wave / S::kAcross) * (16 * S::kM), d0 = n0 + (wave % S::kAcross) * (16 * S::kN);
    if (A.dw_slices > 1) {
        const uint32_t lane = threadIdx.x % kWaveSize;
        static_for<S::kM>([&](auto i) {
            const uint32_t row = row0 + 16 * i + lane % 16, d = d0 + lane / 16 * 4;
            float* const out = A.dw + (static_cast<uint64_t>(slice) * A.piece + row) * width_up + d;
            static_for<S::kN>([&](auto j) {
                if (row < n && d + 16 * j < width_up) *(FF_GLOBAL f32x4*)(out + 16 * j) = sum[int(i)][int(j)];
            });
        });
        return;
    }
    RowsByLds<S::kM, S::kN>::pass(
        lds, [&](auto i, auto j) { return to_half<BF16>(used ? sum[int(i)][int(j)] * scale : f32x4{0, 0, 0, 0}); },
        [&](uint32_t row, uint32_t column, u32x4 v) {
            if (row0 + row < n && d0 + column < width)
                put8_past(A.past, A.dweight + (static_cast<uint64_t>(first) + row0 + row) * A.dweight_stride * 2, d0 + column, width, v);
        });
}

// dW of few tokens, whose products are one step: a workgroup holds G of 64 vocabulary entries in registers and goes through the hidden states, 256
// elements at a time, which lie in the caches; three are on a compute unit, so that one's loads run under another's stores.  What bounds it:
// writing dW.  (260 us for the 1.05 GB of 128,256 x 4096, where 256 x 256 tiles, alone on a compute unit, took 460; with two buffers for the hidden states, and one workgroup, 340.)
constexpr int kFewWaves = 4, kFewEntries = 16 * kFewWaves;
template <bool BF16>
__global__ __launch_bounds__(kFewWaves* kWaveSize) void head_few_dweight_kernel(const HeadArgs A, const uint32_t first, const uint32_t n, const uint32_t parts)
{
    using H = Operand<kAcrossK, 256, kFewWaves>;
    using Out = RowsByLds<1, 4>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[H::kBytes + kFewWaves * Out::kBytes];
    const uint32_t used = A.state->used, width = static_cast<uint32_t>(A.b.width), width_up = A.stride / 2, chunks = (width_up + 255) / 256;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize), lane = threadIdx.x % kWaveSize;
    const uint32_t block = blockIdx.x / parts, part = blockIdx.x - block * parts;
    const uint32_t v0 = block * kFewEntries + wave * 16, v = v0 + lane % 16;  // of [first, first + n), as G's columns are here
    s16x8 g[2] = {};
    if (used)
        static_for<2>([&](auto half) {
            static_for<8>([&](auto e) {
                const uint32_t t = half * 32 + lane / 16 * 8 + e;  // (rows of zeros up to 64)
                g[int(half)][int(e)] = ((const FF_GLOBAL short*)A.grad)[static_cast<uint64_t>(t) * A.piece + first + v];
            });
        });
    const float scale = A.state->scale;
    auto fetch = [&](uint32_t chunk, FF_LDS uint8_t* buffer) {
        const OperandTile t = {A.hidden + chunk * 512, A.stride, width_up - chunk * 256, 64};
        H h;
        h.init(t, wave, lane);
        static_for<H::kLoads>([&](auto i) { h.fetch(i, 0, buffer, wave); });
    };
    FF_LDS uint8_t* const buffer = (FF_LDS uint8_t*)lds;
    for (uint32_t chunk = part; chunk < chunks; chunk += parts) {
        if (chunk != part) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // the last one has been read
        fetch(chunk, buffer);
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        static_for<4>([&](auto q) {
            f32x4 sum[4];
            static_for<4>([&](auto j) {
                sum[int(j)] = multiply<BF16>(H::fragment(buffer, 64 * q + 16 * j, 0, lane), g[0], f32x4{0, 0, 0, 0});
                if (used > 32) sum[int(j)] = multiply<BF16>(H::fragment(buffer, 64 * q + 16 * j, 1, lane), g[1], sum[int(j)]);
            });
            Out::pass(
                buffer + H::kBytes, [&](auto, auto j) { return to_half<BF16>(used ? sum[int(j)] * scale : f32x4{0, 0, 0, 0}); },
                [&](uint32_t row, uint32_t column, u32x4 x) {
                    const uint32_t d = chunk * 256 + 64 * q + column;
                    if (v0 + row < n && d < width) put8_past(A.past, A.dweight + (static_cast<uint64_t>(first) + v0 + row) * A.dweight_stride * 2, d, width, x);
                });
        });
    }
}

// Both: the first `dh_blocks` workgroups make dH, whose sums are longer, the others dW.
template <bool BF16, int BM>
__global__ __launch_bounds__(kProductThreads) __attribute__((amdgpu_waves_per_eu(2))) void head_grads_kernel(const HeadArgs A, const uint32_t first,
                                                                                                            const uint32_t n, const uint32_t column,
                                                                                                            const Sum which, const uint32_t dh_blocks)
{
    constexpr uint32_t kOne = kProductLds<BM, kAlongK, kAcrossK>, kOther = kProductLds<256, kAcrossK, kAcrossK>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kOne > kOther ? kOne : kOther];
    if (blockIdx.x < dh_blocks) dhidden<BF16, BM>(A, first, n, column, which, blockIdx.x, dh_blocks, (FF_LDS uint8_t*)lds);
    else dweight<BF16>(A, first, n, column, blockIdx.x - dh_blocks, gridDim.x - dh_blocks, (FF_LDS uint8_t*)lds);
}

__global__ void head_of_nothing_kernel(ff_head_stats* stats) { *stats = {}; }

// ---- the workspace ----------------------------------------------------------------------------------

constexpr uint64_t kPieceElements = 1ull << 29;  // of G, and of a piece's packed rows
constexpr uint64_t kFewDweightFrom = 1 << 23;    // elements of W, from which on dW of few tokens has its own launch
constexpr uint32_t kFewDweightBlocks = 1024;    // workgroups of head_few_dweight_kernel, about
constexpr uint32_t kKeptBlocks = 2048;           // workgroups that make G of kept logits, about

bool weight_as_it_is(const ff_head_batch& b)
{
    return reinterpret_cast<uint64_t>(b.weight) % 16 == 0 && b.weight_stride % 8 == 0 && b.width % 8 == 0 && b.weight_stride <= (1u << 22);
}

bool few(const ff_head_batch& b) { return b.n_tokens <= kFewTokens; }
// Is it better to keep the logits of the last piece than to make them again?  Eight bytes of memory to and fro stand against 2 * width
// operations: equal at a width of about 1000.  (Us, kept / made again: 1492 tokens on 34,257 x 1016 452 / 478, 4096 on 32,000 x 512 654 / 597, 2870 on 109,803 x
// 128 1115 / 823.)  Up to kKeptElements lie in the caches, and a launch is saved: 374 on 1922 x 185 42 / 48.
constexpr uint64_t kKeptElements = 1 << 22;
bool keeps(const ff_head_batch& b) { return few(b) || b.width >= 1024 || b.n_tokens * b.vocab <= kKeptElements; }
// Do the logits come from head_stream_kernel?  (Figures there.)
bool streams(const ff_head_batch& b, bool grad) { return weight_as_it_is(b) ? b.n_tokens <= 16 : !grad && b.n_tokens <= 32; }
// Tiles 256 tokens high, or 64: a round of the latter takes two thirds as long.  (Us, 256 / 64: scoring 256, 300, 512 tokens on 32,000 x 4096 121, 126, 129 / 162, 220,
// 287; 128 tokens 119 / 101.)
bool high_tiles(const ff_head_batch& b)
{
    const uint64_t across = up(b.vocab, kTile) / kTile, rounds = (up(b.n_tokens, kTile) / kTile * across + kComputeUnits - 1) / kComputeUnits;
    return !few(b) && up(b.n_tokens, 64) / 64 * across * 2 > kComputeUnits * 3 * rounds;
}
uint32_t up64(uint64_t n) { return static_cast<uint32_t>(up(std::max<uint64_t>(n, 1), 64)); }
// Vocabulary entries that a workgroup of head_stream_kernel takes.
uint32_t stream_entries(uint64_t n_tokens) { return n_tokens <= 16 ? Stream<1>::kEntries : Stream<2>::kEntries; }

struct Places {
    uint64_t state, index, weights, targets, rows, losses, picked, parts, hidden, weight, grad, logits, dh, dw, bytes;
};

Places place(const ff_head_batch& b, bool grad, HeadArgs* A)
{
    const uint64_t n = b.n_tokens, width_up = up(b.width, kStepK);
    const uint32_t high = high_tiles(b) ? kTile : 64, tile = streams(b, grad) ? stream_entries(n) : kTile;
    A->tokens_up = static_cast<uint32_t>(up(std::max<uint64_t>(n, 1), high));
    A->tiles = static_cast<uint32_t>((b.vocab + tile - 1) / tile);
    A->stride = static_cast<uint32_t>(width_up * 2);
    const bool packed = !weight_as_it_is(b);
    const uint64_t whole = up(b.vocab, kTile), least = kTile;
    // G is of a piece, rows are copied for a piece: of few tokens it is whole, and they may still be copied in several
    uint64_t piece = few(b) ? whole : std::min<uint64_t>(whole, most_groups(kProductThreads) / (A->tokens_up / high) * kTile);
    if (grad && !few(b)) piece = std::min(piece, std::max(kPieceElements / A->tokens_up / kTile * kTile, least));
    uint64_t step = piece;
    if (packed) step = std::min(piece, std::max(kPieceElements / width_up / kTile * kTile, least));
    if (!few(b)) piece = step;
    A->piece = static_cast<uint32_t>(piece);
    A->step = static_cast<uint32_t>(step);
    // dH's sum over a piece in so many slices that its tiles fill the chip, of four steps at least
    const uint64_t dh_tiles = A->tokens_up / high * (up(width_up, kTile) / kTile), steps = (step + kStepK - 1) / kStepK;
    A->slices = static_cast<uint32_t>(std::max<uint64_t>(std::min(kComputeUnits / dh_tiles, steps / 4), 1));
    // The logits' sums in so many slices that their tiles fill the chip, of four steps at least, where that saves more than a row's workgroup takes:
    // a step, 0.9 us, for every 512 entries.  (Us, without / with: 21 tokens on 1240 x 8128 126 / 50, 256 on 256 x 4096 73 / 36, 64 on 8000 x 4096, scored,
    // 61 / 41; 120 on 9023 x 768 would take 58 instead of 52.)
    const uint64_t z_tiles = A->tokens_up / high * (whole / kTile), z_steps = width_up / kStepK;
    uint64_t splits = high == 64 && !streams(b, grad) && step >= b.vocab ? std::max<uint64_t>(std::min(kComputeUnits / z_tiles, z_steps / 4), 1) : 1;
    if ((z_steps - z_steps / splits) * 512 < b.vocab) splits = 1;
    A->splits = static_cast<uint32_t>(splits);
    // dW's over the tokens likewise, where the steps that it saves take longer than what writing and reading the slices does, at 5 TB/s.  (Us, without / with: 3185
    // tokens on 1332 x 384 119 / 92, 4096 on 256 x 4096 150 / 114, on 4099 x 768 228 / 200; 1000 on 4099 x 768 would take 96 instead of 90.)
    const uint64_t dw_tiles = whole / kTile * (up(width_up, kTile) / kTile), dw_steps = up(n, kStepK) / kStepK;
    uint64_t dw_slices = !few(b) && step >= b.vocab ? std::max<uint64_t>(std::min(kComputeUnits / dw_tiles, dw_steps / 4), 1) : 1;
    if ((dw_steps - dw_steps / dw_slices) << 22 < whole * width_up * (8 * dw_slices + 2)) dw_slices = 1;
    A->dw_slices = static_cast<uint32_t>(dw_slices);
    Places p = {};
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    p.state = take(sizeof(State));
    p.index = take(n * 4);
    p.weights = take(n * 4);
    p.targets = take(n * 4);
    p.rows = take(n * sizeof(Row));
    p.losses = take(n * 8);
    p.picked = take(n * 4);
    // (never less for more tokens, entries or elements, whatever tiles and pieces come to)
    p.parts = take(std::max(n * (whole / kTile), std::min<uint64_t>(n, 32) * (whole / 64)) * sizeof(float2));
    const uint64_t rows = few(b) ? kFewTokens : up(n, kTile);
    p.hidden = take(rows * A->stride);
    auto piece_of = [&](uint64_t r) { return std::max(std::min(r * whole, kPieceElements), r * kTile) * 2; };
    p.weight = take(packed && (grad || !streams(b, grad)) ? piece_of(width_up) : 0);
    const uint64_t split = std::min<uint64_t>(rows * whole * z_steps, kComputeUnits * 64 * kTile) * 4;  // of any slices
    if (!grad) p.logits = take(split);
    if (grad) {
        const uint64_t all = piece_of(rows), smaller = std::max(kFewTokens * whole, kKeptElements + kTile * (rows + whole + kTile)) * 4;
        p.grad = take(all);
        p.logits = take(std::max(split, keeps(b) ? 2 * all : std::min(2 * all, smaller)));
        const uint64_t dh = rows * width_up;
        p.dw = take(std::min<uint64_t>(whole * width_up * (rows / kStepK), kComputeUnits * kTile * kTile) * 4);
        p.dh = take(std::max(dh, std::min<uint64_t>(dh * (whole / kTile), kComputeUnits * kTile * kTile)) * 4);
    }
    p.bytes = at;
    return p;
}

template <bool BF16, int BM>
hipError_t launch(const HeadArgs& A, hipStream_t stream)
{
    const uint32_t n = static_cast<uint32_t>(A.b.n_tokens), vocab = static_cast<uint32_t>(A.b.vocab), tiles_m = A.tokens_up / BM;
    const uint32_t tiles_d = (A.stride / 2 + kTile - 1) / kTile;
    const uint32_t n_pieces = static_cast<uint32_t>((static_cast<uint64_t>(vocab) + A.step - 1) / A.step);
    const bool grad = A.dhidden || A.dweight, keep = grad && (A.splits > 1 || keeps(A.b)), whole = few(A.b);
    const bool few_dweight = whole && static_cast<uint64_t>(vocab) * A.b.width >= kFewDweightFrom;
    const bool copies = A.weight && n;  // (without tokens W is not read: there may be none)
    uint32_t first = 0, m = 0, tiles = 0, packed = ~0u;
    if (n <= kSelectFew) {
        const uint32_t rows = copies && !streams(A.b, grad) ? std::min(A.step, vocab) : 0, blocks = up64(n);
        hipLaunchKernelGGL(head_few_kernel, dim3(blocks + std::min(rows, kPackBlocks)), dim3(256), 0, stream, A, blocks, rows);
        if (rows) packed = 0;
    } else {
        hipLaunchKernelGGL(head_select_kernel, dim3(1), dim3(kSelectThreads), 0, stream, A);
        hipLaunchKernelGGL(head_gather_kernel, dim3(std::min(A.tokens_up, 4096u)), dim3(256), 0, stream, A);
    }
    // makes piece i the one that the following launches are for
    auto take = [&](uint32_t i, bool rows) {
        first = i * A.step;
        m = std::min(A.step, vocab - first);
        tiles = (m + kTile - 1) / kTile;
        if (!copies || !rows || packed == i) return;
        hipLaunchKernelGGL(head_pack_kernel, dim3(std::min(m, kPackBlocks)), dim3(256), 0, stream, A, first, m);
        packed = i;
    };
    const dim3 threads(kProductThreads);
    if (A.splits > 1) {
        take(0, true);
        if constexpr (BM == 64) hipLaunchKernelGGL((head_logits_kernel<BF16, BM, kSplit>), dim3(tiles * tiles_m * A.splits), threads, 0, stream, A, first, m);
    } else if (streams(A.b, grad)) {
        const auto kernel = grad ? head_stream_kernel<BF16, 1, kKeep> : n <= 16 ? head_stream_kernel<BF16, 1, kSums> : head_stream_kernel<BF16, 2, kSums>;
        hipLaunchKernelGGL(kernel, dim3(A.tiles), dim3(kStreamThreads), 0, stream, A);
    } else {
        for (uint32_t i = 0; i < n_pieces; i++) {
            take(i, true);
            const dim3 grid(tiles * tiles_m);
            if (keep && (whole || i == n_pieces - 1)) hipLaunchKernelGGL((head_logits_kernel<BF16, BM, kKeep>), grid, threads, 0, stream, A, first, m);
            else hipLaunchKernelGGL((head_logits_kernel<BF16, BM, kSums>), grid, threads, 0, stream, A, first, m);
        }
    }
    if (A.splits > 1) {
        hipLaunchKernelGGL(head_row_kernel<BF16>, dim3(up64(n)), dim3(256), 0, stream, A, grad);
    } else if (keep) {
        const uint32_t from = whole ? 0 : first, of = vocab - from, rows = up64(n);
        const uint32_t wide = std::min((of + 2047) / 2048, (kKeptBlocks + rows - 1) / rows);
        hipLaunchKernelGGL(head_kept_kernel<BF16>, dim3(rows * wide), dim3(256), 0, stream, A, from, of, wide);
    } else {
        hipLaunchKernelGGL(head_finish_kernel<BF16>, dim3(n / 4 + 1), dim3(256), 0, stream, A);
    }
    if (n > kCountFew) hipLaunchKernelGGL(head_sum_kernel, dim3(1), dim3(kSelectThreads), 0, stream, A);
    if (!grad) return hipGetLastError();
    const Sum start = n_pieces == 1 && A.slices == 1 ? kOnly : kFirst;
    for (uint32_t i = n_pieces; i-- > 0;) {  // from the last one, whose logits and packed rows are at hand
        const bool last = i == n_pieces - 1, logits = !whole && (!keep || !last);
        take(i, A.dhidden || logits);
        if (logits) hipLaunchKernelGGL((head_logits_kernel<BF16, BM, kGrad>), dim3(tiles * tiles_m), threads, 0, stream, A, first, m);
        const uint32_t dh_blocks = A.dhidden ? tiles_m * tiles_d * A.slices : 0, dw_blocks = A.dweight && !few_dweight ? tiles * tiles_d * A.dw_slices : 0;
        if (A.dweight && few_dweight) {
            const uint32_t blocks = (m + kFewEntries - 1) / kFewEntries, parts = std::min(tiles_d, (kFewDweightBlocks + blocks - 1) / blocks);
            hipLaunchKernelGGL(head_few_dweight_kernel<BF16>, dim3(blocks * parts), dim3(kFewWaves * kWaveSize), 0, stream, A, first, m, parts);
        }
        if (dh_blocks + dw_blocks)
            hipLaunchKernelGGL((head_grads_kernel<BF16, BM>), dim3(dh_blocks + dw_blocks), threads, 0, stream, A, first, m, whole ? first : 0,
                           last ? start : kNext, dh_blocks);
    }
    const uint32_t dh_rows = A.dhidden && start != kOnly ? std::min(n, kPutRows) : 0, dw_rows = A.dweight && A.dw_slices > 1 ? std::min(vocab, kPutRows) : 0;
    if (dh_rows + dw_rows) {
        const uint32_t blocks_of_row = static_cast<uint32_t>((A.b.width + 4 * kPutThreads - 1) / (4 * kPutThreads));
        hipLaunchKernelGGL(head_put_kernel<BF16>, dim3(dh_rows + dw_rows, blocks_of_row), dim3(kPutThreads), 0, stream, A, dh_rows);
    }
    return hipGetLastError();
}

}  // namespace

uint64_t head_workspace(const ff_head_batch& b, bool grad)
{
    HeadArgs A = {};
    return place(b, grad, &A).bytes;
}

hipError_t launch_head(const ff_head_batch& b, float* logp, void* dhidden, uint64_t dhidden_stride, void* dweight, uint64_t dweight_stride,
                       ff_head_stats* stats, void* workspace, hipStream_t stream)
{
    if (!b.n_tokens && !dweight) {
        hipLaunchKernelGGL(head_of_nothing_kernel, dim3(1), dim3(1), 0, stream, stats);
        return hipGetLastError();
    }
    HeadArgs A = {};
    const Places p = place(b, dhidden || dweight, &A);
    uint8_t* const w = static_cast<uint8_t*>(workspace);
    A.b = b;
    A.logp = logp;
    A.dhidden = static_cast<uint8_t*>(dhidden);
    A.dweight = static_cast<uint8_t*>(dweight);
    A.dhidden_stride = dhidden_stride;
    A.dweight_stride = dweight_stride;
    A.stats = stats;
    A.state = reinterpret_cast<State*>(w + p.state);
    A.index = reinterpret_cast<uint32_t*>(w + p.index);
    A.weights = reinterpret_cast<float*>(w + p.weights);
    A.targets = reinterpret_cast<int32_t*>(w + p.targets);
    A.rows = reinterpret_cast<Row*>(w + p.rows);
    A.losses = reinterpret_cast<double*>(w + p.losses);
    A.picked = reinterpret_cast<float*>(w + p.picked);
    A.parts = reinterpret_cast<float2*>(w + p.parts);
    A.hidden = w + p.hidden;
    A.weight = weight_as_it_is(b) ? nullptr : w + p.weight;
    A.grad = w + p.grad;
    A.logits = reinterpret_cast<float*>(w + p.logits);
    A.dh = reinterpret_cast<float*>(w + p.dh);
    A.dw = reinterpret_cast<float*>(w + p.dw);
    A.grad_scale = b.loss_scale * (b.dtype == FF_BF16 ? 1.f : 0x1p-14f);
    A.past = reinterpret_cast<uint64_t>(dweight) % 16 == 0 && dweight_stride % 8 == 0;
    const bool high = high_tiles(b);
    if (b.dtype == FF_BF16) return high ? launch<true, 256>(A, stream) : launch<true, 64>(A, stream);
    return high ? launch<false, 256>(A, stream) : launch<false, 64>(A, stream);
}

}  // namespace ffsnap
