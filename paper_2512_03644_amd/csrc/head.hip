// Cross entropy over a large vocabulary from hidden states, and its gradients, for gfx950.
//
// z = H W^T is made in tiles of 256 vocabulary entries and never stored: a tile leaves, for each token, its largest logit, the sum of
// exponentials against it, and the target's logit.  Joined over the tiles these give the log-probability.  For the
// gradients the vocabulary is taken in pieces: a piece's logits are made once more, become G = (softmax - [target]) * weight in 16 bits, and two
// products take G: dH += G W, in 32 bits over the pieces, and dW = G^T H.  Four products of 2 * tokens * vocab * width operations in all, where
// three would do if all logits were kept.
//
// G is rounded to 16 bits, for the matrix instructions; nothing else is, in front of the outputs.  Weights are divided
// by the largest one first, so that tokens of equal weight have exact factors of 1 (a factor rounded with G would
// be the same error in every token); it comes back, with the loss scale, on 32-bit sums.  For fp16, G is 2^14 times that: a
// softmax of 2^-28 is still a normal number.
#include "head.hpp"

#include <algorithm>

#include "product.h"
#include "xcd_order.h"

namespace ffsnap {

namespace {

constexpr uint32_t kTile = 256;        // vocabulary entries of a tile
constexpr uint32_t kFewTokens = 64;    // up to so many, tiles are 64 tokens high
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
    float scale;             // of the gradients: what G has been divided by
    uint32_t unused;
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
    Row* rows;
    double* losses;     // of each of them, times its weight
    float* picked;      // logit of the target
    float2* parts;      // [token][tile]: largest logit, sum of exponentials
    uint8_t* hidden;    // packed rows of those tokens: `stride` bytes, zeros behind the width and behind the last up to 64 rows
    uint8_t* weight;    // packed rows of a piece, if W's own do not lie as the loads want them; or null
    uint8_t* grad;      // G of a piece: [tokens up to a tile][piece]
    float* dh;          // [slice][token][width up to 64]: dH so far
    uint32_t tokens_up; // tokens, up to a whole tile
    uint32_t tiles;     // of the vocabulary
    uint32_t stride;    // bytes of a packed row
    uint32_t piece;     // vocabulary entries of a piece, a multiple of 256
    uint32_t slices;    // of dH's sum over a piece
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

// In their order; the largest weight.  One workgroup: a few thousand tokens are a few rounds.
constexpr int kSelectThreads = 1024;
__global__ __launch_bounds__(kSelectThreads) void head_select_kernel(const HeadArgs A)
{
    __shared__ uint32_t count[kSelectThreads / kWaveSize];
    __shared__ float largest[kSelectThreads / kWaveSize];
    const uint32_t n = static_cast<uint32_t>(A.b.n_tokens), wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    uint32_t used = 0, invalid = 0;
    float most = 0.f;
    for (uint64_t first = 0; first < n; first += kSelectThreads) {
        const uint64_t t = first + threadIdx.x;
        const float w = t < n ? A.b.weights[t] : 0.f;
        const int64_t y = t < n ? A.b.targets[t] : -1;
        const bool wanted = !(w == 0.f), inside = y >= 0 && static_cast<uint64_t>(y) < A.b.vocab, mine = wanted && inside;
        const uint64_t who = __ballot(mine);
        if (lane == 0) count[wave] = __popcll(who);
        __syncthreads();
        uint32_t before = used, all = 0;
        for (uint32_t k = 0; k < kSelectThreads / kWaveSize; k++) {
            if (k < wave) before += count[k];
            all += count[k];
        }
        __syncthreads();
        if (mine) {
            const uint32_t at = before + __popcll(who & ((1ull << lane) - 1));
            A.index[at] = static_cast<uint32_t>(t);
            A.rows[at].factor = w;
            A.rows[at].y = static_cast<int32_t>(y);
            if (__builtin_isfinite(w)) most = fmaxf(most, fabsf(w));
        } else if (t < n) {
            A.logp[t] = 0.f;
        }
        used += all;
        invalid += __syncthreads_count(wanted && !inside);
    }
    for (int d = 32; d; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
    if (lane == 0) largest[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (uint32_t k = 0; k < kSelectThreads / kWaveSize; k++) most = fmaxf(most, largest[k]);
        A.state->used = used;
        A.state->invalid = invalid;
        A.state->scale = most;
    }
}

// `width` elements of a row to a packed one; elements behind them are zeros.
__device__ __forceinline__ void copy_row(uint8_t* to, uint32_t bytes, const uint8_t* from, uint32_t width)
{
    for (uint32_t i = threadIdx.x; i < bytes / 16; i += blockDim.x) {
        u32x4 v = {0, 0, 0, 0};
        if (i * 8 + 8 <= width) {
            v = *(const FF_GLOBAL u32x4_a2*)(from + 16ull * i);
        } else {
            uint16_t x[8] = {};
            for (uint32_t k = i * 8; k < width; k++) x[k % 8] = as_global(reinterpret_cast<const uint16_t*>(from))[k];
            v = u32x4{x[0] | uint32_t(x[1]) << 16, x[2] | uint32_t(x[3]) << 16, x[4] | uint32_t(x[5]) << 16, x[6] | uint32_t(x[7]) << 16};
        }
        *(FF_GLOBAL u32x4*)(to + 16ull * i) = v;
    }
}

// Hidden states of the tokens that count, one behind the other, and zeros up to 64 rows; gradients of the other tokens.
__global__ __launch_bounds__(256) void head_gather_kernel(const HeadArgs A)
{
    const uint32_t used = A.state->used, until = (used + 63) / 64 * 64, n = static_cast<uint32_t>(A.b.n_tokens);
    for (uint32_t r = blockIdx.x; r < until; r += gridDim.x) {
        const uint64_t t = r < used ? A.index[r] : 0;
        copy_row(A.hidden + static_cast<uint64_t>(r) * A.stride, A.stride,
                 static_cast<const uint8_t*>(A.b.hidden) + t * A.b.hidden_stride * 2, r < used ? static_cast<uint32_t>(A.b.width) : 0);
    }
    if (!A.dhidden) return;
    for (uint64_t t = blockIdx.x; t < n; t += gridDim.x) {
        const float w = A.b.weights[t];
        const int64_t y = A.b.targets[t];
        if (!(w == 0.f) && y >= 0 && static_cast<uint64_t>(y) < A.b.vocab) continue;
        uint16_t* const to = reinterpret_cast<uint16_t*>(A.dhidden + t * A.dhidden_stride * 2);
        for (uint32_t i = threadIdx.x; i < A.b.width; i += blockDim.x) as_global(to)[i] = 0;
    }
}

// Rows [first, first + n) of W, packed.
__global__ __launch_bounds__(256) void head_pack_kernel(const HeadArgs A, const uint32_t first, const uint32_t n)
{
    for (uint32_t r = blockIdx.x; r < n; r += gridDim.x)
        copy_row(A.weight + static_cast<uint64_t>(r) * A.stride, A.stride,
                 static_cast<const uint8_t*>(A.b.weight) + (static_cast<uint64_t>(first) + r) * A.b.weight_stride * 2, static_cast<uint32_t>(A.b.width));
}

// ---- logits ---------------------------------------------------------------------------------------

// The tiles of vocabulary entries [first, first + n).  Without GRAD the tile's part of the sums, with GRAD its G.
template <bool BF16, int BM, bool GRAD>
__global__ __launch_bounds__(kProductThreads) __attribute__((amdgpu_waves_per_eu(2))) void head_logits_kernel(const HeadArgs A, const uint32_t first,
                                                                                                             const uint32_t n)
{
    using S = Share<BM>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kProductLds<BM, kAlongK, kAlongK>];
    const uint32_t used = A.state->used;
    uint32_t m0, n0;
    tile_at(xcd_order(blockIdx.x, gridDim.x, kXcdTiles), A.tokens_up / BM, (n + kTile - 1) / kTile, &m0, &n0);
    m0 *= BM;
    n0 *= kTile;
    if (m0 >= used) return;
    const uint32_t v0 = first + n0, vocab = static_cast<uint32_t>(A.b.vocab);
    OperandTile b;
    b.base = weight_row(A, first, v0, &b.stride);
    b.valid = n - n0;
    b.k_valid = A.weight ? A.stride / 2 : static_cast<uint32_t>(A.b.width);
    const uint32_t steps = A.stride / (2 * kStepK);
    f32x4 z[S::kM][S::kN];
    product<BF16, BM, kAlongK, kAlongK>(hidden_tile(A, m0, used), b, 0, steps, b.k_valid % kStepK ? steps - 1 : ~0u, (FF_LDS uint8_t*)lds, z);
    const int wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    const uint32_t m = m0 + (wave / S::kAcross) * (16 * S::kM) + lane % 16;                    // + 16 i
    const uint32_t v = v0 + (wave % S::kAcross) * (16 * S::kN) + 4 * (lane / 16);              // + 16 j + e
    if constexpr (GRAD) {
        const uint32_t at = v - first;
        for (int i = 0; i < S::kM; i++) {
            const uint32_t t = m + 16 * i;
            Row r = {0.f, 0.f, 0.f, -1};
            if (t < used) r = A.rows[t];
            const bool there = t < used;
            uint8_t* const out = A.grad + (static_cast<uint64_t>(t) * A.piece + at) * 2;
            for (int j = 0; j < S::kN; j++) {
                f32x4 g;
                for (int e = 0; e < 4; e++) {
                    const uint32_t vocab_entry = v + 16 * j + e;
                    float p = __builtin_amdgcn_exp2f(fmaf(z[i][j][e], kLog2E, -r.lse2)) * r.factor;
                    p = static_cast<int32_t>(vocab_entry) == r.y ? r.target : p;
                    g[e] = there && vocab_entry < vocab ? p : 0.f;
                }
                *(FF_GLOBAL u32x2*)(out + 32 * j) = to_half<BF16>(g);
            }
        }
    } else {
        __shared__ float2 part[S::kAcross][BM];
        for (int i = 0; i < S::kM; i++) {
            const uint32_t t = m + 16 * i;
            const int32_t y = t < used ? A.rows[t].y : -1;
            float top = -INFINITY, total = 0.f, target = 0.f;
            bool mine = false;
            for (int j = 0; j < S::kN; j++)
                for (int e = 0; e < 4; e++) {
                    const uint32_t vocab_entry = v + 16 * j + e;
                    if (static_cast<int32_t>(vocab_entry) == y) {
                        mine = true;
                        target = z[i][j][e];
                    }
                    if (vocab_entry >= vocab) z[i][j][e] = -INFINITY;
                    // (a NaN or +inf stays in the sum, as exp(NaN - top) or exp(inf - inf))
                    top = fmaxf(top, z[i][j][e]);
                }
            if (mine) A.picked[t] = target;
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float against = top == -INFINITY ? 0.f : top;
            for (int j = 0; j < S::kN; j++)
                for (int e = 0; e < 4; e++) total += __builtin_amdgcn_exp2f((z[i][j][e] - against) * kLog2E);
            total += __shfl_xor(total, 16);
            total += __shfl_xor(total, 32);
            if (lane < 16) part[wave % S::kAcross][(wave / S::kAcross) * (16 * S::kM) + 16 * i + lane] = float2{top, total};
        }
        __syncthreads();
        for (uint32_t r = threadIdx.x; r < BM; r += kProductThreads) {
            if (m0 + r >= used) break;
            float top = -INFINITY, total = 0.f;
            for (int k = 0; k < S::kAcross; k++) top = fmaxf(top, part[k][r].x);
            const float against = top == -INFINITY ? 0.f : top;
            for (int k = 0; k < S::kAcross; k++) total += part[k][r].y * __builtin_amdgcn_exp2f((part[k][r].x - against) * kLog2E);
            A.parts[static_cast<uint64_t>(m0 + r) * A.tiles + v0 / kTile] = float2{top, total};
        }
    }
}

// ---- log-probabilities ----------------------------------------------------------------------------

// A wavefront joins the tiles' parts of a token, in 64 bits from the exponentials on.
template <bool BF16>
__global__ __launch_bounds__(256) void head_finish_kernel(const HeadArgs A)
{
    const uint32_t used = A.state->used, lane = threadIdx.x % kWaveSize;
    const float largest = A.state->scale;
    const uint32_t r = blockIdx.x * (256 / kWaveSize) + threadIdx.x / kWaveSize;
    if (r >= used) return;
    const float2* const parts = A.parts + static_cast<uint64_t>(r) * A.tiles;
    float top = -INFINITY;
    for (uint32_t k = lane; k < A.tiles; k += kWaveSize) top = fmaxf(top, parts[k].x);
    for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float against = top == -INFINITY ? 0.f : top;
    double total = 0;
    for (uint32_t k = lane; k < A.tiles; k += kWaveSize) {
        const float2 p = parts[k];
        total += static_cast<double>(p.y) * exp(static_cast<double>(p.x) - static_cast<double>(against));
    }
    for (int d = 32; d; d /= 2) total += __shfl_xor(total, d);
    if (lane == 0) {
        const double rest = log(total);
        const double logp = (static_cast<double>(A.picked[r]) - static_cast<double>(against)) - rest;
        const uint32_t t = A.index[r];
        const float w = A.rows[r].factor;
        A.logp[t] = static_cast<float>(logp);
        A.losses[r] = -static_cast<double>(w) * logp;
        const float f = w / largest * (BF16 ? 1.f : 0x1p14f);
        A.rows[r].lse2 = static_cast<float>((static_cast<double>(against) + rest) * 1.4426950408889634);
        A.rows[r].factor = f;
        A.rows[r].target = f * static_cast<float>(expm1(logp));
    }
}

// The loss, in an order that the number of tokens gives.
__global__ __launch_bounds__(kSelectThreads) void head_sum_kernel(const HeadArgs A, const float grad_scale)
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
    if (threadIdx.x == 0) {
        A.stats->loss = static_cast<float>(sum[0]);
        A.stats->reserved = 0;
        A.stats->n_tokens = used;
        A.stats->n_invalid = A.state->invalid;
        A.state->scale *= grad_scale;
    }
}

// ---- gradients ------------------------------------------------------------------------------------

// dH (+)= G W over a slice of the piece [first, first + n).
template <bool BF16, int BM>
__global__ __launch_bounds__(kProductThreads) __attribute__((amdgpu_waves_per_eu(2))) void head_dhidden_kernel(const HeadArgs A, const uint32_t first,
                                                                                                              const uint32_t n)
{
    using S = Share<BM>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kProductLds<BM, kAlongK, kAcrossK>];
    const uint32_t used = A.state->used, width_up = A.stride / 2;
    const uint32_t tiles_m = A.tokens_up / BM, tiles_n = (width_up + kTile - 1) / kTile;
    const uint32_t tile = xcd_order(blockIdx.x, gridDim.x, kXcdTiles), slice = tile / (tiles_m * tiles_n);
    uint32_t m0, n0;
    tile_at(tile - slice * (tiles_m * tiles_n), tiles_m, tiles_n, &m0, &n0);
    m0 *= BM;
    n0 *= kTile;
    if (m0 >= used) return;
    const uint32_t steps = (n + kStepK - 1) / kStepK, each = (steps + A.slices - 1) / A.slices;
    const uint32_t from = slice * each, to = from + each < steps ? from + each : steps;
    if (first && from >= to) return;
    const OperandTile a = {A.grad + static_cast<uint64_t>(m0) * A.piece * 2, static_cast<uint64_t>(A.piece) * 2, A.tokens_up - m0, A.piece};
    OperandTile b;
    b.base = weight_row(A, first, first, &b.stride) + n0 * 2;
    b.valid = (A.weight ? width_up : static_cast<uint32_t>(A.b.width)) - n0;
    b.k_valid = n;
    f32x4 sum[S::kM][S::kN];
    product<BF16, BM, kAlongK, kAcrossK>(a, b, from, to, n % kStepK ? steps - 1 : ~0u, (FF_LDS uint8_t*)lds, sum);
    const int wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    const uint32_t m = m0 + (wave / S::kAcross) * (16 * S::kM) + lane % 16;
    const uint32_t d = n0 + (wave % S::kAcross) * (16 * S::kN) + 4 * (lane / 16);
    for (int i = 0; i < S::kM; i++) {
        const uint32_t t = m + 16 * i;
        if (t >= used) continue;
        float* const out = A.dh + (static_cast<uint64_t>(slice) * A.tokens_up + t) * width_up + d;
        for (int j = 0; j < S::kN; j++) {
            if (d + 16 * j >= width_up) continue;
            FF_GLOBAL f32x4* const p = (FF_GLOBAL f32x4*)(out + 16 * j);
            *p = first ? *p + sum[i][j] : sum[i][j];
        }
    }
}

// Elements [at, at + 4) of a row of `width`, rounded.
template <bool BF16>
__device__ __forceinline__ void put4(uint8_t* row, uint32_t at, uint32_t width, f32x4 v)
{
    const u32x2 h = to_half<BF16>(v);
    uint8_t* const p = row + 2ull * at;
    if (at + 4 <= width) {
        *(FF_GLOBAL u32x2_a2*)p = h;
    } else {
        for (uint32_t e = 0; at + e < width; e++) as_global(reinterpret_cast<uint16_t*>(p))[e] = static_cast<uint16_t>((e & 2 ? h.y : h.x) >> (e & 1) * 16);
    }
}

// dH of all pieces and slices, in its place.
template <bool BF16>
__global__ __launch_bounds__(256) void head_put_kernel(const HeadArgs A)
{
    const uint32_t used = A.state->used, width_up = A.stride / 2, width = static_cast<uint32_t>(A.b.width);
    const float scale = A.state->scale;
    for (uint32_t r = blockIdx.x; r < used; r += gridDim.x) {
        uint8_t* const out = A.dhidden + A.index[r] * A.dhidden_stride * 2;
        for (uint32_t d = 4 * threadIdx.x; d < width; d += 4 * blockDim.x) {
            f32x4 s = {0, 0, 0, 0};
            for (uint32_t k = 0; k < A.slices; k++)
                s += *(const FF_GLOBAL f32x4*)(A.dh + (static_cast<uint64_t>(k) * A.tokens_up + r) * width_up + d);
            put4<BF16>(out, d, width, s * scale);
        }
    }
}

// dW = G^T H of the piece [first, first + n).
template <bool BF16>
__global__ __launch_bounds__(kProductThreads) __attribute__((amdgpu_waves_per_eu(2))) void head_dweight_kernel(const HeadArgs A, const uint32_t first,
                                                                                                              const uint32_t n)
{
    using S = Share<256>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kProductLds<256, kAcrossK, kAcrossK>];
    const uint32_t used = A.state->used, width = static_cast<uint32_t>(A.b.width);
    uint32_t m0, n0;
    tile_at(xcd_order(blockIdx.x, gridDim.x, kXcdTiles), (n + kTile - 1) / kTile, (A.stride / 2 + kTile - 1) / kTile, &m0, &n0);
    m0 *= kTile;
    n0 *= kTile;
    const uint32_t steps = (used + kStepK - 1) / kStepK;
    const OperandTile a = {A.grad + m0 * 2, static_cast<uint64_t>(A.piece) * 2, A.piece - m0, A.tokens_up};
    const OperandTile b = {A.hidden + n0 * 2, A.stride, A.stride / 2 - n0, A.tokens_up};
    f32x4 sum[S::kM][S::kN];
    product<BF16, 256, kAcrossK, kAcrossK>(a, b, 0, steps, ~0u, (FF_LDS uint8_t*)lds, sum);
    const float scale = A.state->scale;
    const int wave = threadIdx.x / kWaveSize, lane = threadIdx.x % kWaveSize;
    const uint32_t m = m0 + (wave / S::kAcross) * (16 * S::kM) + lane % 16;
    const uint32_t d = n0 + (wave % S::kAcross) * (16 * S::kN) + 4 * (lane / 16);
    for (int i = 0; i < S::kM; i++) {
        if (m + 16 * i >= n) continue;
        uint8_t* const out = A.dweight + (static_cast<uint64_t>(first) + m + 16 * i) * A.dweight_stride * 2;
        for (int j = 0; j < S::kN; j++)
            if (d + 16 * j < width) put4<BF16>(out, d + 16 * j, width, used ? sum[i][j] * scale : f32x4{0, 0, 0, 0});
    }
}

__global__ void head_of_nothing_kernel(ff_head_stats* stats) { *stats = {}; }

// ---- the workspace ----------------------------------------------------------------------------------

constexpr uint64_t kPieceElements = 1ull << 27;  // of G, and of a piece's packed rows
constexpr uint32_t kSliceTokens = 2048;          // tokens times slices, up to so many

bool weight_as_it_is(const ff_head_batch& b)
{
    return reinterpret_cast<uint64_t>(b.weight) % 16 == 0 && b.weight_stride % 8 == 0 && b.width % 8 == 0 && b.weight_stride <= (1u << 22);
}

struct Places {
    uint64_t state, index, rows, losses, picked, parts, hidden, weight, grad, dh, bytes;
};

Places place(const ff_head_batch& b, bool grad, HeadArgs* A)
{
    const uint64_t n = b.n_tokens, width_up = up(b.width, kStepK);
    A->tokens_up = static_cast<uint32_t>(n <= kFewTokens ? kFewTokens : up(n, kTile));
    A->tiles = static_cast<uint32_t>((b.vocab + kTile - 1) / kTile);
    A->stride = static_cast<uint32_t>(width_up * 2);
    const bool packed = !weight_as_it_is(b);
    const uint32_t tiles_m = A->tokens_up / (n <= kFewTokens ? kFewTokens : kTile);
    uint64_t piece = std::min<uint64_t>(up(b.vocab, kTile), most_groups(kProductThreads) / tiles_m * kTile);
    if (grad) piece = std::min(piece, std::max<uint64_t>(kPieceElements / A->tokens_up / kTile, 1) * kTile);
    if (packed) piece = std::min(piece, std::max<uint64_t>(kPieceElements / width_up / kTile, 1) * kTile);
    A->piece = static_cast<uint32_t>(piece);
    A->slices = std::max(kSliceTokens / A->tokens_up, 1u);
    Places p = {};
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += up(bytes, 256);
        return here;
    };
    p.state = take(sizeof(State));
    p.index = take(n * 4);
    p.rows = take(n * sizeof(Row));
    p.losses = take(n * 8);
    p.picked = take(n * 4);
    p.parts = take(n * A->tiles * sizeof(float2));
    p.hidden = take(static_cast<uint64_t>(A->tokens_up) * A->stride);
    // (never less for more tokens, entries or elements, whatever the pieces come to)
    const uint64_t whole = up(b.vocab, kTile);
    auto piece_of = [&](uint64_t rows) { return std::max(std::min(rows * whole, kPieceElements), rows * kTile) * 2; };
    p.weight = take(packed ? piece_of(width_up) : 0);
    if (grad) {
        p.grad = take(piece_of(A->tokens_up));
        p.dh = take(static_cast<uint64_t>(std::max(A->tokens_up, kSliceTokens)) * width_up * 4);
    }
    p.bytes = at;
    return p;
}

template <bool BF16, int BM>
hipError_t launch(const HeadArgs& A, hipStream_t stream)
{
    const uint32_t n = static_cast<uint32_t>(A.b.n_tokens), vocab = static_cast<uint32_t>(A.b.vocab), tiles_m = A.tokens_up / BM;
    const uint32_t tiles_d = (A.stride / 2 + kTile - 1) / kTile;
    hipLaunchKernelGGL(head_select_kernel, dim3(1), dim3(kSelectThreads), 0, stream, A);
    hipLaunchKernelGGL(head_gather_kernel, dim3(std::min(A.tokens_up, 4096u)), dim3(256), 0, stream, A);
    auto pieces = [&](auto&& fn) {
        for (uint64_t first = 0; first < vocab; first += A.piece) {
            const uint32_t m = static_cast<uint32_t>(std::min<uint64_t>(A.piece, vocab - first));
            fn(static_cast<uint32_t>(first), m, (m + kTile - 1) / kTile);
        }
    };
    auto pack = [&](uint32_t first, uint32_t m) {
        if (A.weight) hipLaunchKernelGGL(head_pack_kernel, dim3(std::min(m, 8192u)), dim3(256), 0, stream, A, first, m);
    };
    pieces([&](uint32_t first, uint32_t m, uint32_t tiles) {
        pack(first, m);
        hipLaunchKernelGGL((head_logits_kernel<BF16, BM, false>), dim3(tiles * tiles_m), dim3(kProductThreads), 0, stream, A, first, m);
    });
    hipLaunchKernelGGL(head_finish_kernel<BF16>, dim3(n / 4 + 1), dim3(256), 0, stream, A);
    hipLaunchKernelGGL(head_sum_kernel, dim3(1), dim3(kSelectThreads), 0, stream, A, A.b.loss_scale * (BF16 ? 1.f : 0x1p-14f));
    if (!A.dhidden && !A.dweight) return hipGetLastError();
    const bool one = A.piece >= vocab;
    pieces([&](uint32_t first, uint32_t m, uint32_t tiles) {
        if (!one) pack(first, m);
        hipLaunchKernelGGL((head_logits_kernel<BF16, BM, true>), dim3(tiles * tiles_m), dim3(kProductThreads), 0, stream, A, first, m);
        if (A.dhidden)
            hipLaunchKernelGGL((head_dhidden_kernel<BF16, BM>), dim3(tiles_m * tiles_d * A.slices), dim3(kProductThreads), 0, stream, A, first, m);
        if (A.dweight) hipLaunchKernelGGL(head_dweight_kernel<BF16>, dim3(tiles * tiles_d), dim3(kProductThreads), 0, stream, A, first, m);
    });
    if (A.dhidden) hipLaunchKernelGGL(head_put_kernel<BF16>, dim3(std::min(n + 1, 4096u)), dim3(256), 0, stream, A);
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
    A.rows = reinterpret_cast<Row*>(w + p.rows);
    A.losses = reinterpret_cast<double*>(w + p.losses);
    A.picked = reinterpret_cast<float*>(w + p.picked);
    A.parts = reinterpret_cast<float2*>(w + p.parts);
    A.hidden = w + p.hidden;
    A.weight = weight_as_it_is(b) ? nullptr : w + p.weight;
    A.grad = w + p.grad;
    A.dh = reinterpret_cast<float*>(w + p.dh);
    if (b.dtype == FF_BF16) return b.n_tokens <= kFewTokens ? launch<true, 64>(A, stream) : launch<true, 256>(A, stream);
    return b.n_tokens <= kFewTokens ? launch<false, 64>(A, stream) : launch<false, 256>(A, stream);
}

}  // namespace ffsnap
