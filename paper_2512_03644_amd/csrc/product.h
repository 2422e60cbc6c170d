// Matrix products of 16-bit operands on gfx950's matrix instructions, 32-bit sums, as building blocks of kernels with epilogues
// of their own: C[m][n] = sum over k of A[m][k] B[n][k], a tile of BM x 256 to a workgroup of 512 threads.
//
// Either operand lies in memory with k contiguous (kAlongK: a row of m or n holds its k) or with m, n contiguous (kAcrossK:
// a row holds one k).  A step is 64 k: 16 bytes a lane go from memory straight into LDS, into one of two buffers, while the
// products of the other are made; the order in which a lane fetches the 16-byte pieces of a row is permuted, so that the
// reads of fragments are spread over all banks though LDS is written in lane order.  kAlongK fragments are plain 16-byte reads;
// kAcrossK ones come transposed (ds_read_b64_tr_b16), four k of one column to a lane.
//
// In a step a wavefront has the first half's fragments in registers; it asks for the second half's, multiplies the first's, meets the
// others -- all fragments of this buffer are read then, and the next buffer has arrived -- asks memory for the step after the next
// and LDS for the first fragments of the next, and multiplies the second half's: one barrier a step, and always 32 products
// between a read and its use.
//
// What bounds it: power, and the matrix instructions.  In logits of 3686 x 128,256 x 8192 (bf16, 6.6 ms with their epilogue, 1.18 PFLOP/s; both gradients' products 1.30; a library's product of
// that form reaches 1.55 alone, of the gradients' forms 1.35 and 1.17) the matrix units are at work for 62 % of the cycles, at 1.88 GHz, in the gradients for 68 % at 1.84; there LDS
// works for 44 % of the cycles, 17 % of them all in conflicts between banks (logits: 24 and 0.1).  Four wavefronts with parts of 128 x 128 (a third fewer reads of LDS) 2 % slower; loads earlier or later among the
// products, bands of 4 or 16 tiles, strides off the powers of two, a raised priority, reads sooner: within 2 % either way, or worse.
#pragma once
#include "fold.h"

namespace ffsnap {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

enum Layout { kAlongK, kAcrossK };
constexpr int kProductThreads = 512, kProductWaves = 8, kStepK = 64;

// Where an operand's tile lies.
struct OperandTile {
    const uint8_t* base;  // of the tile's first row (kAlongK) or column (kAcrossK), at k = 0 of the product
    uint64_t stride;      // bytes between rows; times 256 below 2^32
    uint32_t valid;       // kAlongK: rows that are there; kAcrossK: columns, a multiple of 8.  Others repeat the last.
    uint32_t k_valid;     // kAlongK: a multiple of 8, zeros stand for what is behind; kAcrossK: rows behind repeat the last
};

template <Layout LAYOUT, int SIZE, int WAVES = kProductWaves>
struct Operand {
    static constexpr int kLoads = SIZE / 8 / WAVES;  // of a wavefront a step, 1 KiB each
    // What a load brings lies together; between those of a kAcrossK tile, two rows each, 64 bytes are left free, and in odd rows the two
    // halves of every 64 bytes are exchanged: the four rows that a transposing read of 16 lanes takes are in different banks (not those of all 64 lanes).
    static constexpr uint32_t kChunk = LAYOUT == kAlongK ? 1024 : 1024 + 64;
    static constexpr uint32_t kBytes = WAVES * kLoads * kChunk;
    static constexpr uint32_t kRowBytes = LAYOUT == kAlongK ? kStepK * 2 : SIZE * 2;
    static_assert(LAYOUT == kAlongK || SIZE == 256, "a row is 32 pieces of 16 bytes");

    const uint8_t* base;
    uint64_t step;
    uint32_t at[kLoads];

    // A load's row of the tile, and the piece of that row, by lane.
    static __device__ __forceinline__ uint32_t row_of(int i, int wave, int lane)
    {
        const int load = wave * kLoads + i;
        return LAYOUT == kAlongK ? 8 * load + lane / 8 : 2 * load + lane / 32;
    }
    static __device__ __forceinline__ uint32_t piece_of(int i, int wave, int lane)
    {
        return LAYOUT == kAlongK ? (lane & 7) ^ (lane >> 3) : (lane & 31) ^ (lane >> 5) << 1;
    }
    __device__ __forceinline__ void init(const OperandTile& t, int wave, int lane)
    {
        base = t.base;
        step = LAYOUT == kAlongK ? kStepK * 2 : kStepK * t.stride;
        for (int i = 0; i < kLoads; i++) {
            uint32_t row = row_of(i, wave, lane), piece = piece_of(i, wave, lane);
            if (LAYOUT == kAlongK) row = row < t.valid ? row : t.valid - 1;
            if (LAYOUT == kAcrossK) piece = piece * 8 < t.valid ? piece : t.valid / 8 - 1;
            at[i] = row * static_cast<uint32_t>(t.stride) + piece * 16;
        }
    }
    // Load i of step k of the product, into a buffer: 16 bytes a lane, to consecutive places.  (By hand: behind the builtin for this the compiler waits
    // for all of them in front of any read of LDS, as it cannot tell the two buffers apart.  There is no result in registers; `meet` waits.)
    __device__ __forceinline__ void fetch(int i, uint32_t k, FF_LDS uint8_t* buffer, int wave) const
    {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :
                     : "s"(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(buffer + (wave * kLoads + i) * kChunk))), "v"(at[i]), "s"(base + k * step)
                     : "m0");
    }
    // In front of the fetch of a last step of which only a part is there.
    __device__ __forceinline__ void cut(const OperandTile& t, uint32_t k, int wave, int lane)
    {
        const uint32_t left = t.k_valid - k * kStepK;
        if (left >= kStepK) return;
        for (int i = 0; i < kLoads; i++) {
            const uint32_t row = row_of(i, wave, lane), piece = piece_of(i, wave, lane);
            if (LAYOUT == kAlongK && piece * 8 >= left) at[i] -= (piece - (left / 8 - 1)) * 16;
            if (LAYOUT == kAcrossK && row >= left) at[i] -= (row - (left - 1)) * static_cast<uint32_t>(step / kStepK);
        }
    }
    // And when it has arrived: zeros for what is not there.
    static __device__ __forceinline__ void clear(const OperandTile& t, uint32_t k, FF_LDS uint8_t* buffer)
    {
        const uint32_t left = t.k_valid - k * kStepK;
        if (LAYOUT != kAlongK || left >= kStepK) return;
        for (uint32_t i = threadIdx.x; i < SIZE * 8; i += WAVES * kWaveSize) {
            const uint32_t row = i / 8, piece = i % 8;
            if (piece * 8 >= left) *(FF_LDS u32x4*)(buffer + row * kRowBytes + (piece ^ (row & 7)) * 16) = u32x4{0, 0, 0, 0};
        }
    }
    // Fragment of 16 rows (columns) from `first` on for the step's 32 k from 32 * half on: lane l has row l % 16, k 8 (l / 16) + 0..7.
    static __device__ __forceinline__ s16x8 fragment(const FF_LDS uint8_t* buffer, int first, int half, int lane)
    {
        if constexpr (LAYOUT == kAlongK) {
            const uint32_t piece = (half * 4 + lane / 16) ^ (lane & 7);
            return *(const FF_LDS s16x8*)(buffer + (lane % 16) * kRowBytes + piece * 16 + first * kRowBytes);
        } else {
            const uint32_t row = 8 * (lane / 16) + (lane % 16) / 4, odd = row & 1;  // and row + 4
            const uint32_t at = row / 2 * kChunk + odd * kRowBytes + (lane % 4) * 8 + (first / 16 % 2 ? 1 - odd : odd) * 32;
            const FF_LDS uint8_t* const p = buffer + at + half * 16 * kChunk + first / 32 * 64;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FF_LDS s16x4*)p);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FF_LDS s16x4*)(p + 2 * kChunk));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

template <bool BF16>
__device__ __forceinline__ f32x4 multiply(s16x8 a, s16x8 b, f32x4 c)
{
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Four values rounded to the nearest 16-bit ones.
template <bool BF16>
__device__ __forceinline__ u32x2 to_half(f32x4 v)
{
    if constexpr (BF16) return __builtin_bit_cast(u32x2, __builtin_convertvector(v, bf16x4));
    else return __builtin_bit_cast(u32x2, __builtin_convertvector(v, f16x4));
}

// The eight wavefronts share a tile of BM x 256 as 2 x 4 parts of 128 x 64, or 1 x 8 parts of 64 x 32.
template <int BM>
struct Share {
    static constexpr int kAcross = BM == 256 ? 4 : 8;  // wavefronts along n
    static constexpr int kM = BM == 256 ? 8 : 4, kN = BM == 256 ? 4 : 2;  // fragments of a wavefront
};

template <int BM, Layout A_LAYOUT, Layout B_LAYOUT>
constexpr uint32_t kProductLds = 2 * (Operand<A_LAYOUT, BM>::kBytes + Operand<B_LAYOUT, 256>::kBytes);

// The sums of a wavefront's part over steps [k_from, k_to): fragment (i, j), lane l, element e is row 16 i + l % 16,
// column 16 j + 4 (l / 16) + e of the part (operands in exchanged places: a lane's elements follow each other along n).
// The last step of the whole product is `end` if a part of it is missing.  lds: kProductLds<...>.
template <bool BF16, int BM, Layout A_LAYOUT, Layout B_LAYOUT>
__device__ __forceinline__ void product(const OperandTile& a_tile, const OperandTile& b_tile, uint32_t k_from, uint32_t k_to, uint32_t end,
                                        FF_LDS uint8_t* lds, f32x4 (&sum)[Share<BM>::kM][Share<BM>::kN])
{
    using S = Share<BM>;
    using A = Operand<A_LAYOUT, BM>;
    using B = Operand<B_LAYOUT, 256>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize), lane = threadIdx.x % kWaveSize;
    for (int i = 0; i < S::kM; i++)
        for (int j = 0; j < S::kN; j++) sum[i][j] = f32x4{0, 0, 0, 0};
    if (k_from >= k_to) return;
    A a;
    B b;
    a.init(a_tile, wave, lane);
    b.init(b_tile, wave, lane);
    const int m0 = (wave / S::kAcross) * (16 * S::kM), n0 = (wave % S::kAcross) * (16 * S::kN);
    constexpr uint32_t kBuffer = A::kBytes + B::kBytes;
    auto cut = [&](uint32_t k) {
        if (k != end) return;
        a.cut(a_tile, k, wave, lane);
        b.cut(b_tile, k, wave, lane);
    };
    // load i of a step, of A's and B's
    auto fetch = [&](int i, uint32_t k, FF_LDS uint8_t* buffer) {
        if (i < A::kLoads) a.fetch(i, k, buffer, wave);
        else if (i < A::kLoads + B::kLoads) b.fetch(i - A::kLoads, k, buffer + A::kBytes, wave);
    };
    auto fetch_all = [&](uint32_t k, FF_LDS uint8_t* buffer) {
        cut(k);
        static_for<A::kLoads + B::kLoads>([&](auto i) { fetch(i, k, buffer); });
    };
    struct Half {
        s16x8 a[S::kM], b[S::kN];
    } first, second;
    // fragment i of a half, in the order in which they are used
    auto read = [&](auto i, Half& h, const FF_LDS uint8_t* buffer, int half) {
        if constexpr (i < S::kN) h.b[int(i)] = B::fragment(buffer + A::kBytes, n0 + 16 * i, half, lane);
        else if constexpr (i < S::kN + S::kM) h.a[i - S::kN] = A::fragment(buffer, m0 + 16 * (i - S::kN), half, lane);
    };
    // The products of a half, and between them the reads of the next one and the loads of a step.
    constexpr int kGroups = S::kM, kReads = (S::kN + S::kM + kGroups - 3) / (kGroups - 2), kFetches = (A::kLoads + B::kLoads + kGroups - 1) / kGroups;
    auto multiply_all = [&](const Half& h, Half& to, const FF_LDS uint8_t* from, int half, uint32_t k, FF_LDS uint8_t* into, auto fetches) {
        static_for<kGroups>([&](auto g) {
            static_for<S::kN>([&](auto j) { sum[int(g)][int(j)] = multiply<BF16>(h.b[int(j)], h.a[int(g)], sum[int(g)][int(j)]); });
            static_for<kReads>([&](auto i) { read(std::integral_constant<int, g * kReads + i>{}, to, from, half); });
            if constexpr (fetches) static_for<kFetches>([&](auto i) { fetch(g * kFetches + i, k, into); });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // all of this wavefront's loads are here, and all it has read from LDS
    auto meet = [&] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto clear = [&](uint32_t k, FF_LDS uint8_t* buffer) {
        if (k != end) return;
        A::clear(a_tile, k, buffer);
        B::clear(b_tile, k, buffer + A::kBytes);
        meet();
    };
    uint32_t mine = 0;  // the buffer of the step
    fetch_all(k_from, lds);
    meet();
    clear(k_from, lds);
    if (k_from + 1 < k_to) fetch_all(k_from + 1, lds + kBuffer);
    static_for<S::kN + S::kM>([&](auto i) { read(i, first, lds, 0); });
    // (behind the last step there is nothing to read, and what is read is not used)
    auto step = [&](uint32_t now, auto fetches) {
        FF_LDS uint8_t *const here = lds + mine, *const next = lds + (kBuffer - mine);
        multiply_all(first, second, here, 1, 0, here, std::false_type{});
        meet();
        if (now + 1 == end) clear(end, next);
        if (fetches && now + 2 == end) cut(end);
        multiply_all(second, first, next, 0, now + 2, here, fetches);
        mine = kBuffer - mine;
    };
    uint32_t k = k_from;
    for (; k + 2 < k_to; k++) step(k, std::true_type{});
    for (; k < k_to; k++) step(k, std::false_type{});
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");  // LDS is free
}

// A wavefront's part on its way to memory by rows: a lane's elements are four of a row, 16 rows apart in place; through LDS they become 16 bytes of
// one row, 16 N columns of it side by side.  to16(i, j): the four rounded elements of fragment (i, j); fn(row, column, eight elements).
// Stores of 32 bytes of 16 rows instead: 1.05 GB of gradient of few tokens took 600 us.
template <int M, int N>
struct RowsByLds {
    static constexpr int kAtOnce = M < 4 ? M : 4, kLanes = 2 * N;
    static constexpr uint32_t kPitch = 32 * N + 16, kBytes = 16 * kAtOnce * kPitch;  // of a wavefront
    template <class To16, class Fn>
    static __device__ __forceinline__ void pass(FF_LDS uint8_t* lds, To16&& to16, Fn&& fn)
    {
        const uint32_t lane = threadIdx.x % kWaveSize;
        FF_LDS uint8_t* const mine = lds + threadIdx.x / kWaveSize * kBytes;
        static_for<M / kAtOnce>([&](auto h) {
            static_for<kAtOnce>([&](auto i) {
                static_for<N>([&](auto j) {
                    *(FF_LDS u32x2*)(mine + (16 * i + lane % 16) * kPitch + 32 * j + lane / 16 * 8) =
                        to16(std::integral_constant<int, h * kAtOnce + i>{}, j);
                });
            });
            static_for<kAtOnce * 16 * kLanes / kWaveSize>([&](auto k) {
                const uint32_t at = k * kWaveSize + lane, row = at / kLanes, piece = at % kLanes;
                fn(h * kAtOnce * 16 + row, piece * 8, *(const FF_LDS u32x4*)(mine + row * kPitch + piece * 16));
            });
        });
    }
};

// Tiles in an order in which those that run at one time share operands: bands of 8 tiles along m, within them along n; the
// workgroups of an XCD take 32 in a row.
constexpr uint32_t kBand = 8, kXcdTiles = 32;
__device__ __forceinline__ void tile_at(uint32_t tile, uint32_t tiles_m, uint32_t tiles_n, uint32_t* m, uint32_t* n)
{
    const uint32_t band = tile / (kBand * tiles_n), first = band * kBand, in = tile - first * tiles_n;
    const uint32_t high = tiles_m - first < kBand ? tiles_m - first : kBand;
    *n = in / high;
    *m = first + in - *n * high;
}

}  // namespace ffsnap
