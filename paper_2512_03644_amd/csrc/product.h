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
    const uint8_t* base;   // of the tile's first row (kAlongK) or column (kAcrossK), at k = 0 of the product
    uint64_t stride;       // bytes between rows; times 256 below 2^32
    uint32_t valid;        // kAlongK: rows that are there; kAcrossK: columns, a multiple of 8.  Others repeat the last.
    uint32_t k_valid;      // kAlongK: a multiple of 8, `zeros` stand for what is behind; kAcrossK: rows behind repeat the last
    const uint8_t* zeros;  // 16 bytes
};

// What spreads the rows of a kAcrossK tile over the banks: rows that one transposing read takes differ in it.
__device__ __forceinline__ uint32_t row_spread(uint32_t k) { return (k & 3) | (k >> 1 & 12); }

template <Layout LAYOUT, int SIZE>
struct Operand {
    static constexpr int kLoads = SIZE / 64;            // of a wavefront a step, 1 KiB each
    static constexpr uint32_t kBytes = SIZE * kStepK * 2;
    static constexpr uint32_t kRowBytes = LAYOUT == kAlongK ? kStepK * 2 : SIZE * 2;
    static_assert(LAYOUT == kAlongK || SIZE == 256, "a row is 32 pieces of 16 bytes");

    const uint8_t* base;
    uint64_t step;
    uint32_t at[kLoads];

    // A load's row of the tile, and the piece of that row, by lane.
    static __device__ __forceinline__ uint32_t row_of(int i, int wave, int lane)
    {
        return LAYOUT == kAlongK ? wave * (SIZE / kProductWaves) + 8 * i + lane / 8 : wave * 8 + 2 * i + lane / 32;
    }
    static __device__ __forceinline__ uint32_t piece_of(int i, int wave, int lane)
    {
        return LAYOUT == kAlongK ? (lane & 7) ^ (lane >> 3) : (lane & 31) ^ row_spread(row_of(i, wave, lane)) << 1;
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
    static __device__ __forceinline__ void load(const uint8_t* p, FF_LDS uint8_t* to)
    {
        __builtin_amdgcn_global_load_lds((const FF_GLOBAL void*)p, (FF_LDS void*)to, 16, 0, 0);
    }
    // Step k of the product, into a buffer.
    __device__ __forceinline__ void fetch(uint32_t k, FF_LDS uint8_t* buffer, int wave) const
    {
        const uint8_t* const p = base + k * step;
        for (int i = 0; i < kLoads; i++) load(p + at[i], buffer + (wave * kLoads + i) * 1024);
    }
    // The same for a step of which only a part is there.
    __device__ __forceinline__ void fetch_end(const OperandTile& t, uint32_t k, FF_LDS uint8_t* buffer, int wave, int lane) const
    {
        const uint8_t* const p = base + k * step;
        const uint32_t left = t.k_valid - k * kStepK;
        for (int i = 0; i < kLoads; i++) {
            const uint8_t* q = p + at[i];
            const uint32_t row = row_of(i, wave, lane);
            if (LAYOUT == kAlongK && piece_of(i, wave, lane) * 8 >= left) q = t.zeros;
            if (LAYOUT == kAcrossK && row >= left) q -= (row - (left - 1)) * t.stride;
            load(q, buffer + (wave * kLoads + i) * 1024);
        }
    }
    // Fragment of 16 rows (columns) from `first` on for the step's 32 k from 32 * half on: lane l has row l % 16, k 8 (l / 16) + 0..7.
    static __device__ __forceinline__ s16x8 fragment(const FF_LDS uint8_t* buffer, int first, int half, int lane)
    {
        if constexpr (LAYOUT == kAlongK) {
            const uint32_t piece = (half * 4 + lane / 16) ^ (lane & 7);
            return *(const FF_LDS s16x8*)(buffer + (lane % 16) * kRowBytes + piece * 16 + first * kRowBytes);
        } else {
            const uint32_t row = 8 * (lane / 16) + (lane % 16) / 4;  // and row + 4
            const uint32_t unit = (first / 16) ^ row_spread(row);
            const FF_LDS uint8_t* const p = buffer + (half * 32 + row) * kRowBytes + unit * 32 + (lane % 4) * 8;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FF_LDS s16x4*)p);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FF_LDS s16x4*)(p + 4 * kRowBytes));
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
    static constexpr uint32_t kLdsBytes = 2 * (BM + 256) * kStepK * 2;
};

// The sums of a wavefront's part over steps [k_from, k_to): fragment (i, j), lane l, element e is row 16 i + l % 16,
// column 16 j + 4 (l / 16) + e of the part (operands in exchanged places: a lane's elements follow each other along n).
// The last step of the whole product is `end` if a part of it is missing.  lds: Share<BM>::kLdsBytes.
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
    FF_LDS uint8_t* const buffers[2] = {lds, lds + A::kBytes + B::kBytes};
    auto fetch = [&](uint32_t k, FF_LDS uint8_t* buffer) {
        if (k == end) {
            a.fetch_end(a_tile, k, buffer, wave, lane);
            b.fetch_end(b_tile, k, buffer + A::kBytes, wave, lane);
        } else {
            a.fetch(k, buffer, wave);
            b.fetch(k, buffer + A::kBytes, wave);
        }
    };
    struct Half {
        s16x8 a[S::kM], b[S::kN];
    } first, second;
    auto read = [&](Half& h, const FF_LDS uint8_t* buffer, int half) {
        for (int j = 0; j < S::kN; j++) h.b[j] = B::fragment(buffer + A::kBytes, n0 + 16 * j, half, lane);
        for (int i = 0; i < S::kM; i++) h.a[i] = A::fragment(buffer, m0 + 16 * i, half, lane);
    };
    auto multiply_all = [&](const Half& h) {
        for (int i = 0; i < S::kM; i++)
            for (int j = 0; j < S::kN; j++) sum[i][j] = multiply<BF16>(h.b[j], h.a[i], sum[i][j]);
    };
    // all of this wavefront's loads are here, and all it has read from LDS
    auto meet = [&] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    fetch(k_from, buffers[0]);
    meet();
    if (k_from + 1 < k_to) fetch(k_from + 1, buffers[1]);
    read(first, buffers[0], 0);
    for (uint32_t k = k_from; k < k_to; k += 2) {
        static_for<2>([&](auto which) {
            const uint32_t now = k + which;
            if (now < k_to) {
                FF_LDS uint8_t* const mine = buffers[int(which)];
                FF_LDS uint8_t* const next = buffers[1 - int(which)];
                read(second, mine, 1);
                multiply_all(first);
                meet();
                if (now + 2 < k_to) fetch(now + 2, mine);
                if (now + 1 < k_to) read(first, next, 0);
                multiply_all(second);
            }
        });
    }
}

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
