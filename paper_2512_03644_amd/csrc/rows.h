// Rows of 16- and 32-bit floats, eight elements to a lane: at any element's address, and with any number of elements.
#pragma once
#include "fold.h"
#include "../../include/ffsnap.h"

namespace ffsnap {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8v __attribute__((ext_vector_type(8)));

constexpr int kLaneItems = 8;

// Outputs of so many bytes go past the caches: of what is larger than all L2s together little is there when it is read next.  (Us, through them / past
// them: layer norm of 16,384 rows of 8192 bf16 elements, forward and backward, 256 and 238, with the inputs of the latter past them too 233; 16,384 embedded tokens of
// 8192 92 and 84.  Inputs of 3001 rows of 1003 fp32 elements past them 24.2 where 21.7 are taken.)
constexpr uint64_t kPastBytes = 32ull << 20;

// WHOLE: rows are multiples of eight elements.  (What others need at their ends costs all rows registers: layer norm of 16,384 x 8192 bf16 elements, forward
// and backward, 248 us where they are treated like the others, 231 so; 16,384 embedded tokens of 8192 85 and 82.)
template <uint32_t DTYPE, bool WHOLE>
struct Items {
    static constexpr uint32_t kBytes = DTYPE == FF_F32 ? 4 : 2;
    using Wide = Items<FF_F32, WHOLE>;  // of sums

    // Where the eight elements lie that a lane holds for its [at, at + 8) of a row of `width`, at < width: those, or, where the row has fewer, its last
    // eight, which it holds in part for another lane.  (Element by element, a lane would wait for each row's in turn, and its wavefront with it: 3001 rows of
    // 257 fp32 elements added to a table's gradient 17.4 us, so 12.5.)  A row of less than eight is filled up with its last one.
    static __device__ __forceinline__ uint32_t window(uint32_t at, uint32_t width)
    {
        return WHOLE || at + kLaneItems <= width || width < kLaneItems ? at : width - kLaneItems;
    }
    // Is element i of those the lane's own?
    static __device__ __forceinline__ bool owns(uint32_t i, uint32_t at, uint32_t width)
    {
        return WHOLE || (window(at, width) + i >= at && window(at, width) + i < width);
    }
    // Zeros for those that are not.
    static __device__ __forceinline__ f32x8 cut(f32x8 v, uint32_t at, uint32_t width)
    {
        if (!WHOLE && at + kLaneItems > width)
            for (uint32_t i = 0; i < kLaneItems; i++) v[i] = owns(i, at, width) ? v[i] : 0.f;
        return v;
    }

    static __device__ __forceinline__ float one(const uint8_t* p)
    {
        if constexpr (DTYPE == FF_F32) return *(const FF_GLOBAL float*)p;
        else if constexpr (DTYPE == FF_BF16) return __builtin_bit_cast(float, static_cast<uint32_t>(*(const FF_GLOBAL uint16_t*)p) << 16);
        else return static_cast<float>(*(const FF_GLOBAL _Float16*)p);
    }
    static __device__ __forceinline__ void put(uint8_t* p, float v)
    {
        if constexpr (DTYPE == FF_F32) *(FF_GLOBAL float*)p = v;
        else if constexpr (DTYPE == FF_BF16) *(FF_GLOBAL __bf16*)p = static_cast<__bf16>(v);
        else *(FF_GLOBAL _Float16*)p = static_cast<_Float16>(v);
    }
    // What eight elements lie in memory as: values are held like this until they are used.
    struct Held {
        u32x4 w[kBytes / 2];
    };
    static __device__ __forceinline__ f32x8 wide(const Held& h)
    {
        f32x8 v;
        if constexpr (DTYPE == FF_F32) {
            v = __builtin_bit_cast(f32x8, h);
        } else if constexpr (DTYPE == FF_BF16) {
            for (int i = 0; i < 8; i++) {
                const uint32_t both = h.w[0][i / 2];
                v[i] = __builtin_bit_cast(float, i % 2 ? both & 0xFFFF0000u : both << 16);
            }
        } else {
            v = __builtin_convertvector(__builtin_bit_cast(f16x8v, h.w[0]), f32x8);
        }
        return v;
    }
    static __device__ __forceinline__ Held narrow(f32x8 v)
    {
        Held h;
        if constexpr (DTYPE == FF_F32) {
            h = __builtin_bit_cast(Held, v);
        } else if constexpr (DTYPE == FF_BF16) {
            h.w[0] = __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8v));
        } else {
            h.w[0] = __builtin_bit_cast(u32x4, __builtin_convertvector(v, f16x8v));
        }
        return h;
    }
    // A lane's elements [at, at + 8) of a row of `width`, at < width.  PAST: not to be kept in the caches.
    template <bool PAST = false>
    static __device__ __forceinline__ Held load(const uint8_t* row, uint32_t at, uint32_t width)
    {
        const uint8_t* const p = row + static_cast<uint64_t>(window(at, width)) * kBytes;
        if (WHOLE || width >= kLaneItems) {
            Held h;
            for (uint32_t i = 0; i < kBytes / 2; i++) {
                const auto* const q = (const FF_GLOBAL u32x4_a2*)p + i;
                h.w[i] = PAST ? __builtin_nontemporal_load(q) : *q;
            }
            return h;
        }
        f32x8 v;
        for (uint32_t i = 0; i < kLaneItems; i++) v[i] = one(p + (i < width ? i : width - 1) * kBytes);
        return narrow(v);
    }
    template <bool PAST = false>
    static __device__ __forceinline__ void store(uint8_t* row, uint32_t at, uint32_t width, const Held& h)
    {
        uint8_t* const p = row + static_cast<uint64_t>(window(at, width)) * kBytes;
        if (WHOLE || at + kLaneItems <= width) {
            for (uint32_t i = 0; i < kBytes / 2; i++) {
                auto* const q = (FF_GLOBAL u32x4_a2*)p + i;
                if (PAST) __builtin_nontemporal_store(h.w[i], q);
                else *q = h.w[i];
            }
            return;
        }
        const f32x8 v = wide(h);
        for (uint32_t i = 0; i < kLaneItems; i++)
            if (owns(i, at, width)) put(p + i * kBytes, v[i]);
    }
};

// fn(the items) of rows of this width.
template <class Fn>
void with_items(uint32_t dtype, uint64_t width, Fn&& fn)
{
    const bool whole = width % kLaneItems == 0;
    if (dtype == FF_BF16) whole ? fn(Items<FF_BF16, true>{}) : fn(Items<FF_BF16, false>{});
    else if (dtype == FF_F16) whole ? fn(Items<FF_F16, true>{}) : fn(Items<FF_F16, false>{});
    else whole ? fn(Items<FF_F32, true>{}) : fn(Items<FF_F32, false>{});
}

}  // namespace ffsnap
