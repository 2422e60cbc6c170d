// What embed.hip, norm.hip and rows.h take from the library's header of this name, for the CPU.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#define FF_GLOBAL

namespace ffsnap {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
constexpr int kWaveSize = 64;

template <class T>
T* as_global(T* p) { return p; }
template <class V>
V table_entry(const V* table, const uint32_t i) { return table[i]; }
template <class Fn, int... Is>
void static_for_impl(Fn&& fn, std::integer_sequence<int, Is...>) { (fn(std::integral_constant<int, Is>{}), ...); }
template <int N, class Fn>
void static_for(Fn&& fn) { static_for_impl(fn, std::make_integer_sequence<int, N>{}); }

}  // namespace ffsnap
