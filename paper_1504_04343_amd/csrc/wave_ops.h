// Reductions over a wave without LDS: within rows of 16 lanes by data-parallel moves, over the rows by lane swaps.
#pragma once
#include <type_traits>

#include "cct_internal.h"

namespace cct {
namespace {

// `join` of 16 neighbouring lanes' values, in all of them.
template <class F>
__device__ __forceinline__ unsigned row_reduce(unsigned v, F join) {
  auto other = [](unsigned x, auto how) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, decltype(how)::value, 0xf, 0xf, true); };
  v = join(v, other(v, std::integral_constant<int, 0xb1>()));          // neighbours
  v = join(v, other(v, std::integral_constant<int, 0x4e>()));          // pairs of them
  v = join(v, other(v, std::integral_constant<int, 0x141>()));         // fours of a half row, mirrored
  return join(v, other(v, std::integral_constant<int, 0x140>()));      // eights of a row, mirrored
}
// Of a wave's lanes.
template <class F>
__device__ __forceinline__ unsigned wave_reduce(unsigned v, F join) {
  v = row_reduce(v, join);
  const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const unsigned r0 = rows[0], r1 = rows[1];
  const unsigned h = join(r0, r1);
  const auto halves = __builtin_amdgcn_permlane32_swap(h, h, false, false);
  const unsigned h0 = halves[0], h1 = halves[1];
  return join(h0, h1);
}

__device__ __forceinline__ unsigned add_floats(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float row_sum(float v) {
  return __builtin_bit_cast(float, row_reduce(__builtin_bit_cast(unsigned, v), [](unsigned a, unsigned b) { return add_floats(a, b); }));
}
__device__ __forceinline__ float wave_sum(float v) {
  return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(unsigned, v), [](unsigned a, unsigned b) { return add_floats(a, b); }));
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
  return wave_reduce(v, [](unsigned a, unsigned b) { return a > b ? a : b; });
}
__device__ __forceinline__ unsigned wave_min(unsigned v) {
  return wave_reduce(v, [](unsigned a, unsigned b) { return a < b ? a : b; });
}

}  // namespace
}  // namespace cct
