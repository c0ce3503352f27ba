// A step of the contraction of a product of few rows: 64 bytes of 16 rows of each operand, from memory straight into the registers
// that the matrix cores take.
#pragma once
#include "ff_tile.h"

namespace cct {
namespace {

template <int TYPE>
struct Step {  // 16-bit types
  typedef s16x8 V;
  static constexpr int CH = 8, K = 32;  // values per lane, per step
  static __device__ __forceinline__ V load(const void* p, long long at) {
    typedef s16x8 U __attribute__((aligned(2)));
    return *(const U*)((const short*)p + at);
  }
  // Eight values at any even address, from the four words that hold the first seven and the eighth by itself.  The first word's
  // lower half may lie in front of the value, in the same four bytes and so in the same page.
  static __device__ __forceinline__ V load_odd(const void* p, long long at) {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    typedef i32x4 U __attribute__((aligned(4)));
    const unsigned long long a = (unsigned long long)((const short*)p + at);
    const i32x4 d = *(const U*)(a & ~3ull);
    const int last = ((const unsigned short*)p)[at + 7], by = a & 2 ? 16 : 0;
    const i32x4 v = {(int)__builtin_amdgcn_alignbit(d[1], d[0], by), (int)__builtin_amdgcn_alignbit(d[2], d[1], by),
                     (int)__builtin_amdgcn_alignbit(d[3], d[2], by), by ? (int)__builtin_amdgcn_alignbit(last, d[3], 16) : d[3]};
    return __builtin_bit_cast(V, v);
  }
  static __device__ __forceinline__ V part(const void* p, long long at, int n) {
    V v = {};
#pragma unroll
    for (int e = 0; e < CH; ++e)
      if (e < n) v[e] = ((const short*)p)[at + e];
    return v;
  }
  static __device__ __forceinline__ f32x4 mfma(V w, V x, f32x4 c) { return tile_mfma<TYPE>(w, x, c); }
};
template <>
struct Step<CCT_TYPE_F32> {
  typedef f32x4 V;
  static constexpr int CH = 4, K = 16;
  static __device__ __forceinline__ V load(const void* p, long long at) {
    typedef f32x4 U __attribute__((aligned(4)));
    return *(const U*)((const float*)p + at);
  }
  static __device__ __forceinline__ V part(const void* p, long long at, int n) {
    V v = {};
#pragma unroll
    for (int e = 0; e < CH; ++e)
      if (e < n) v[e] = ((const float*)p)[at + e];
    return v;
  }
  static __device__ __forceinline__ f32x4 mfma(V w, V x, f32x4 c) {
#pragma unroll
    for (int e = 0; e < CH; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], c, 0, 0, 0);
    return c;
  }
};

}  // namespace
}  // namespace cct
