// The types of the feed-forward operators' tensors: values in registers are fp32, 8 consecutive ones at a time in memory.
#pragma once
#include "cct_internal.h"

namespace cct {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// What a type is in memory, and 8 of its values at any address that is a multiple of one of them: gfx950 loads and stores
// 16 bytes at any address, the alignment only tells the compiler so.
template <int TYPE>
struct Number;
template <>
struct Number<CCT_TYPE_F32> {
  typedef float T;
  typedef f32x8 V8;
  typedef f32x8 __attribute__((aligned(4))) U8;
};
template <>
struct Number<CCT_TYPE_BF16> {
  typedef __bf16 T;
  typedef bf16x8 V8;
  typedef bf16x8 __attribute__((aligned(2))) U8;
};
template <>
struct Number<CCT_TYPE_F16> {
  typedef _Float16 T;
  typedef f16x8 V8;
  typedef f16x8 __attribute__((aligned(2))) U8;
};

template <int TYPE>
__device__ __forceinline__ float load1(const void* p, long long i) {
  return (float)((const typename Number<TYPE>::T*)p)[i];
}
template <int TYPE>
__device__ __forceinline__ void store1(void* p, long long i, float v) {
  ((typename Number<TYPE>::T*)p)[i] = (typename Number<TYPE>::T)v;
}
template <int TYPE>
__device__ __forceinline__ f32x8 load8(const void* p, long long i) {
  const auto* at = (const typename Number<TYPE>::T*)p + i;
  return __builtin_convertvector((typename Number<TYPE>::V8)*(const typename Number<TYPE>::U8*)at, f32x8);
}
template <int TYPE>
__device__ __forceinline__ void store8(void* p, long long i, const f32x8& v) {
  auto* at = (typename Number<TYPE>::T*)p + i;
  *(typename Number<TYPE>::U8*)at = __builtin_convertvector(v, typename Number<TYPE>::V8);
}

// Moves values `by` places to the front, 0 <= by < 8; zeros follow.
template <class V8>
__device__ __forceinline__ V8 move_down(V8 v, int by) {
  if constexpr (sizeof(V8) == 16) {
    typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
    u64x2 u = __builtin_bit_cast(u64x2, v);
    const int s = by * 16, in = s & 63;
    if (s >= 64) u = u64x2{u[1], 0};
    u[0] = u[0] >> in | (in ? u[1] << (64 - in) : 0);
    u[1] >>= in;
    return __builtin_bit_cast(V8, u);
  } else {
#pragma unroll
    for (int step = 1; step < 8; step *= 2)
      if (by & step)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e + step < 8 ? v[(e + step) & 7] : 0.f;
    return v;
  }
}
// 8 values from column c on of a row that begins at `row` and has c + n values, zeros behind its end: as they come from memory
// (of a row's last columns the eight that end with it), and brought into place, which waits for them.  One by one the last values were up
// to 7 trips to memory, in place as they come one for each load (backward pass of norms, 1531 x 2049: 53, 41 and 39 us).
template <int TYPE>
__device__ __forceinline__ typename Number<TYPE>::V8 load_row_raw(const void* p, long long row, int c, int n) {
  const auto* at = (const typename Number<TYPE>::T*)p + row;
  if (c + n >= 8) return *(const typename Number<TYPE>::U8*)(at + min(c, c + n - 8));
  typename Number<TYPE>::V8 v = {};
  if (c == 0)
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) v[e] = at[e];
  return v;
}
template <int TYPE>
__device__ __forceinline__ typename Number<TYPE>::V8 settle_row(typename Number<TYPE>::V8 v, int c, int n) {
  if (n >= 8 || c + n < 8) return v;
  if (n <= 0) return typename Number<TYPE>::V8{};
  return move_down(v, 8 - n);
}
template <int TYPE>
__device__ __forceinline__ f32x8 load_row(const void* p, long long row, int c, int n) {
  return __builtin_convertvector(settle_row<TYPE>(load_row_raw<TYPE>(p, row, c, n), c, n), f32x8);
}
// The first n of 8 values.
template <int TYPE>
__device__ __forceinline__ void store_first(void* p, long long i, const f32x8& v, int n) {
  if (n >= 8) return store8<TYPE>(p, i, v);
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) store1<TYPE>(p, i + e, v[e]);
}

inline int type_bytes(int type) { return type == CCT_TYPE_F32 ? 4 : 2; }
inline bool type_known(int type) { return type >= CCT_TYPE_F32 && type <= CCT_TYPE_F16; }

}  // namespace
}  // namespace cct
