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

inline int type_bytes(int type) { return type == CCT_TYPE_F32 ? 4 : 2; }
inline bool type_known(int type) { return type >= CCT_TYPE_F32 && type <= CCT_TYPE_F16; }

}  // namespace
}  // namespace cct
