// A step of a product of microscaled 4-bit matrices: 128 values of the contraction, four blocks, of 16 rows of each.  Lane l has
// block l / 16 of row l % 16 (16 bytes) and its scale in byte BY of a register.
#pragma once
#include "gemm_common.h"
#include "number_types.h"

namespace cct {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int BYA, int BYB>
__device__ __forceinline__ f32x4 mx_mfma(i32x4 a, i32x4 b, f32x4 c, int sa, int sb) {
  // the instruction takes 8 registers of 8-bit operands, of 4-bit ones (format 4) the first four
  const i32x8 a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, BYA, sa, BYB, sb);
}

// The scales of four steps from s0 on: a word each, which holds its four blocks'.  Rows have room for whole words; those behind
// the last one are the last one.
__device__ __forceinline__ i32x4 mx_scales4(const unsigned char* row, int s0, int blocks) {
  typedef i32x4 U __attribute__((aligned(4)));
  const int words = (blocks + 3) >> 2;
  if (s0 + 4 <= words) return *(const U*)(row + 4LL * s0);
  i32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = *(const int*)(row + 4LL * min(s0 + j, words - 1));
  return v;
}

// A block of a row of values (four chunks of 8, zeros behind the row's end) as mx_quantize_kernel rounds it: its codes, its scale.
template <int TYPE>
__device__ __forceinline__ i32x4 mx_quantize_block(const typename Number<TYPE>::V8 (&v)[4], int* scale) {
  unsigned most = 0;
  if constexpr (TYPE == CCT_TYPE_F32) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, __builtin_bit_cast(unsigned, (float)v[q][e]) & 0x7fffffffu);
  } else {  // sizes of 16-bit values compare as whole numbers too, two at a time
    typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
    u16x8 m = __builtin_bit_cast(u16x8, v[0]) & (unsigned short)0x7fff;
#pragma unroll
    for (int q = 1; q < 4; ++q) m = __builtin_elementwise_max(m, (u16x8)(__builtin_bit_cast(u16x8, v[q]) & (unsigned short)0x7fff));
    unsigned short t = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) t = max(t, m[e]);
    most = TYPE == CCT_TYPE_BF16 ? (unsigned)t << 16 : __builtin_bit_cast(unsigned, (float)__builtin_bit_cast(_Float16, t));
  }
  const unsigned field = most >> 23;
  *scale = field == 255 ? 255 : max((int)field - 2, 0);
  const float s = __builtin_bit_cast(float, (unsigned)*scale << 23);
  i32x4 codes;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    unsigned c = 0;
    auto two = [&](auto byte) {
      constexpr int B = decltype(byte)::value;
      if constexpr (TYPE == CCT_TYPE_F32)
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[q][2 * B], v[q][2 * B + 1], s, B);
      else if constexpr (TYPE == CCT_TYPE_BF16)
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_shufflevector(v[q], v[q], 2 * B, 2 * B + 1), s, B);
      else
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_shufflevector(v[q], v[q], 2 * B, 2 * B + 1), s, B);
    };
    two(std::integral_constant<int, 0>());
    two(std::integral_constant<int, 1>());
    two(std::integral_constant<int, 2>());
    two(std::integral_constant<int, 3>());
    codes[q] = field == 255 ? 0 : (int)c;
  }
  return codes;
}

}  // namespace
}  // namespace cct
