// A step of a product of microscaled 4-bit matrices: 128 values of the contraction, four blocks, of 16 rows of each.  Lane l has
// block l / 16 of row l % 16 (16 bytes) and its scale in byte BY of a register.
#pragma once
#include "gemm_common.h"

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

}  // namespace
}  // namespace cct
