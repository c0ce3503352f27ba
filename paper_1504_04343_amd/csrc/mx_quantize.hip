// Microscaled 4-bit floating point: values to codes and scales, and back.  Both are bound by memory: a thread takes 8 neighbouring
// values of a block of 32, four threads share their largest size, gfx950's conversions do the rest (v_cvt_scalef32_pk_fp4_f32:
// x / 2^e to nearest, ties to even, at most 6, and v_cvt_scalef32_pk_f32_fp4; checked against these rules over all scales, codes,
// middles and their neighbours).  8192 x 8192 bf16: quantise 40 us, back 27 (4.3 and 6.4 TB/s, the codes still in a cache); rows of
// 2049 fp32 at odd distances, 1531 of them: 7 and 6 us, of which launching and a trip to memory are half.
#include <algorithm>

#include "mx.h"
#include "number_types.h"

namespace cct {
namespace {

constexpr int kThreads = 256, kRows = 4;  // rows that a thread has on their way at once

template <class F>
void with_type(int type, F f) {
  if (type == CCT_TYPE_F32)
    f(std::integral_constant<int, CCT_TYPE_F32>());
  else if (type == CCT_TYPE_BF16)
    f(std::integral_constant<int, CCT_TYPE_BF16>());
  else
    f(std::integral_constant<int, CCT_TYPE_F16>());
}

struct MxJob {
  int rows, cols, chunks;  // chunks of 8 values: 4 times the blocks
  int wide;                // threads along a row, a power of two
  long long ldx, ldc, lds;
};

// e2m1's scale as the float whose exponent field it is
__device__ __forceinline__ float scale_float(unsigned s) { return __builtin_bit_cast(float, s << 23); }

template <int TYPE>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(MxJob j, const void* __restrict__ x, unsigned char* __restrict__ codes,
                                                               unsigned char* __restrict__ scales) {
  const int down = kThreads / j.wide, lane = threadIdx.x & (j.wide - 1), own = threadIdx.x / j.wide;
  const long long at = (long long)blockIdx.x * j.wide + lane;
  if (at >= j.chunks) return;  // whole fours of threads
  const int chunk = (int)at, c = chunk * 8, n = j.cols - c;
  const long long step = (long long)gridDim.y * down * kRows;
  for (long long r0 = (long long)blockIdx.y * down * kRows + own; r0 < j.rows; r0 += step) {
    typename Number<TYPE>::V8 raw[kRows];
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const long long row = min(r0 + q * down, (long long)j.rows - 1);
      raw[q] = load_row_raw<TYPE>(x, row * j.ldx, c, n);
    }
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const long long row = r0 + q * down;
      const f32x8 v = __builtin_convertvector(settle_row<TYPE>(raw[q], c, n), f32x8);
      unsigned most = 0;  // sizes compare as whole numbers, infinities and NaN above all others
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, __builtin_bit_cast(unsigned, (float)v[e]) & 0x7fffffffu);
      most = max(most, (unsigned)__builtin_amdgcn_mov_dpp((int)most, 0xb1, 0xf, 0xf, true));
      most = max(most, (unsigned)__builtin_amdgcn_mov_dpp((int)most, 0x4e, 0xf, 0xf, true));
      const unsigned field = most >> 23, scale = field == 255 ? 255 : (unsigned)max((int)field - 2, 0);
      unsigned code = 0;
      if (field != 255) {
        const float s = scale_float(scale);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], s, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], s, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], s, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], s, 3);
      }
      if (row >= j.rows) continue;
      *(unsigned*)(codes + row * j.ldc + chunk * 4LL) = code;
      if ((chunk & 3) == 0) scales[row * j.lds + (chunk >> 2)] = (unsigned char)scale;
    }
  }
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(MxJob j, const unsigned char* __restrict__ codes,
                                                                 const unsigned char* __restrict__ scales, void* __restrict__ x) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const int down = kThreads / j.wide, lane = threadIdx.x & (j.wide - 1), own = threadIdx.x / j.wide;
  const long long at = (long long)blockIdx.x * j.wide + lane;
  if (at >= j.chunks) return;
  const int chunk = (int)at, c = chunk * 8, n = j.cols - c;
  const long long step = (long long)gridDim.y * down * kRows;
  for (long long r0 = (long long)blockIdx.y * down * kRows + own; r0 < j.rows; r0 += step) {
    unsigned code[kRows], scale[kRows];
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const long long row = min(r0 + q * down, (long long)j.rows - 1);
      code[q] = *(const unsigned*)(codes + row * j.ldc + chunk * 4LL);
      scale[q] = scales[row * j.lds + (chunk >> 2)];
    }
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const long long row = r0 + q * down;
      if (row >= j.rows) continue;
      const float s = scale_float(scale[q]);
      const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[q], s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[q], s, 1),
                  d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[q], s, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[q], s, 3);
      store_first<TYPE>(x, row * j.ldx + c, f32x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]}, n);
    }
  }
}

MxJob job_of(int rows, int cols, long long ldx, long long ldc, long long lds, dim3* grid) {
  MxJob j = {rows, cols, 4 * mx_blocks(cols), 4, ldx, ldc, lds};
  while (j.wide < kThreads && j.wide < j.chunks) j.wide *= 2;
  // rows a little longer than that leave most threads of their last workgroup idle: half as wide (2049 columns: 256 and 4 chunks)
  while (j.wide > 64 && pieces(j.chunks, j.wide / 2) * (j.wide / 2) < pieces(j.chunks, j.wide) * j.wide * 7 / 8) j.wide /= 2;
  const int across = pieces(j.chunks, j.wide);
  const long long most = std::min(65535LL, std::max(1LL, kMostThreads / kThreads / across));
  *grid = dim3(across, (unsigned)std::min(most, (long long)pieces(rows, kThreads / j.wide * kRows)));
  return j;
}

}  // namespace

int launch_mx_quantize(int rows, int cols, int type, const void* x, long long ldx, unsigned char* codes, long long ldc,
                       unsigned char* scales, long long lds, hipStream_t st) {
  ProfScope ps("mx_quantize_kernel", 0.0, (double)rows * cols * (type_bytes(type) + 17.0 / 32), st);
  dim3 grid;
  const MxJob j = job_of(rows, cols, ldx, ldc, lds, &grid);
  with_type(type, [&](auto t) {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_quantize_kernel<decltype(t)::value>), grid, dim3(kThreads), 0, st, j, x, codes, scales);
  });
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

int launch_mx_dequantize(int rows, int cols, int type, const MxMatrix& m, void* x, long long ldx, hipStream_t st) {
  ProfScope ps("mx_dequantize_kernel", 0.0, (double)rows * cols * (type_bytes(type) + 17.0 / 32), st);
  dim3 grid;
  const MxJob j = job_of(rows, cols, ldx, m.ldc, m.lds, &grid);
  with_type(type, [&](auto t) {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_dequantize_kernel<decltype(t)::value>), grid, dim3(kThreads), 0, st, j, m.codes, m.scales, x);
  });
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
