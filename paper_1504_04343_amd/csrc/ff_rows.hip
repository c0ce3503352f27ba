// Forward products of few rows (serving: one token, or a batch of sequences with one each): the weights are read once and
// nothing else matters.
//
// A workgroup takes 16 rows of the weight (gated: of both) and all rows of x, its eight waves every eighth step of the
// contraction: 64 bytes of each weight row, which go from memory straight into the registers that the matrix cores take (32
// values of 16 bits per instruction, 4 of fp32 in an order of their own that x follows).  No LDS and no meeting in the loop;
// eight steps' loads are in flight per wave, and x comes from L2 the same way.  The waves' sums meet in LDS in a fixed
// order.  fp32 runs on v_mfma_f32_16x16x4_f32, which memory outlasts.
//
// One row, bf16, weights from memory: 4096 x 4096 7.9 us (4.3 TB/s; 6.8 at the rate of a large copy), 16384 x 4096 25.6 (5.2
// TB/s), gated 2 x 8192 x 4096 27.0 (5.0).  With two batches of four steps in turn 9.0, 29.1 and 29.8: the compiler waits
// for all of a batch before it loads the next one into the same registers, so that they are only smaller; with sixteen waves
// 8.0, 26.8 and 26.8.
//
// Any alignment: gfx950 loads 16 bytes at any address.  A last step that is not whole is loaded value by value.
#include <algorithm>

#include "activation.h"
#include "feed_forward.h"
#include "ff_tile.h"

namespace cct {
namespace {

constexpr int kWaves = 8;

template <int TYPE>
struct Step {  // 16-bit types
  typedef s16x8 V;
  static constexpr int CH = 8, K = 32;  // values per lane, per step
  static __device__ __forceinline__ V load(const void* p, long long at) {
    typedef s16x8 U __attribute__((aligned(2)));
    return *(const U*)((const short*)p + at);
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

// RM: blocks of 16 rows of x
template <int TYPE, int RM, int EPI>
__global__ __launch_bounds__(kWaves * 64) void ff_rows_kernel(FfProduct p) {
  typedef Step<TYPE> S;
  typedef typename S::V V;
  constexpr int NB = EPI == kFfGated ? 2 : 1, BATCH = RM == 4 ? 4 : 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16, lo = lane & 15, kq = (lane >> 4) * S::CH;
  long long w_at = (long long)min(n0 + lo, p.N - 1) * p.B[0].rs, u_at = (long long)min(n0 + lo, p.N - 1) * p.B[NB - 1].rs, x_at[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) x_at[i] = (long long)min(i * 16 + lo, p.M - 1) * p.A[0].rs;

  f32x4 acc[NB][RM];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < RM; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int whole = p.K / S::K;  // steps
  V w[BATCH][NB], x[BATCH][RM];
  // steps past the last one load it again and multiply zeros
  auto load = [&](int s0) {
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const long long k = (long long)min(s0 + q * kWaves, whole - 1) * S::K + kq;
      w[q][0] = S::load(p.B[0].p, w_at + k);
      if constexpr (NB == 2) w[q][1] = S::load(p.B[1].p, u_at + k);
#pragma unroll
      for (int i = 0; i < RM; ++i) x[q][i] = S::load(p.A[0].p, x_at[i] + k);
    }
  };
  auto multiply = [&](int s0) {
    __builtin_amdgcn_sched_barrier(0);  // the loads in front of it are not moved behind
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const bool live = s0 + q * kWaves < whole;
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const V xv = live ? x[q][i] : V{};
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b][i] = S::mfma(live ? w[q][b] : V{}, xv, acc[b][i]);
      }
    }
  };
  for (int s = wave; s < whole; s += BATCH * kWaves) {
    load(s);
    multiply(s);
  }
  if (p.K % S::K && whole % kWaves == wave) {
    const int k = whole * S::K + kq, n = max(0, min(S::CH, p.K - k));
    V wv[NB];
    wv[0] = S::part(p.B[0].p, w_at + k, n);
    if constexpr (NB == 2) wv[1] = S::part(p.B[1].p, u_at + k, n);
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const V xv = S::part(p.A[0].p, x_at[i] + k, n);
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][i] = S::mfma(wv[b], xv, acc[b][i]);
    }
  }

  __shared__ f32x4 sums[kWaves][NB * RM][64];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < RM; ++i) sums[wave][b * RM + i][lane] = acc[b][i];
  __syncthreads();
  for (int i = wave; i < RM; i += kWaves) {
    f32x4 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      s[b] = sums[0][b * RM + i][lane];
#pragma unroll
      for (int q = 1; q < kWaves; ++q) s[b] += sums[q][b * RM + i][lane];
    }
    const int m = i * 16 + lo, n = n0 + (lane >> 4) * 4;
    if (m >= p.M || n >= p.N) continue;
    float v[4], u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = s[0][e];
      u[e] = s[NB - 1][e];
    }
    finish<TYPE, EPI>(p, m, n, v, u);
  }
}

template <int TYPE, int EPI>
void launch(const FfProduct& p, hipStream_t st) {
  const dim3 grid((p.N + 15) / 16), block(kWaves * 64);
  if (p.M <= 16)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_rows_kernel<TYPE, 1, EPI>), grid, block, 0, st, p);
  else if (p.M <= 32)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_rows_kernel<TYPE, 2, EPI>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_rows_kernel<TYPE, 4, EPI>), grid, block, 0, st, p);
}
template <int TYPE>
void launch(const FfProduct& p, hipStream_t st) {
  if (p.epilogue == kFfGated)
    launch<TYPE, kFfGated>(p, st);
  else
    launch<TYPE, kFfLinear>(p, st);
}

}  // namespace

int launch_ff_rows(const FfProduct& p, hipStream_t st) {
  const double e = type_bytes(p.type), mn = (double)p.M * p.N, ops = p.epilogue == kFfGated ? 2 : 1;
  const double bytes = e * ((double)p.M * p.K + ops * p.N * p.K +
                            mn * (1 + (p.residual != nullptr) + (p.z != nullptr) + (p.z2 != nullptr)));
  ProfScope ps("ff_rows_kernel", 2.0 * mn * p.K * ops, bytes, st);
  if (p.type == CCT_TYPE_F32)
    launch<CCT_TYPE_F32>(p, st);
  else if (p.type == CCT_TYPE_BF16)
    launch<CCT_TYPE_BF16>(p, st);
  else
    launch<CCT_TYPE_F16>(p, st);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
