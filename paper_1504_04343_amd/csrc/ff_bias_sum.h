// dbias from the rows of partial sums that ff_dz_kernel leaves: a workgroup takes 16 columns, 64 runs of rows whose sums meet
// always in the same order, whether 1024 threads take a run each (a kernel of its own, ff_backward.hip) or 256 take four
// (workgroups of a launch that multiplies).
#pragma once
#include "feed_forward.h"

namespace cct {

constexpr int kBiasColumns = 16, kBiasRuns = 64, kBiasMost = 1 << 20;  // workgroups next to products

template <int TYPE, int THREADS>
__device__ __forceinline__ void sum_bias(const FfBiasSum& p, int group, float (*sums)[kBiasColumns + 1]) {
  constexpr int TOP = THREADS / kBiasColumns, MINE = kBiasRuns / TOP;  // runs that meet in LDS, runs of a thread
  const int c = threadIdx.x % kBiasColumns, col = group * kBiasColumns + c, q = threadIdx.x / kBiasColumns;
  float s[MINE] = {};
  if (col < p.N)
#pragma unroll 4
    for (int r0 = 0; r0 < p.rows; r0 += kBiasRuns)
#pragma unroll
      for (int k = 0; k < MINE; ++k) {
        const int r = r0 + q + k * TOP;
        if (r < p.rows) s[k] += p.part[(long long)r * p.N + col];
      }
#pragma unroll
  for (int half = MINE / 2; half > 0; half >>= 1)
#pragma unroll
    for (int k = 0; k < half; ++k) s[k] += s[k + half];
  sums[q][c] = s[0];
  __syncthreads();
#pragma unroll
  for (int half = TOP / 2; half > 0; half >>= 1) {
    if (q < half) sums[q][c] += sums[q + half][c];
    __syncthreads();
  }
  if (q == 0 && col < p.N) store1<TYPE>(p.dbias, col, sums[0][c]);
}

}  // namespace cct
