// The matrix products of the feed-forward operators with their epilogues.
//
// 16-bit types: ff_tile.h.  fp32: a workgroup computes 64 x 64 results, 4 x 4 per thread, from LDS tiles of 16 k.
#include <algorithm>

#include "activation.h"
#include "feed_forward.h"
#include "ff_tile.h"

namespace cct {
namespace {

constexpr int NT = 256, BT = 64, BK = 16;

template <int TYPE, bool GATED>
__global__ __launch_bounds__(NT) void ff_product_kernel(FfProduct p, int tiles_m) {
  constexpr int NB = GATED ? 2 : 1;
  __shared__ float As[BK][BT + 1], Bs[NB][BK][BT + 1];
  const int tile_n = blockIdx.x / tiles_m, tile_m = blockIdx.x - tile_n * tiles_m;
  const int m0 = tile_m * BT, n0 = tile_n * BT;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[NB][4][4] = {};
  for (int s = 0; s < (GATED ? 1 : p.segments); ++s)
    for (int k0 = 0; k0 < p.K; k0 += BK) {
      __syncthreads();
      auto stage = [&](float(&to)[BK][BT + 1], const FfOperand& o, int r0, int rows) {
        for (int i = threadIdx.x; i < BT * BK; i += NT) {
          // consecutive threads along the consecutive dimension
          const int r = o.across ? i % BT : i / BK, k = o.across ? i / BT : i % BK;
          to[k][r] = r0 + r < rows && k0 + k < p.K ? load1<TYPE>(o.p, (r0 + r) * o.rs + (k0 + k) * o.ks) : 0.f;
        }
      };
      stage(As, p.A[s], m0, p.M);
      stage(Bs[0], p.B[s], n0, p.N);
      if constexpr (GATED) stage(Bs[1], p.B[1], n0, p.N);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < BK; ++k)
#pragma unroll
        for (int q = 0; q < NB; ++q)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[q][i][j] = fmaf(As[k][ty * 4 + i], Bs[q][k][tx * 4 + j], acc[q][i][j]);
    }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m >= p.M || n >= p.N) continue;
      float v[1] = {acc[0][i][j]};
      if constexpr (GATED) {
        const float u = acc[NB - 1][i][j];
        if (p.z) {
          store1<TYPE>(p.z, m * p.ldz + n, v[0]);
          store1<TYPE>(p.z2, m * p.ldz2 + n, u);
        }
        activate(p.activation, v);
        v[0] *= u;
      } else {
        if (p.bias) v[0] += load1<TYPE>(p.bias, n);
        if (p.z) store1<TYPE>(p.z, m * p.ldz + n, v[0]);
        activate(p.activation, v);
        if (p.residual) v[0] += load1<TYPE>(p.residual, m * p.ldr + n);
      }
      store1<TYPE>(p.out, m * p.ldo + n, v[0]);
    }
}

template <int TYPE>
void launch(const FfProduct& p, hipStream_t st) {
  const int tiles_m = (p.M + BT - 1) / BT, tiles_n = (p.N + BT - 1) / BT;
  if (p.epilogue == kFfGated)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_product_kernel<TYPE, true>), dim3(tiles_m * tiles_n), dim3(NT), 0, st, p, tiles_m);
  else
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_product_kernel<TYPE, false>), dim3(tiles_m * tiles_n), dim3(NT), 0, st, p, tiles_m);
}

template <int TYPE, int BM, int BN, int WM, int WN, bool AX, bool BX, int EPI>
int launch_tile(const FfProduct& p, hipStream_t st) {
  constexpr int lds = 2 * (BM + BN) * kStageK * 2;
  constexpr auto kernel = ff_tile_kernel<TYPE, BM, BN, WM, WN, AX, BX, EPI>;
  const int rc = ensure_dynamic_lds<kernel>(lds);
  if (rc != CCT_OK) return rc;
  constexpr int cols = EPI == kFfGated ? BN / 2 : BN;
  const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + cols - 1) / cols;
  hipLaunchKernelGGL(kernel, dim3(tiles_m * tiles_n), dim3(WM * WN * 64), lds, st, p, tiles_m, tiles_n);
  return CCT_OK;
}

template <int TYPE, int BM, int BN, int WM, int WN>
int launch_mode(const FfProduct& p, hipStream_t st) {
  const bool ax = p.A[0].across, bx = p.B[0].across;
  if (p.epilogue == kFfGated) return launch_tile<TYPE, BM, BN, WM, WN, false, false, kFfGated>(p, st);
  if (ax) return launch_tile<TYPE, BM, BN, WM, WN, true, true, kFfLinear>(p, st);
  if (bx) return launch_tile<TYPE, BM, BN, WM, WN, false, true, kFfLinear>(p, st);
  return launch_tile<TYPE, BM, BN, WM, WN, false, false, kFfLinear>(p, st);
}

// Tiles of 256 x 256 where they fill the card, else of 128 x 128.
template <int TYPE>
int launch_sized(const FfProduct& p, hipStream_t st) {
  const long long cols = p.epilogue == kFfGated ? 2LL * p.N : p.N;
  if ((long long)((p.M + 255) / 256) * ((cols + 255) / 256) >= 200) return launch_mode<TYPE, 256, 256, 2, 4>(p, st);
  return launch_mode<TYPE, 128, 128, 2, 2>(p, st);
}

}  // namespace

int launch_ff_product(const FfProduct& p, hipStream_t st) {
  const double e = type_bytes(p.type), mn = (double)p.M * p.N, ops = p.epilogue == kFfGated ? 2 : p.segments;
  const double flops = 2.0 * mn * p.K * ops;
  const double bytes = e * ((double)(p.epilogue == kFfGated ? 1 : p.segments) * p.M * p.K + ops * p.N * p.K +
                            mn * (1 + (p.residual != nullptr) + (p.z != nullptr) + (p.z2 != nullptr)));
  ProfScope ps("ff_product_kernel", flops, bytes, st);
  int rc = CCT_OK;
  if (p.type == CCT_TYPE_F32)
    launch<CCT_TYPE_F32>(p, st);
  else if (p.type == CCT_TYPE_BF16)
    rc = launch_sized<CCT_TYPE_BF16>(p, st);
  else
    rc = launch_sized<CCT_TYPE_F16>(p, st);
  if (rc != CCT_OK) return rc;
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
