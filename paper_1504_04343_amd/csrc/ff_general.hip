// The products of the feed-forward operators that no other kernel addresses: any type, strides of any length (fp32 rows 2^22
// values apart and more, 16-bit rows that are that long or longer: see `reaches` in ff_product.hip), empty contractions.
//
// 64 x 64 results per workgroup, 4 x 4 per thread in fp32, from LDS tiles of 16 k; every address in 64 bits.  Nothing is loaded
// ahead, so that 16 steps of the contraction take a workgroup about 4 us; few results of a long contraction are cut into splits
// (70 x 70 results of 17 million steps, bf16: 3.9 s whole, 21 ms so).
#include <algorithm>

#include "ff_tile.h"

namespace cct {
namespace {

constexpr int NT = 256, BT = 64, BK = 16;

template <int TYPE, bool GATED>
__global__ __launch_bounds__(NT) void ff_general_kernel(FfProduct p, int tiles_m, int first, FfPart part) {
  constexpr int NB = GATED ? 2 : 1;
  __shared__ float As[BK][BT + 1], Bs[NB][BK][BT + 1];
  const int tile = first + blockIdx.x, tile_n = tile / tiles_m, tile_m = tile - tile_n * tiles_m, split = blockIdx.y;
  const int m0 = tile_m * BT, n0 = tile_n * BT;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[NB][4][4] = {};
  const int per = pieces(p.K, BK), all = per * (GATED ? 1 : p.segments);
  const int end = part.splits > 1 ? min((split + 1) * part.stages, all) : all;
  for (int t = part.splits > 1 ? split * part.stages : 0; t < end; ++t) {
    const int s = t >= per, k0 = (t - s * per) * BK;
    __syncthreads();
    auto stage = [&](float(&to)[BK][BT + 1], const FfOperand& o, bool across, int r0, int rows) {
      for (int i = threadIdx.x; i < BT * BK; i += NT) {
        // consecutive threads along the consecutive dimension
        const int r = across ? i % BT : i / BK, k = across ? i / BT : i % BK;
        const long long at = across ? (r0 + r) + (k0 + k) * o.ld : (r0 + r) * o.ld + (k0 + k);
        to[k][r] = r0 + r < rows && k0 + k < p.K ? load1<TYPE>(o.p, at) : 0.f;
      }
    };
    stage(As, p.A[s], p.a_across, m0, p.M);
    stage(Bs[0], p.B[s], p.b_across, n0, p.N);
    if constexpr (GATED) stage(Bs[1], p.B[1], p.b_across, n0, p.N);
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
  const int n = n0 + tx * 4;
  if (n >= p.N) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + ty * 4 + i;
    if (m >= p.M) continue;
    if (part.splits > 1) {
#pragma unroll
      for (int q = 0; q < NB; ++q)
        *(f32x4*)(part.p + (((long long)split * NB + q) * p.M + m) * part.ld + n) = f32x4{acc[q][i][0], acc[q][i][1], acc[q][i][2], acc[q][i][3]};
    } else {
      finish<TYPE, GATED ? kFfGated : kFfLinear>(p, m, n, acc[0][i], acc[NB - 1][i]);
    }
  }
}

template <int TYPE, int EPI>
void launch(const FfProduct& p, const FfPart& part, hipStream_t st) {
  const int tiles_m = pieces(p.M, BT), tiles = tiles_m * pieces(p.N, BT), most = (int)(kMostThreads / NT);
  for (int first = 0; first < tiles; first += most)
    hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_general_kernel<TYPE, EPI == kFfGated>), dim3(std::min(most, tiles - first), part.splits),
                       dim3(NT), 0, st, p, tiles_m, first, part);
  if (part.splits > 1) launch_join<TYPE, EPI>(p, part, st);
}
template <int TYPE>
void launch(const FfProduct& p, const FfPart& part, hipStream_t st) {
  if (p.epilogue == kFfGated)
    launch<TYPE, kFfGated>(p, part, st);
  else
    launch<TYPE, kFfLinear>(p, part, st);
}

}  // namespace

// Up to four workgroups per CU, of at least 256 steps of 16 k each.
FfGeneralPlan ff_general_plan(const FfProduct& p) {
  const long long tiles = (long long)pieces(p.M, BT) * pieces(p.N, BT), products = p.epilogue == kFfGated ? 2 : 1;
  const long long steps = (long long)pieces(p.K, BK) * (p.epilogue == kFfGated ? 1 : p.segments);
  const int splits = (int)std::max(1LL, std::min(1024 / tiles, steps / 256));
  FfGeneralPlan plan;
  plan.steps = (int)((steps + splits - 1) / splits);
  plan.splits = plan.steps ? (int)((steps + plan.steps - 1) / plan.steps) : 1;
  plan.part_bytes = plan.splits > 1 ? 4LL * plan.splits * products * p.M * ((p.N + 3LL) / 4 * 4) : 0;
  return plan;
}

int launch_ff_general(const FfProduct& p, const FfGeneralPlan& plan, float* ws, hipStream_t st) {
  const FfPart part = {ws, (p.N + 3) / 4 * 4, plan.splits, plan.steps};
  const double e = type_bytes(p.type), mn = (double)p.M * p.N, ops = p.epilogue == kFfGated ? 2 : p.segments;
  const double bytes = e * ((double)(p.epilogue == kFfGated ? 1 : p.segments) * p.M * p.K + ops * p.N * p.K +
                            mn * (1 + (p.residual != nullptr) + (p.z != nullptr) + (p.z2 != nullptr)));
  ProfScope ps("ff_general_kernel", 2.0 * mn * p.K * ops, bytes, st);
  if (p.type == CCT_TYPE_F32)
    launch<CCT_TYPE_F32>(p, part, st);
  else if (p.type == CCT_TYPE_BF16)
    launch<CCT_TYPE_BF16>(p, part, st);
  else
    launch<CCT_TYPE_F16>(p, part, st);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace cct
