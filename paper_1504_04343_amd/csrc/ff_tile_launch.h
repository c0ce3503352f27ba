// Launches of ff_tile.h's kernels for one type, as a plan says; a translation unit per type instantiates it.
#pragma once
#include "ff_tile.h"

namespace cct {
namespace {

template <int TYPE, int BM, int BN, int WM, int WN, int RING, bool AX, bool BX, int EPI, bool SPLIT>
int launch_tile(const FfProduct& p, const FfPart& part, hipStream_t st) {
  constexpr int ring = RING * (BM + BN) * SK * 2, out = TileEpilogue<BM, BN, WM, WN>::BYTES, lds = ring > out ? ring : out;
  constexpr auto kernel = ff_tile_kernel<TYPE, BM, BN, WM, WN, RING, AX, BX, EPI, SPLIT>;
  const int rc = ensure_dynamic_lds<kernel>(lds);
  if (rc != CCT_OK) return rc;
  constexpr int cols = EPI == kFfGated ? BN / 2 : BN;
  const int tiles_m = pieces(p.M, BM), tiles_n = pieces(p.N, cols);
  hipLaunchKernelGGL(kernel, dim3(tiles_m * tiles_n * part.splits), dim3(WM * WN * 64), lds, st, p, tiles_m, tiles_n, part);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

template <int TYPE, int BM, int BN, int WM, int WN, int RING, bool SPLIT>
int launch_mode(const FfProduct& p, const FfPart& part, hipStream_t st) {
  const bool ax = p.a_across, bx = p.b_across;
  if (p.epilogue == kFfGated) return launch_tile<TYPE, BM, BN, WM, WN, RING, false, false, kFfGated, SPLIT>(p, part, st);
  if (ax) return launch_tile<TYPE, BM, BN, WM, WN, RING, true, true, kFfLinear, SPLIT>(p, part, st);
  if (bx) return launch_tile<TYPE, BM, BN, WM, WN, RING, false, true, kFfLinear, SPLIT>(p, part, st);
  return launch_tile<TYPE, BM, BN, WM, WN, RING, false, false, kFfLinear, SPLIT>(p, part, st);
}

template <int TYPE>
int launch_planned(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st) {
  const FfPart part = {ws, (p.N + 3) / 4 * 4, plan.splits, plan.stages};
  if (plan.splits == 1) switch (plan.tile) {
      case kTile256: return launch_mode<TYPE, 256, 256, 2, 4, 2, false>(p, part, st);
      case kTile192: return launch_mode<TYPE, 192, 256, 2, 4, 2, false>(p, part, st);
      case kTile128: return launch_mode<TYPE, 128, 128, 2, 2, 2, false>(p, part, st);
      case kTile64x128: return launch_mode<TYPE, 64, 128, 2, 2, 3, false>(p, part, st);
      default: return launch_mode<TYPE, 64, 64, 2, 2, 4, false>(p, part, st);
    }
  int rc;
  switch (plan.tile) {
    case kTile128: rc = launch_mode<TYPE, 128, 128, 2, 2, 2, true>(p, part, st); break;
    case kTile64x128: rc = launch_mode<TYPE, 64, 128, 2, 2, 3, true>(p, part, st); break;
    default: rc = launch_mode<TYPE, 64, 64, 2, 2, 4, true>(p, part, st);
  }
  if (rc != CCT_OK) return rc;
  if (p.epilogue == kFfGated)
    launch_join<TYPE, kFfGated>(p, part, st);
  else
    launch_join<TYPE, kFfLinear>(p, part, st);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

template <int TYPE, int BM, int BN, int WM, int WN, int RING>
int launch_together(FfTogether a, hipStream_t st) {
  constexpr int ring = RING * (BM + BN) * SK * 2, out = TileEpilogue<BM, BN, WM, WN>::BYTES, lds = ring > out ? ring : out;
  constexpr auto kernel = ff_tile_kernel_together<TYPE, BM, BN, WM, WN, RING>;
  const int rc = ensure_dynamic_lds<kernel>(lds);
  if (rc != CCT_OK) return rc;
  int groups = a.sum.dbias ? pieces(a.sum.N, kBiasColumns) : 0;
  for (int i = 0; i < a.count; ++i) {
    a.first[i] = groups;
    a.tiles_m[i] = pieces(a.p[i].M, BM);
    a.tiles_n[i] = pieces(a.p[i].N, BN);
    groups += a.tiles_m[i] * a.tiles_n[i] * a.part[i].splits;
  }
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(WM * WN * 64), lds, st, a);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}
template <int TYPE>
int launch_together(const FfProduct* p, int count, const FfBiasSum& sum, const FfTogetherPlan& plan, char* ws, hipStream_t st) {
  FfTogether a = {}, joined = {};
  a.count = count;
  a.sum = sum;
  int groups = 0;
  for (int i = 0; i < count; ++i) {
    a.p[i] = p[i];
    a.part[i] = {(float*)(ws + plan.at[i]), (p[i].N + 3) / 4 * 4, plan.splits[i], plan.stages[i]};
    if (plan.splits[i] == 1) continue;
    joined.p[joined.count] = p[i];
    joined.part[joined.count] = a.part[i];
    joined.first[joined.count++] = groups;
    groups += (int)(((long long)p[i].M * a.part[i].ld / 4 + 255) / 256);
  }
  int rc;
  switch (plan.tile) {
    case kTile128: rc = launch_together<TYPE, 128, 128, 2, 2, 2>(a, st); break;
    case kTile64x128: rc = launch_together<TYPE, 64, 128, 2, 2, 3>(a, st); break;
    default: rc = launch_together<TYPE, 64, 64, 2, 2, 4>(a, st);
  }
  if (rc != CCT_OK || groups == 0) return rc;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(ff_join_kernel_together<TYPE>), dim3(groups), dim3(256), 0, st, joined);
  CCT_CHECK_LAUNCH();
  return CCT_OK;
}

}  // namespace
}  // namespace cct
