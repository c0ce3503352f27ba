// How the matrix products of the feed-forward operators are cut into tiles and splits (16-bit types: ff_tile.h; fp32:
// ff_f32.hip).
#include <algorithm>

#include "feed_forward.h"

namespace cct {
namespace {

// Microseconds of a stage (64 steps of the contraction) with one workgroup on a CU and with as many as fit, measured with all
// 256 CUs busy on products of 1024 to 8192 rows, all three directions (within 8 % of each other).
struct TileCost {
  int bm, bn, per_cu;
  double alone, full;
};
constexpr TileCost kTileCosts[] = {{256, 256, 1, 1.62, 1.62}, {128, 128, 2, 0.65, 1.10}, {64, 128, 2, 0.39, 0.72}, {64, 64, 2, 0.29, 0.54}};
constexpr double kJoinMicros = 4.0, kJoinBytesPerMicro = 7.5e6;  // a launch and its gap; partial sums, written and read
constexpr int kCus = 256, kLeastStages = 4;                       // of a split

}  // namespace

// The tile and the number of splits of the contraction with the least estimate: rounds of workgroups over the card times the
// stages of one, and what joining the splits costs.  Few large tiles leave CUs idle, small ones read LDS more often per
// product.  1024 x 4096 x 9216 (forward, bf16): 181 us in tiles of 256 (64 of them), 96 in 128, 82 in 128 and two splits.
FfTilePlan ff_tile_plan(int M, int N, int K, int epilogue, int segments) {
  const long long cols = epilogue == kFfGated ? 2LL * N : N;
  const int stages = std::max((K + kFfStage - 1) / kFfStage, 1) * (epilogue == kFfGated ? 1 : segments);
  FfTilePlan best = {kTile128, 1, stages, 0};
  double least = 1e30;
  for (int tile = kTile256; tile <= kTile64; ++tile) {
    const TileCost& c = kTileCosts[tile];
    const long long tiles = ((M + c.bm - 1LL) / c.bm) * ((cols + c.bn - 1) / c.bn);
    for (int splits = 1; splits <= 32; splits *= 2) {
      if (splits > 1 && (tile == kTile256 || stages < splits * kLeastStages || tiles * splits > 4 * kCus)) break;
      const int each = (stages + splits - 1) / splits;
      const long long groups = tiles * splits, slots = (long long)kCus * c.per_cu, rest = groups % slots;
      double us = (double)(groups / slots) * c.full + (rest == 0 ? 0.0 : rest <= kCus ? c.alone : c.full);
      us *= each;
      if (splits > 1) us += kJoinMicros + 8.0 * splits * M * cols / kJoinBytesPerMicro;
      if (us < least) {
        least = us;
        best = {tile, (stages + each - 1) / each, each, 0};
      }
    }
  }
  best.part_bytes = best.splits > 1 ? 4LL * best.splits * M * (cols + 8) : 0;
  return best;
}

int launch_ff_product(const FfProduct& p, char* pack, float* ws, hipStream_t st) {
  if (p.type == CCT_TYPE_F32) return launch_ff_f32(p, pack, ws, st);
  const double mn = (double)p.M * p.N, ops = p.epilogue == kFfGated ? 2 : p.segments;
  const double bytes = 2.0 * ((double)(p.epilogue == kFfGated ? 1 : p.segments) * p.M * p.K + ops * p.N * p.K +
                              mn * (1 + (p.residual != nullptr) + (p.z != nullptr) + (p.z2 != nullptr)));
  const FfTilePlan plan = ff_tile_plan(p.M, p.N, p.K, p.epilogue, p.segments);
  const char* const names[] = {"256x256", "128x128", "64x128", "64x64"};
  ProfScope ps(2.0 * mn * p.K * ops, bytes, st, "ff_tile_kernel<%s, %d splits>", names[plan.tile], plan.splits);
  return p.type == CCT_TYPE_BF16 ? launch_ff_tile_bf16(p, plan, ws, st) : launch_ff_tile_f16(p, plan, ws, st);
}

}  // namespace cct
