// The tiled products of bf16 operands (ff_tile.h).
#include "ff_tile_launch.h"

namespace cct {
int launch_ff_tile_bf16(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st) {
  return launch_planned<CCT_TYPE_BF16>(p, plan, ws, st);
}
int launch_ff_together_bf16(const FfProduct* p, int count, const FfBiasSum& sum, const FfTogetherPlan& plan, char* ws, hipStream_t st) {
  return launch_together<CCT_TYPE_BF16>(p, count, sum, plan, ws, st);
}
}  // namespace cct
