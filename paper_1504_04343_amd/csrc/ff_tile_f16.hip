// The tiled products of f16 operands (ff_tile.h).
#include "ff_tile_launch.h"

namespace cct {
int launch_ff_tile_f16(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st) {
  return launch_planned<CCT_TYPE_F16>(p, plan, ws, st);
}
int launch_ff_together_f16(const FfProduct* p, int count, const FfBiasSum& sum, const FfTogetherPlan& plan, char* ws, hipStream_t st) {
  return launch_together<CCT_TYPE_F16>(p, count, sum, plan, ws, st);
}
}  // namespace cct
