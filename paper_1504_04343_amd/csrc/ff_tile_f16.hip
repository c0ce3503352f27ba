// The tiled products of f16 operands (ff_tile.h).
#include "ff_tile_launch.h"

namespace cct {
int launch_ff_tile_f16(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st) {
  return launch_planned<CCT_TYPE_F16>(p, plan, ws, st);
}
}  // namespace cct
