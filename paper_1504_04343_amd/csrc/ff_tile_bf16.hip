// The tiled products of bf16 operands (ff_tile.h).
#include "ff_tile_launch.h"

namespace cct {
int launch_ff_tile_bf16(const FfProduct& p, const FfTilePlan& plan, float* ws, hipStream_t st) {
  return launch_planned<CCT_TYPE_BF16>(p, plan, ws, st);
}
}  // namespace cct
