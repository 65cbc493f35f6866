// fp32 instances of the feed-forward block's tiled products.
#include "ffn_tile_launch.h"

namespace bkmoo {
hipError_t launch_ffn_tile_f32(Mode mode, const TileArgs &g, int tasks, bool aligned, int side, hipStream_t s) {
  return launch_ffn_tile_of<float>(mode, g, tasks, aligned, side, s);
}
}  // namespace bkmoo
