// The launcher of one element type's tiled products.
#pragma once

#include "ffn_tile.h"

namespace bkmoo {

// Tiles of 256 x 256 on eight waves, of 128 x 128 or 64 x 64 on four.
template <typename T, Mode MODE, bool ALIGNED>
hipError_t launch_mode(TileArgs g, int tasks, int side, hipStream_t s) {
  const int64_t rows = g.M, cols = MODE == kGateUp ? 2 * g.N : g.N;
  g.tiles_m = (int)((rows + side - 1) / side);
  g.tiles_n = (int)((cols + side - 1) / side);
  g.problems = MODE == kWeightGrad ? 3 * tasks : g.splits > 1 ? g.splits : 1;
  const int64_t n = (int64_t)g.tiles_m * g.tiles_n * g.problems;
  if (n == 0) return hipSuccess;
  if (n > 0x3fffffff) return hipErrorInvalidConfiguration;
  // As many workgroups as the chip holds at once (a CU one of the largest, two of the next or four of
  // the smallest), each with tiles to the end: a tile's first steps travel while the one before is stored
  // (M=4096, D=2048, F=6144, us, a workgroup a tile / these: gate and up 178 / 167, down 114 /
  // 95, weight gradients 324 / 301; 8192 x 4096 x 14336: 1772 / 1749, 857 / 852, 2564 / 2525;
  // with loads and reads placed by rows of pieces).
  // The hidden gradient's epilogue waits for loads of its own, which the next tile's would
  // hold up: a workgroup a tile (963 / 1079).
  constexpr bool tile_each = MODE == kHiddenGrad || MODE == kHiddenPart;
  const int64_t cus = tile_each ? n : device_cu_count();
  auto workgroups = [&](int64_t most) {
    if (!tile_each && g.workgroups > 0) most = g.workgroups;
    return (unsigned)(n < most ? n : most);
  };
  if constexpr (ALIGNED) {
    if (side == 256) {
      const unsigned grid = workgroups(cus);
      ffn_tile_kernel<T, MODE, 256, 256, 2, 4, true><<<dim3(grid), dim3(512), 0, s>>>(g);
      return hipGetLastError();
    }
  }
  if (side == 64) {
    const unsigned grid = workgroups(4 * cus);
    ffn_tile_kernel<T, MODE, 64, 64, 4, 1, ALIGNED><<<dim3(grid), dim3(256), 0, s>>>(g);
    return hipGetLastError();
  }
  const unsigned grid = workgroups(2 * cus);
  ffn_tile_kernel<T, MODE, 128, 128, 2, 2, ALIGNED><<<dim3(grid), dim3(256), 0, s>>>(g);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_ffn_tile_of(Mode mode, const TileArgs &g, int tasks, bool aligned, int side, hipStream_t s) {
  switch (mode) {
    case kGateUp:
      return aligned ? launch_mode<T, kGateUp, true>(g, tasks, side, s) : launch_mode<T, kGateUp, false>(g, tasks, side, s);
    case kDown:
      return aligned ? launch_mode<T, kDown, true>(g, tasks, side, s) : launch_mode<T, kDown, false>(g, tasks, side, s);
    case kHiddenGrad:
      return aligned ? launch_mode<T, kHiddenGrad, true>(g, tasks, side, s)
                     : launch_mode<T, kHiddenGrad, false>(g, tasks, side, s);
    case kHiddenPart:
      return aligned ? launch_mode<T, kHiddenPart, true>(g, tasks, side, s)
                     : launch_mode<T, kHiddenPart, false>(g, tasks, side, s);
    case kInputGrad:
      return aligned ? launch_mode<T, kInputGrad, true>(g, tasks, side, s)
                     : launch_mode<T, kInputGrad, false>(g, tasks, side, s);
    default:
      return aligned ? launch_mode<T, kWeightGrad, true>(g, tasks, side, s)
                     : launch_mode<T, kWeightGrad, false>(g, tasks, side, s);
  }
}

}  // namespace bkmoo
