// The gated feed-forward block's products: shared by its launchers and kernels.
#pragma once

#include "internal.h"

namespace bkmoo {

enum GateAct : int { kSilu = 0, kGelu = 1 };

// The tiled products.  x, y [M][D]; u, v, h [M][F]; Wg, Wu [F][D]; Wd [D][F].
enum Mode : int {
  kGateUp,      // u = x Wg^T, v = x Wu^T -> h = a(u) v (and u, v)
  kDown,        // y = h Wd^T
  kHiddenGrad,  // dh = dy Wd -> du = dh v a'(u), dv = dh a(u), h = a(u) v
  kHiddenPart,  // a part of dh's sum
  kInputGrad,   // dx = du Wg + dv Wu
  kWeightGrad   // per task: dWg = du^T x, dWu = dv^T x, dWd = dy^T h
};

struct TileArgs {
  const void *a[3], *b[3];  // operands (kWeightGrad: of the three matrices)
  void *out[3];
  const void *u, *v;        // kHiddenGrad
  float *partial;           // [splits][M][N], where the sum is split
  int64_t M, N, K;          // output rows and columns (kWeightGrad: of the first two matrices), length of the sum
  int64_t task_stride;      // elements from one task's gradient row to the next
  int tiles_m, tiles_n, problems, splits, act;
  int workgroups;           // at most so many, but for the hidden gradient; 0: as many as the chip holds
  int64_t rows[kMaxK + 1];  // kWeightGrad: the tasks' rows
};

hipError_t launch_ffn_tile_f32(Mode mode, const TileArgs &g, int tasks, bool aligned, int side, hipStream_t s);
hipError_t launch_ffn_tile_bf16(Mode mode, const TileArgs &g, int tasks, bool aligned, int side, hipStream_t s);
// aligned: operands start at multiples of four bytes and so do all their rows.  side: of the tiles, 64, 128 or
// (aligned) 256.
hipError_t launch_ffn_tile(int dt, Mode mode, const TileArgs &g, int tasks, bool aligned, int side, hipStream_t s);

// The whole forward pass for at most kFewRows rows; h [M][F] is scratch, for at most kFewExact rows of
// bf16 two of them.  More rows take the
// tiles (us in all, D=4096 F=14336: 64 rows 95 here, 65 as tiles 104, 96 115 where here is about
// 120; D=2048 F=6144: 64 rows 25, 65 37).
constexpr int64_t kFewRows = 64, kFewExact = 8;
hipError_t launch_ffn_few(int dt, const void *x, const void *wg, const void *wu, const void *wd, void *h, void *y,
                          void *u, void *v, int64_t M, int64_t D, int64_t F, int act, bool aligned, hipStream_t s);

}  // namespace bkmoo
