// Tiled matrix products of the gated feed-forward block on the matrix cores.
//
// C[m][n] = sum_k A(m, k) B(n, k), the sum in fp32.  An operand is either
// K-contiguous (element (m, k) at m * ld + k: activations and weights used as a
// linear layer holds them) or K-strided (at k * ld + m: the weights' transposes in the
// backward pass, and both operands of a weight gradient, whose sum runs over
// rows).  The five products of the block are instances with an epilogue each
// (Mode), so that the gate's activation, its product and their derivatives
// never travel through memory as fp32.
//
// A workgroup computes a BM x BN tile in steps of 128 bytes along k through two LDS
// buffers, filled straight from memory (buffer loads with the LDS as their destination:
// no registers, no LDS write instructions).  While the first half of step t is multiplied
// the second half's fragments are read into registers; then one barrier, behind which
// step t's buffer is refilled with step t + 2 and the first half of step t + 1 is read
// while the second half of step t is multiplied: the barrier finds every wave with its
// next operands in registers.  Rows past the end of a matrix fall outside the
// descriptor's range and arrive as zeros; what a K-contiguous operand's last step brings of
// the next rows is cleared in LDS.  (The loads need rows at
// multiples of four bytes: rows of an odd number of bf16 go through registers instead.)
//
// LDS layouts (16-byte chunks; the loads fill LDS in lane order, so a layout is
// made by choosing what each lane reads):
//   K-contiguous  row r: 128 bytes, chunk c at place c ^ (r / 2 mod 8): the 16 rows
//                 that a 128-bit fragment read touches at one c cover all banks once
//   K-strided     row k: BM elements.  bf16: 32-byte segments s at place s ^ f(k), f the
//                 eight rows that two 16-lane groups of a transposing read touch (rows of 128
//                 bytes: four of each parity); fp32:
//                 64-byte segments at s ^ (k / 4 mod 4), the four rows of a 32-bit read
// Fragments of K-strided bf16 operands come out of LDS through the transposing 64-bit
// read (16 lanes read 4 k of 16 columns, lane i gets column i's 4 k).
//
// What is rounded: bf16 calls round h between the products, and du, dv and h in the backward pass, to
// bf16, since the matrix cores take them as bf16 (fp32 operands run at a tenth of the rate, see
// below).  The rounding of an element, 2^-9 at most, is of random sign and averages out over the
// next sum: errors of the results 0.0023 (2-norm) where rounding them alone makes 0.0017.  u and v are kept
// in the model's type, as the caller asked for them.  The gate in the epilogue works with the unrounded sums.
//
// The matrix instruction gets B's fragment first, so that a lane ends with four
// consecutive n of one row m: 8- or 16-byte stores.
//
// What bounds it: a step of a 256 x 256 tile is 2048 cycles of each matrix core and, at 128 bytes a cycle,
// 1536 of fragment reads and 512 of arriving loads in LDS; both run at once only if nothing
// waits, so reads and loads are placed between single matrix instructions (all of a row of pieces'
// at its start: 5 % slower).  The card's power sets the clock under this load (zeros as inputs
// run a fifth faster).  Four waves of 128 x 128 read a third less LDS, but alone on a SIMD each
// waits for itself: down 899 us where these take 798.
// Measured, M=8192 D=4096 F=14336 bf16: gate and up 1750-1800 us (1.08 PFLOP/s, with 705 MB stored), down 800-815
// (1.20), hidden gradient 997-1071 (0.94, 1.2 GB through its epilogue), input gradient 1420 (1.36),
// weight gradients of four tasks 2380-2570 (1.17), of one 2215.  Rows at two bytes alone (through registers): the weight
// gradients' kernel keeps 69 registers in scratch memory (fp32 29), gate and up 12.
// fp32, M=1024 D=1024 F=4096: gate and up 142 us (121 TFLOP/s),
// weight gradients 205 (126).
#pragma once

#include <type_traits>

#include "elem.h"
#include "ffn.h"
#include "mfma.h"

namespace bkmoo {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// One step of an operand into LDS.  W rows of the tile along m (or n); the
// workgroup's waves take equal shares of its 1-KiB pieces.
template <typename T, int W, bool KC, int WAVES>
struct Stage {
  static constexpr int kES = sizeof(T);
  static constexpr int kBK = 128 / kES;            // k of a step
  static constexpr int kChunks = W * 8;            // 16-byte chunks of a step
  static constexpr int kPieces = kChunks / 64;     // pieces of a wave's load
  static constexpr int kPer = kPieces / WAVES;     // pieces of each wave
  static constexpr int kBytes = W * 128;
  static constexpr int kCPR = KC ? 8 : W * kES / 16;  // chunks of an LDS row
  static_assert(kPieces % WAVES == 0, "whole pieces");

  // Row of the tile's LDS image (m if KC, else k) and logical chunk in it of
  // piece q's lane.
  static __device__ __forceinline__ void place(int q, int lane, int &row, int &chunk) {
    const int f = q * 64 + lane;
    row = f / kCPR;
    const int p = f % kCPR;
    if (KC)
      chunk = p ^ ((row >> 1) & 7);
    else if (kES == 2)
      chunk = p ^ (2 * (W >= 128 ? (row & 3) | ((row >> 1) & 4) : ((row >> 1) & 1) | ((row >> 2) & 2)));
    else
      chunk = p ^ (4 * ((row >> 2) & 3));
  }

  // Byte offsets of the wave's pieces from the step's first element.  HALF > 0: the
  // rows are HALF of one matrix and HALF of another in turn; the offset is in the
  // row's own matrix.
  template <int HALF>
  static __device__ __forceinline__ void offsets(int wave, int lane, int64_t ld, uint32_t *off) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      int row, chunk;
      place(wave * kPer + i, lane, row, chunk);
      if (HALF > 0) row = row / (2 * HALF) * HALF + row % HALF;
      off[i] = (uint32_t)row * (uint32_t)(ld * kES) + (uint32_t)chunk * 16;
    }
  }

  // Piece i (eight rows) reads the second matrix.
  template <int HALF>
  static __device__ __forceinline__ bool second(int wave, int i) {
    if constexpr (HALF > 0) return ((wave * kPer + i) * 8 / HALF) & 1;
    return false;
  }
};

// The matrix an operand's step is read from: `rows` rows of ld elements.
template <typename T>
struct Source {
  const T *p;
  int64_t ld, rows;
};

template <typename T, int W, bool KC>
struct Reader {
  uint32_t base[2], x;
  // first: the wave's first row in the tile
  __device__ __forceinline__ Reader(int first, int lane) {
    const int g = lane >> 4, j = lane & 15;
    if constexpr (KC) {
      const int s = (j >> 1) & 7;
      base[0] = (uint32_t)((first + j) * 128 + 16 * (g ^ s));
      base[1] = (uint32_t)((first + j) * 128 + 16 * ((4 + g) ^ s));
      x = 0;
    } else if constexpr (sizeof(T) == 2) {
      const int k = 8 * g + (j >> 2);
      base[0] = (uint32_t)(k * W * 2 + 8 * (j & 3));
      const int f = W >= 128 ? (j >> 2) | ((g & 1) << 2) : (j >> 3) | ((g & 1) << 1);
      x = (uint32_t)(32 * f) ^ (uint32_t)(first * 2);
    } else {
      base[0] = (uint32_t)(4 * g * W * 4 + 4 * j);
      x = (uint32_t)(64 * g) ^ (uint32_t)(first * 4);
    }
  }
  // (a pointer, so that what is added to it becomes the instruction's offset)
  static __device__ __forceinline__ const BKMOO_LDS char *at(uint32_t a) {
    return (const BKMOO_LDS char *)(uintptr_t)a;
  }
  // Fragment i of a half of the step at LDS address `lds`.
  __device__ __forceinline__ Frag<T> read(uint32_t lds, int half, int i) const {
    Frag<T> f;
    if constexpr (KC) {
      f.v = *(const BKMOO_LDS decltype(f.v) *)(at(lds + base[half]) + i * 16 * 128);
    } else if constexpr (sizeof(T) == 2) {
      const BKMOO_LDS char *a = at(lds + base[0] + (x ^ (uint32_t)(i * 32))) + half * 32 * W * 2;
      union {
        s16x4 h[2];
        bf16x8 v;
      } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((BKMOO_LDS s16x4 *)a);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((BKMOO_LDS s16x4 *)(a + 4 * W * 2));
      f.v = u.v;
    } else {
      // rows 16 half + 4 g + e: their place depends on g alone
      const BKMOO_LDS char *a = at(lds + base[0] + (x ^ (uint32_t)(i * 64))) + half * 16 * W * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) f.v[e] = *(const BKMOO_LDS float *)(a + e * W * 4);
    }
    return f;
  }
};

// A lane holds four columns, from 4 (lane / 16) on, of each of two neighbouring 16 x 16
// pieces.  Sixteen-lane rows 1 and 3 of the first trade places with rows 0 and 2 of the
// second: eight consecutive columns, from 16 (lane / 16 mod 2) + 8 (lane / 32) on.
__device__ __forceinline__ void eight_columns(f32x4 a, f32x4 b, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[e]), __float_as_uint(b[e]), false, false);
    x[e] = __uint_as_float(r[0]);
    x[e + 4] = __uint_as_float(r[1]);
  }
}

// Tile number -> (row of tiles, column of tiles).  Workgroups go to the eight
// XCDs in turn; each XCD gets a run of consecutive numbers, and consecutive
// numbers cover patches of kPatch rows of tiles, so that the tiles in flight on
// an XCD share rows of A and of B in its L2.
constexpr int kXcds = 8;
constexpr int kPatch = 8;
__device__ __forceinline__ int xcd_order(int id, int n) {
  const int q = n / kXcds, r = n % kXcds, x = id % kXcds;
  return x * q + (x < r ? x : r) + id / kXcds;
}
__device__ __forceinline__ void tile_of(int id, int tm, int tn, int &m, int &n) {
  const int per = kPatch * tn, patch = id / per, first = patch * kPatch;
  const int rows = tm - first < kPatch ? tm - first : kPatch;
  m = first + (id % per) % rows;
  n = (id % per) / rows;
}

// f(0), f(1), ... f(N - 1), each with its number as a constant.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void in_turn(F &&f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    in_turn<N, I + 1>(f);
  }
}
// How many of `count` things spread over `places` places come before place p.
constexpr int due(int count, int places, int p) {
  int n = 0;
  while (n < count && n * places / count < p) ++n;
  return n;
}

// What becomes of a wave's sums.
template <typename T, Mode MODE, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void store_tile(const TileArgs &g, const f32x4 (&acc)[BM / WM / 16][BN / WN / 16], int prob,
                                           int64_t m0, int64_t n0, int64_t Mo, int64_t No, int wm, int wn, int lane) {
  constexpr bool GU = MODE == kGateUp;
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16, kHalf = GU ? BN / WN / 2 : 0;
  // Two neighbouring pieces are exchanged between the lanes so that each holds eight consecutive
  // columns (kPairs of them a row of pieces): 16-byte accesses (bf16).  `whole`: all eight are
  // there, n of them else.
  const int64_t mrow = m0 + wm * TM * 16 + (lane & 15);
  const int64_t nwave = n0 + wn * (GU ? kHalf : TN * 16) + 16 * ((lane >> 4) & 1) + 8 * (lane >> 5);
  const bool inside = m0 + BM <= Mo && n0 + (GU ? BN / 2 : BN) <= No;
  constexpr int kPairs = (GU ? TN / 2 : TN) / 2;
  static_assert(kPairs > 0, "whole pairs of pieces");
  auto each = [&](auto all, auto &&f) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int q = 0; q < kPairs; ++q) {
        const int64_t m = mrow + i * 16, n = nwave + q * 32;
        const int64_t left = decltype(all)::value || m < Mo ? No - n : 0;
        f(all, i, q, m * No + n, decltype(all)::value || left >= 8 ? 8 : left > 0 ? (int)left : 0);
      }
  };
  auto everywhere = [&](auto &&f) {
    if (inside)
      each(std::true_type{}, f);
    else
      each(std::false_type{}, f);
  };
  // eight elements, or the first n of them
  auto put = [](auto all, auto *p, const float (&x)[8], int n) {
    using E = std::remove_reference_t<decltype(*p)>;
    if (decltype(all)::value || n == 8) {
      store8(p, x);
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = (E)x[e];
  };
  if constexpr (MODE == kGateUp) {
    T *h = (T *)g.out[0], *su = (T *)g.out[1], *sv = (T *)g.out[2];
    const bool keep = su != nullptr;
    everywhere([&](auto all, int i, int q, int64_t at, int n) {
      float u[8], v[8], x[8];
      eight_columns(acc[i][2 * q], acc[i][2 * q + 1], u);
      eight_columns(acc[i][TN / 2 + 2 * q], acc[i][TN / 2 + 2 * q + 1], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = gate_act<T>(u[e], g.act) * v[e];
      put(all, h + at, x, n);
      if (keep) {
        put(all, su + at, u, n);
        put(all, sv + at, v, n);
      }
    });
  } else if constexpr (MODE == kHiddenGrad) {
    const T *pu = (const T *)g.u, *pv = (const T *)g.v;
    T *du = (T *)g.out[0], *dv = (T *)g.out[1], *h = (T *)g.out[2];
    auto finish = [&](auto all, int i, int q, int64_t at, int n, const float (&u)[8], const float (&v)[8]) {
      float d[8], xu[8], xv[8], xh[8];
      eight_columns(acc[i][2 * q], acc[i][2 * q + 1], d);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float a, da;
        gate_act_grad<T>(u[e], g.act, a, da);
        xu[e] = d[e] * v[e] * da;
        xv[e] = d[e] * a;
        xh[e] = a * v[e];
      }
      put(all, du + at, xu, n);
      put(all, dv + at, xv, n);
      put(all, h + at, xh, n);
    };
    // u and v of the next row of pieces travel while this one is worked on (past an end: of the
    // last row or zeros; there tiles of 256 load them where they are used: the code for both ends
    // left 21 registers in scratch memory, and 42 with a form for the parts of a split sum beside them, where this
    // has 4: 8192 x 4096 x 14336 1031 us, 1011 and 997)
    Eight<T> nu[2][kPairs], nv[2][kPairs];
    auto ask = [&](auto all, int i) {
#pragma unroll
      for (int q = 0; q < kPairs; ++q) {
        const int64_t m = mrow + i * 16, n = nwave + q * 32;
        if constexpr (decltype(all)::value) {
          nu[i & 1][q] = load8(pu + m * No + n);
          nv[i & 1][q] = load8(pv + m * No + n);
        } else {
          const int64_t row = (m < Mo ? m : Mo - 1) * No;
          nu[i & 1][q] = guarded_load8(pu + row, n, No);
          nv[i & 1][q] = guarded_load8(pv + row, n, No);
        }
      }
    };
    auto work = [&](auto all) {
      ask(all, 0);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i + 1 < TM) ask(all, i + 1);
#pragma unroll
        for (int q = 0; q < kPairs; ++q) {
          float u[8], v[8];
          nu[i & 1][q].get(u);
          nv[i & 1][q].get(v);
          const int64_t m = mrow + i * 16, n = nwave + q * 32;
          const int64_t left = decltype(all)::value || m < Mo ? No - n : 0;
          finish(all, i, q, m * No + n, decltype(all)::value || left >= 8 ? 8 : left > 0 ? (int)left : 0, u, v);
        }
      }
    };
    if (inside)
      work(std::true_type{});
    else if constexpr (BM < 256)
      work(std::false_type{});
    else
      each(std::false_type{}, [&](auto all, int i, int q, int64_t at, int n) {
        float u[8], v[8];
        const int64_t m = mrow + i * 16, row = (m < Mo ? m : Mo - 1) * No;
        guarded_load8(pu + row, nwave + q * 32, No).get(u);
        guarded_load8(pv + row, nwave + q * 32, No).get(v);
        finish(all, i, q, at, n, u, v);
      });
  } else if constexpr (MODE == kHiddenPart) {
    float *part = g.partial + (int64_t)prob * Mo * No;
    everywhere([&](auto all, int i, int q, int64_t at, int n) {
      float x[8];
      eight_columns(acc[i][2 * q], acc[i][2 * q + 1], x);
      put(all, part + at, x, n);
    });
  } else {
    T *out = MODE == kWeightGrad ? (T *)g.out[prob % 3] + (prob / 3) * g.task_stride : (T *)g.out[0];
    float *part = nullptr;
    if constexpr (MODE == kDown || MODE == kInputGrad)
      if (g.splits > 1) part = g.partial + (int64_t)prob * Mo * No;
    everywhere([&](auto all, int i, int q, int64_t at, int n) {
      float x[8];
      eight_columns(acc[i][2 * q], acc[i][2 * q + 1], x);
      if (part)
        put(all, part + at, x, n);
      else
        put(all, out + at, x, n);
    });
  }
}

// The epilogue's stores that a wave has certainly queued after a tile inside the
// matrices (at most what the counter holds).
template <typename T, Mode MODE, int TM, int TN>
constexpr int kTileStores = [] {
  const int pairs = TM * (MODE == kGateUp ? TN / 2 : TN) / 2 * (sizeof(T) == 4 ? 2 : 1);
  const int n = MODE == kHiddenGrad ? 3 * pairs : pairs;
  return n < 63 ? n : 63;
}();

template <typename T, Mode MODE, int BM, int BN, int WM, int WN, bool ALIGNED>
__global__ __launch_bounds__(64 * WM * WN, 2) void ffn_tile_kernel(const TileArgs g) {
  constexpr int kWaves = WM * WN;
  constexpr bool AKC = MODE != kWeightGrad;
  constexpr bool BKC = MODE == kGateUp || MODE == kDown;
  constexpr bool GU = MODE == kGateUp;
  using SA = Stage<T, BM, AKC, kWaves>;
  using SB = Stage<T, BN, BKC, kWaves>;
  constexpr int BK = SA::kBK, ES = sizeof(T);
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 pieces of a wave's tile
  constexpr int kStep = SA::kBytes + SB::kBytes;
  // a wave holds kHalf columns of the gate and the same kHalf of the up product
  constexpr int kHalf = GU ? BN / WN / 2 : 0;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * kStep];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(BKMOO_LDS unsigned char *)lds;
  const int tiles = g.tiles_m * g.tiles_n, total = tiles * g.problems;
  constexpr bool kMany = MODE != kHiddenGrad && MODE != kHiddenPart;  // tiles a workgroup (at least one: the grid is no larger)

  // A tile: its problem, its place, and its steps t0 to t1 (all, or its share of a
  // split sum).
  struct Tile {
    int prob, steps_seg, t0, t1;
    int64_t m0, n0, M, N, K;
  };
  auto tile = [&](int round) {
    const int first = round * (int)gridDim.x, here = total - first < (int)gridDim.x ? total - first : (int)gridDim.x;
    int id = first + xcd_order(blockIdx.x, here);
    Tile x;
    x.prob = id / tiles;
    id -= x.prob * tiles;
    x.M = g.M;
    x.N = g.N;
    x.K = g.K;
    int tm = g.tiles_m, tn = g.tiles_n, im, in;
    if constexpr (MODE == kWeightGrad) {
      // problem: (task, matrix); the sum runs over the task's rows
      const int task = x.prob / 3;
      if (x.prob % 3 == 2) {  // [D][F] = dy^T h: the other two are [F][D]
        x.M = g.N;
        x.N = g.M;
        tm = g.tiles_n;
        tn = g.tiles_m;
      }
      x.K = g.rows[task + 1] - g.rows[task];
    }
    tile_of(id, tm, tn, im, in);
    x.m0 = (int64_t)im * BM;
    x.n0 = (int64_t)in * (GU ? BN / 2 : BN);
    x.steps_seg = (int)((x.K + BK - 1) / BK);
    x.t0 = 0;
    x.t1 = x.steps_seg * (MODE == kInputGrad ? 2 : 1);
    if constexpr (MODE == kDown || MODE == kHiddenPart || MODE == kInputGrad) {
      if (g.splits > 1) {
        const int per = (x.t1 + g.splits - 1) / g.splits;
        x.t0 = x.prob * per < x.t1 ? x.prob * per : x.t1;
        x.t1 = x.t0 + per < x.t1 ? x.t0 + per : x.t1;
      }
    }
    return x;
  };
  // Its operands: the matrix (of the segment of the sum that step t is in) and its rows.
  auto source_a = [&](const Tile &x, int seg) {
    if constexpr (MODE == kWeightGrad) return Source<T>{(const T *)g.a[x.prob % 3] + g.rows[x.prob / 3] * x.M, x.M, x.K};
    return Source<T>{(const T *)(seg ? g.a[1] : g.a[0]), x.K, x.M};
  };
  auto source_b = [&](const Tile &x, int seg) {
    if constexpr (MODE == kWeightGrad) return Source<T>{(const T *)g.b[x.prob % 3] + g.rows[x.prob / 3] * x.N, x.N, x.K};
    const T *p = (const T *)(seg ? g.b[1] : g.b[0]);
    return BKC ? Source<T>{p, x.K, x.N} : Source<T>{p, x.N, x.K};
  };

  // The stream of steps to load (ALIGNED): those of all this workgroup's tiles, one after
  // another, so that the next tile's first steps travel while a tile ends.  Where the
  // next one starts, and the bytes from there to its matrix's end; none after the last
  // step: its loads bring zeros.
  struct Next {
    const char *a, *b, *b2;
    int64_t abytes, bbytes, astep, bstep;
    int left, t, seg_end, t1, round;  // left: of the segment's sum
  } nx = {};
  uint32_t aoff[SA::kPer], boff[SB::kPer];
  auto start_at = [&](const Tile &x, int t) {
    const int seg = MODE == kInputGrad && t >= x.steps_seg ? 1 : 0;
    const int64_t k0 = (int64_t)(t - seg * x.steps_seg) * BK;
    const Source<T> A = source_a(x, seg), B = source_b(x, seg);
    const int64_t ea = AKC ? x.m0 * A.ld + k0 : k0 * A.ld + x.m0;
    const int64_t eb = BKC ? x.n0 * B.ld + k0 : k0 * B.ld + x.n0;
    nx.a = (const char *)(A.p + ea);
    nx.b = (const char *)(B.p + eb);
    nx.b2 = GU ? (const char *)((const T *)g.b[1] + eb) : nx.b;
    nx.abytes = (A.rows * A.ld - ea) * ES;
    nx.bbytes = (B.rows * B.ld - eb) * ES;
    nx.astep = AKC ? 128 : BK * A.ld * ES;
    nx.bstep = BKC ? 128 : BK * B.ld * ES;
    nx.left = (int)(x.K - k0);
    nx.t = t;
    // (a part of a split sum may end before its segment does)
    nx.seg_end = MODE == kInputGrad && seg == 0 && x.steps_seg < x.t1 ? x.steps_seg : x.t1;
    nx.t1 = x.t1;
  };
  auto start_tile = [&](int round) {
    for (; round == 0 || (kMany && round * (int)gridDim.x + (int)blockIdx.x < total); ++round) {
      const Tile x = tile(round);
      if (x.t0 >= x.t1) continue;
      if (MODE == kWeightGrad || nx.t1 == 0) {
        SA::template offsets<0>(wave, lane, source_a(x, 0).ld, aoff);
        SB::template offsets<kHalf>(wave, lane, source_b(x, 0).ld, boff);
      }
      start_at(x, x.t0);
      nx.round = round;
      return;
    }
    nx.abytes = nx.bbytes = nx.astep = nx.bstep = 0;
    nx.seg_end = nx.t1 = 0x7fffffff;
    nx.t = 0;
  };
  struct Step {
    i32x4 a, b, b2;
    uint32_t la, lb;
    int left;
  };
  auto next_step = [&](int buf) {
    Step x;
    x.a = make_desc(nx.a, nx.abytes);
    x.b = make_desc(nx.b, nx.bbytes);
    x.b2 = GU ? make_desc(nx.b2, nx.bbytes) : x.b;
    x.la = lds0 + buf * kStep + wave * SA::kPer * 1024;
    x.lb = lds0 + buf * kStep + SA::kBytes + wave * SB::kPer * 1024;
    x.left = nx.left;
    nx.a += nx.astep;
    nx.b += nx.bstep;
    nx.b2 += nx.bstep;
    nx.abytes -= nx.astep;
    nx.bbytes -= nx.bstep;
    nx.left -= BK;
    ++nx.t;
    return x;
  };
  // Behind the loads of a step: the offsets may be another matrix's from here on.
  auto move_on = [&]() {
    if (nx.t < nx.seg_end) return;
    if (MODE == kInputGrad && nx.t < nx.t1)
      start_at(tile(nx.round), nx.t);
    else
      start_tile(nx.round + 1);
  };
  constexpr int kLoads = SA::kPer + SB::kPer;
  auto piece = [&](const Step &x, int i) {
    if (i < SA::kPer) {
      load_to_lds(x.la + i * 1024, x.a, aoff[i]);
    } else {
      const int q = i - SA::kPer;
      load_to_lds(x.lb + q * 1024, SB::template second<kHalf>(wave, q) ? x.b2 : x.b, boff[q]);
    }
  };

  // The step that a sum ends in: what the loads brought of the next rows is cleared, by the
  // lane that loaded it.
  auto clear = [&](const Step &x) {
    if ((!AKC && !BKC) || x.left >= BK) return;
    int at = lane;
    asm volatile("" : "+v"(at));  // worked out here, once a tile: no registers for it in the loop
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool isa = i < SA::kPer;
      if (isa ? !AKC : !BKC) continue;
      const int q = isa ? i : i - SA::kPer;
      int row, chunk;
      if (isa)
        SA::place(wave * SA::kPer + q, at, row, chunk);
      else
        SB::place(wave * SB::kPer + q, at, row, chunk);
      const int keep = (x.left - chunk * (16 / ES)) * ES;
      if (keep < 16) keep_bytes((isa ? x.la : x.lb) + q * 1024 + at * 16, keep);
    }
  };

  // Steps through registers, element by element where a chunk crosses an end (!ALIGNED).
  u32x4 ra[ALIGNED ? 1 : SA::kPer], rb[ALIGNED ? 1 : SB::kPer];
  auto fetch = [&](const Tile &x, int t) {
    if constexpr (!ALIGNED) {
      const int seg = MODE == kInputGrad && t >= x.steps_seg ? 1 : 0;
      const int64_t k0 = (int64_t)(t - seg * x.steps_seg) * BK;
      const Source<T> A = source_a(x, seg), B = source_b(x, seg);
#pragma unroll
      for (int i = 0; i < SA::kPer; ++i) {
        int row, chunk;
        SA::place(wave * SA::kPer + i, lane, row, chunk);
        const int64_t r = (AKC ? x.m0 : k0) + row, c = (AKC ? k0 : x.m0) + chunk * (16 / ES);
        ra[i] = r < A.rows ? guarded_chunk(A.p + r * A.ld, c, A.ld) : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < SB::kPer; ++i) {
        int row, chunk;
        SB::place(wave * SB::kPer + i, lane, row, chunk);
        const T *p = GU && SB::template second<kHalf>(wave, i) ? (const T *)g.b[1] : B.p;
        if constexpr (GU) row = row / (2 * kHalf) * kHalf + row % kHalf;
        const int64_t r = (BKC ? x.n0 : k0) + row, c = (BKC ? k0 : x.n0) + chunk * (16 / ES);
        rb[i] = r < B.rows ? guarded_chunk(p + r * B.ld, c, B.ld) : u32x4{0, 0, 0, 0};
      }
    }
  };
  auto put = [&](int buf) {
    if constexpr (!ALIGNED) {
      const uint32_t la = lds0 + buf * kStep + wave * SA::kPer * 1024 + lane * 16;
      const uint32_t lb = lds0 + buf * kStep + SA::kBytes + wave * SB::kPer * 1024 + lane * 16;
#pragma unroll
      for (int i = 0; i < SA::kPer; ++i) *(BKMOO_LDS u32x4 *)(uintptr_t)(la + i * 1024) = ra[i];
#pragma unroll
      for (int i = 0; i < SB::kPer; ++i) *(BKMOO_LDS u32x4 *)(uintptr_t)(lb + i * 1024) = rb[i];
    }
  };

  f32x4 acc[TM][TN];
  const int wm = wave / WN, wn = wave % WN;
  const Reader<T, BM, AKC> reada(wm * TM * 16, lane);
  const Reader<T, BN, BKC> readb(wn * TN * 16, lane);

  // Fragments of both halves of a step: one is multiplied while the other is read.
  Frag<T> fa[2][TM], fb[2][TN];
  auto read = [&](int half, int buf, int i) {
    const uint32_t la = lds0 + buf * kStep;
    if (i < TN)
      fb[half][i] = readb.read(la + SA::kBytes, half, i);
    else
      fa[half][i - TN] = reada.read(la, half, i - TN);
  };
  // The products of a half, row by row of pieces, with the reads of the other half (of
  // the step in LDS buffer `buf`) and, LOAD, the loads of a step in between: none holds up
  // another, and every read (within the first three quarters) has arrived when the half ends.
  auto work = [&](auto half, auto loads, int buf, const Step &x) {
    constexpr int HALF = decltype(half)::value;
    constexpr bool LOAD = decltype(loads)::value;
    constexpr int kReads = TM + TN, kAll = TM * TN;
    in_turn<kAll>([&](auto at) {
      constexpr int P = decltype(at)::value;
#pragma unroll
      for (int q = due(kReads, kAll * 3 / 4, P); q < due(kReads, kAll * 3 / 4, P + 1); ++q) read(HALF ^ 1, buf, q);
      if constexpr (LOAD)
#pragma unroll
        for (int q = due(kLoads, kAll, P); q < due(kLoads, kAll, P + 1); ++q) piece(x, q);
      constexpr int i = P / TN, j = P % TN;
      acc[i][j] = multiply(fb[HALF][j], fa[HALF][i], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  using First = std::integral_constant<int, 0>;
  using Second = std::integral_constant<int, 1>;
  using Loads = std::bool_constant<ALIGNED>;

  Step x = {}, ahead = {};  // ahead: the last one loaded
  if constexpr (ALIGNED) {
    start_tile(0);
    x = next_step(0);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) piece(x, q);
    move_on();
    ahead = next_step(1);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) piece(ahead, q);
    move_on();
    wait_loads<kLoads>();
    clear(x);
    barrier_lds();
  }
  int buf = 0;
  bool stored = false;  // since the last wait: a tile inside the matrices
  for (int round = 0; round == 0 || (kMany && round * (int)gridDim.x + (int)blockIdx.x < total); ++round) {
    const Tile z = tile(round);
    const int n = z.t1 - z.t0;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    if constexpr (!ALIGNED) {
      barrier_lds();
      buf = 0;
      for (int i = 0; i < 2 && i < n; ++i) {
        fetch(z, z.t0 + i);
        put(i);
      }
      barrier_lds();
    }
    if (n > 0) {
#pragma unroll
      for (int i = 0; i < TM + TN; ++i) read(0, buf, i);
    }
    for (int t = 0; t < n; ++t, buf ^= 1) {
      if constexpr (ALIGNED)
        x = next_step(buf);
      else if (t + 2 < n)
        fetch(z, z.t0 + t + 2);
      work(First{}, std::false_type{}, buf, x);
      // Step t is in registers and step t + 1 in LDS, for every wave: step t's
      // buffer is free.  (The stores of the tile before need not have ended: they were
      // queued behind the loads waited for.)
      if constexpr (ALIGNED) {
        if (stored)
          wait_loads<kTileStores<T, MODE, TM, TN>>();
        else
          wait_loads<0>();
        stored = false;
        clear(ahead);
        ahead = x;
      }
      barrier_lds();
      work(Second{}, Loads{}, buf ^ 1, x);  // (after the last step: reads what is there)
      if constexpr (ALIGNED)
        move_on();
      else if (t + 2 < n)
        put(buf);
      asm volatile("" ::: "memory");  // the reads stay in this iteration
    }
    stored = z.m0 + BM <= z.M && z.n0 + (GU ? BN / 2 : BN) <= z.N;
    store_tile<T, MODE, BM, BN, WM, WN>(g, acc, z.prob, z.m0, z.n0, z.M, z.N, wm, wn, lane);
  }
  if constexpr (ALIGNED) wait_loads<0>();  // LDS is still being written
}

}  // namespace bkmoo
