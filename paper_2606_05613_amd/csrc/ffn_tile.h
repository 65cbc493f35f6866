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
// A workgroup computes a BM x BN tile.  It takes steps of 128 bytes along k
// through two LDS buffers: while the waves multiply step t, step t + 1 travels
// from memory straight into the other buffer (buffer loads with the LDS as their
// destination: no registers, no LDS write instructions), and one barrier a step
// hands it over.  Rows past the end of a matrix fall outside the descriptor's
// range and arrive as zeros; so do the chunks past K of a K-contiguous operand.
//
// LDS layouts (16-byte chunks; the loads fill LDS in lane order, so a layout is
// made by choosing what each lane reads):
//   K-contiguous  row r: 128 bytes, chunk c at place c ^ (r / 2 mod 8): the 16 rows
//                 that a 128-bit fragment read touches at one c cover all banks once
//   K-strided     row k: BM elements.  bf16: 32-byte segments s at place s ^ f(k), f the
//                 eight rows that two 16-lane groups of a transposing read touch; fp32:
//                 64-byte segments at s ^ (k / 4 mod 4), the four rows of a 32-bit read
// Fragments of K-strided bf16 operands come out of LDS through the transposing 64-bit
// read (16 lanes read 4 k of 16 columns, lane i gets column i's 4 k).
//
// The matrix instruction gets B's fragment first, so that a lane ends with four
// consecutive n of one row m: 8- or 16-byte stores.
#pragma once

#include "elem.h"
#include "ffn.h"

namespace bkmoo {

#define BKMOO_LDS __attribute__((address_space(3)))

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Gate activation and its derivative.
__device__ __forceinline__ float gate_act(float u, int act) {
  if (act == kSilu) return u / (1.0f + expf(-u));
  // GELU's tanh form: u times the logistic function of twice tanh's argument
  const float z = 1.5957691216057308f * (u + 0.044715f * u * u * u);
  return u / (1.0f + expf(-z));
}
__device__ __forceinline__ void gate_act_grad(float u, int act, float &a, float &da) {
  float z = u, dz = 1.0f;
  if (act != kSilu) {
    z = 1.5957691216057308f * (u + 0.044715f * u * u * u);
    dz = 1.5957691216057308f * (1.0f + 0.134145f * u * u);
  }
  const float s = 1.0f / (1.0f + expf(-z));
  a = u * s;
  // u s (1 - s) dz: 1 - s as the logistic function of -z, exact for large z
  const float r = 1.0f / (1.0f + expf(z));
  const float q = s * r;
  da = q == 0.0f ? s : s + u * q * dz;
}

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
      chunk = p ^ (2 * ((row & 3) | ((row >> 1) & 4)));
    else
      chunk = p ^ (4 * ((row >> 2) & 3));
  }

  // Byte offsets of the wave's pieces from the step's first element.  GU: the
  // rows are 32 of one matrix and 32 of another in turn; the offset is in the
  // row's own matrix.
  template <bool GU>
  static __device__ __forceinline__ void offsets(int wave, int lane, int64_t ld, uint32_t *off) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      int row, chunk;
      place(wave * kPer + i, lane, row, chunk);
      if (GU) row = (row >> 6) * 32 + (row & 31);
      off[i] = (uint32_t)row * (uint32_t)(ld * kES) + (uint32_t)chunk * 16;
    }
  }

  // Piece i reads the second matrix (GU).
  static __device__ __forceinline__ bool second(int wave, int i) { return ((wave * kPer + i) >> 2) & 1; }
};

__device__ __forceinline__ i32x4 make_desc(const void *p, int64_t bytes) {
  const uint64_t a = (uint64_t)p;
  const int64_t n = bytes < 0 ? 0 : bytes < 0x7fffffff ? bytes : 0x7fffffff;
  i32x4 r;
  r.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r.y = __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffff));
  r.z = __builtin_amdgcn_readfirstlane((int)n);
  r.w = 0x00020000;
  return r;
}

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane; beyond the descriptor's
// range zeros.  No register is written: what it leaves outstanding is waited for
// by wait_loads() alone.  (M0 holds the LDS address; nothing else here uses it.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, i32x4 desc, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(off), "s"(desc)
               : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Every wave's LDS reads have returned and its LDS writes are done.
__device__ __forceinline__ void barrier_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
constexpr uint32_t kNowhere = 0x80000000u;  // beyond every descriptor's range

// The matrix an operand's step is read from: `rows` rows of ld elements.
template <typename T>
struct Source {
  const T *p;
  int64_t ld, rows;
};

// Fragments: 16 rows (or columns) of an operand and 64 bytes of k.
template <typename T>
struct Frag;
template <>
struct Frag<__bf16> {
  bf16x8 v;
};
template <>
struct Frag<float> {
  f32x4 v;
};

template <typename T, int W, bool KC>
struct Reader {
  uint32_t base[2];
  uint32_t x;
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
      base[1] = 0;
      x = (uint32_t)(32 * ((j >> 2) | ((g & 1) << 2))) ^ (uint32_t)(first * 2);
    } else {
      base[0] = (uint32_t)(4 * g * W * 4 + 4 * j);
      base[1] = 0;
      x = (uint32_t)(64 * g) ^ (uint32_t)(first * 4);
    }
  }
  // Fragment i of half kk of the step at LDS address `lds`.
  __device__ __forceinline__ Frag<T> read(uint32_t lds, int kk, int i) const {
    Frag<T> f;
    if constexpr (KC) {
      f.v = *(const BKMOO_LDS decltype(f.v) *)(uintptr_t)(lds + base[kk] + i * 16 * 128);
    } else if constexpr (sizeof(T) == 2) {
      const uint32_t a = lds + base[0] + (x ^ (uint32_t)(i * 32)) + kk * 32 * W * 2;
      union {
        s16x4 h[2];
        bf16x8 v;
      } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((BKMOO_LDS s16x4 *)(uintptr_t)a);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((BKMOO_LDS s16x4 *)(uintptr_t)(a + 4 * W * 2));
      f.v = u.v;
    } else {
      // rows 16 kk + 4 g + e: their place depends on g alone
      const uint32_t a = lds + base[0] + (x ^ (uint32_t)(i * 64)) + kk * 16 * W * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) f.v[e] = *(const BKMOO_LDS float *)(uintptr_t)(a + e * W * 4);
    }
    return f;
  }
};

__device__ __forceinline__ f32x4 multiply(const Frag<__bf16> &n, const Frag<__bf16> &m, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(n.v, m.v, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(const Frag<float> &n, const Frag<float> &m, f32x4 acc) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(n.v[e], m.v[e], acc, 0, 0, 0);
  return acc;
}

// Tile number -> (row of tiles, column of tiles).  Workgroups go to the eight
// XCDs in turn; each XCD gets a run of consecutive numbers, and consecutive
// numbers cover patches of kPatch rows of tiles, so that the tiles in flight on
// an XCD share rows of A and of B in its L2.
constexpr int kXcds = 8;
constexpr int kPatch = 4;
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

template <typename T, Mode MODE, int BM, int BN, int WM, int WN, bool ALIGNED>
__global__ __launch_bounds__(64 * WM * WN) void ffn_tile_kernel(const TileArgs g) {
  constexpr int kWaves = WM * WN;
  constexpr bool AKC = MODE != kWeightGrad;
  constexpr bool BKC = MODE == kGateUp || MODE == kDown;
  constexpr bool GU = MODE == kGateUp;
  using SA = Stage<T, BM, AKC, kWaves>;
  using SB = Stage<T, BN, BKC, kWaves>;
  constexpr int BK = SA::kBK, ES = sizeof(T);
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 pieces of a wave's tile
  constexpr int kStep = SA::kBytes + SB::kBytes;
  static_assert(!GU || BN / WN == 64, "a wave holds 32 columns of the gate and the same 32 of the up product");
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * kStep];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

  // this workgroup's problem and tile
  const int tiles = g.tiles_m * g.tiles_n;
  int id = xcd_order(blockIdx.x, gridDim.x);
  const int prob = id / tiles;
  id -= prob * tiles;
  Source<T> a[2] = {}, b[2] = {};
  int segs = 1, tm = g.tiles_m, tn = g.tiles_n;
  int64_t Mo = g.M, No = g.N, K = g.K;
  T *out = (T *)g.out[0];
  if constexpr (MODE == kWeightGrad) {
    // problem: (task, matrix); the sum runs over the task's rows
    const int task = prob / 3, mat = prob % 3;
    const int64_t r0 = g.rows[task], r1 = g.rows[task + 1];
    if (mat == 2) {  // [D][F] = dy^T h: the other two are [F][D]
      const int64_t s = Mo;
      Mo = No;
      No = s;
      tm = g.tiles_n;
      tn = g.tiles_m;
    }
    K = r1 - r0;
    a[0] = {(const T *)g.a[mat] + r0 * Mo, Mo, K};
    b[0] = {(const T *)g.b[mat] + r0 * No, No, K};
    out = (T *)g.out[mat] + task * g.task_stride;
  } else {
    a[0] = {(const T *)g.a[0], K, Mo};
    b[0] = BKC ? Source<T>{(const T *)g.b[0], K, No} : Source<T>{(const T *)g.b[0], No, K};
    if constexpr (MODE == kGateUp) b[1] = {(const T *)g.b[1], K, No};
    if constexpr (MODE == kInputGrad) {
      segs = 2;
      a[1] = {(const T *)g.a[1], K, Mo};
      b[1] = {(const T *)g.b[1], No, K};
    }
  }
  int im, in;
  tile_of(id, tm, tn, im, in);
  const int64_t m0 = (int64_t)im * BM, n0 = (int64_t)in * (GU ? BN / 2 : BN);

  // the steps of this workgroup: all of them, or its share of a split sum
  const int steps_seg = (int)((K + BK - 1) / BK);
  int t0 = 0, t1 = steps_seg * segs;
  if constexpr (MODE == kDown || MODE == kInputGrad) {
    if (g.splits > 1) {
      const int per = (t1 + g.splits - 1) / g.splits;
      t0 = prob * per < t1 ? prob * per : t1;
      t1 = t0 + per < t1 ? t0 + per : t1;
    }
  }

  const uint32_t lds0 = (uint32_t)(uintptr_t)(BKMOO_LDS unsigned char *)lds;
  uint32_t aoff[SA::kPer], boff[SB::kPer];
  SA::template offsets<false>(wave, lane, a[0].ld, aoff);
  SB::template offsets<GU>(wave, lane, b[0].ld, boff);

  // step t to LDS buffer `buf` (ALIGNED)
  auto load = [&](int t, int buf) {
    const int seg = MODE == kInputGrad && t >= steps_seg ? 1 : 0;
    const int64_t k0 = (int64_t)(t - seg * steps_seg) * BK;
    const Source<T> &A = seg ? a[1] : a[0];
    const Source<T> &B = seg ? b[1] : b[0];
    const int64_t ea = AKC ? m0 * A.ld + k0 : k0 * A.ld + m0;
    const int64_t eb = BKC ? n0 * B.ld + k0 : k0 * B.ld + n0;
    const i32x4 da = make_desc(A.p + ea, (A.rows * A.ld - ea) * ES);
    const i32x4 db = make_desc(B.p + eb, (B.rows * B.ld - eb) * ES);
    i32x4 db2 = db;
    if constexpr (GU) db2 = make_desc(b[1].p + eb, (b[1].rows * b[1].ld - eb) * ES);
    const uint32_t la = lds0 + buf * kStep + wave * SA::kPer * 1024;
    const uint32_t lb = lds0 + buf * kStep + SA::kBytes + wave * SB::kPer * 1024;
    const bool tail = K - k0 < BK;
#pragma unroll
    for (int i = 0; i < SA::kPer; ++i) {
      uint32_t off = aoff[i];
      if (AKC && tail) {
        int row, chunk;
        SA::place(wave * SA::kPer + i, lane, row, chunk);
        if (k0 + chunk * (16 / ES) >= K) off = kNowhere;
      }
      load_to_lds(la + i * 1024, da, off);
    }
#pragma unroll
    for (int i = 0; i < SB::kPer; ++i) {
      uint32_t off = boff[i];
      if (BKC && tail) {
        int row, chunk;
        SB::place(wave * SB::kPer + i, lane, row, chunk);
        if (k0 + chunk * (16 / ES) >= K) off = kNowhere;
      }
      load_to_lds(lb + i * 1024, GU && SB::second(wave, i) ? db2 : db, off);
    }
  };

  // the same through registers, element by element where a chunk crosses an end
  u32x4 ra[ALIGNED ? 1 : SA::kPer], rb[ALIGNED ? 1 : SB::kPer];
  auto fetch = [&](int t) {
    const int seg = MODE == kInputGrad && t >= steps_seg ? 1 : 0;
    const int64_t k0 = (int64_t)(t - seg * steps_seg) * BK;
    const Source<T> &A = seg ? a[1] : a[0];
    if constexpr (!ALIGNED) {
#pragma unroll
      for (int i = 0; i < SA::kPer; ++i) {
        int row, chunk;
        SA::place(wave * SA::kPer + i, lane, row, chunk);
        const int64_t r = (AKC ? m0 : k0) + row, c = (AKC ? k0 : m0) + chunk * (16 / ES);
        ra[i] = r < A.rows ? guarded_chunk(A.p + r * A.ld, c, A.ld) : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < SB::kPer; ++i) {
        int row, chunk;
        SB::place(wave * SB::kPer + i, lane, row, chunk);
        const Source<T> &B = (GU ? SB::second(wave, i) : seg != 0) ? b[1] : b[0];
        if (GU) row = (row >> 6) * 32 + (row & 31);
        const int64_t r = (BKC ? n0 : k0) + row, c = (BKC ? k0 : n0) + chunk * (16 / ES);
        rb[i] = r < B.rows ? guarded_chunk(B.p + r * B.ld, c, B.ld) : u32x4{0, 0, 0, 0};
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
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  const int wm = wave / WN, wn = wave % WN;
  const Reader<T, BM, AKC> reada(wm * TM * 16, lane);
  const Reader<T, BN, BKC> readb(wn * TN * 16, lane);

  if (t0 < t1) {
    if (ALIGNED) {
      load(t0, 0);
    } else {
      fetch(t0);
      put(0);
    }
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    // step t has arrived, and nobody reads the other buffer any more
    if (ALIGNED) wait_loads();
    barrier_lds();
    if (t + 1 < t1) {
      if (ALIGNED)
        load(t + 1, buf ^ 1);
      else
        fetch(t + 1);
    }
    const uint32_t la = lds0 + buf * kStep, lb = la + SA::kBytes;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      Frag<T> fa[TM], fb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j] = readb.read(lb, kk, j);
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[i] = reada.read(la, kk, i);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = multiply(fb[j], fa[i], acc[i][j]);
    }
    if (!ALIGNED && t + 1 < t1) put(buf ^ 1);
  }

  // lane: row m of piece i, four columns from n of piece j
  const int64_t mrow = m0 + wm * TM * 16 + (lane & 15);
  const int nq = 4 * (lane >> 4);
  if constexpr (MODE == kGateUp) {
    T *h = (T *)g.out[0], *su = (T *)g.out[1], *sv = (T *)g.out[2];
    const bool keep = su != nullptr;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = mrow + i * 16;
      if (m >= Mo) continue;
#pragma unroll
      for (int j = 0; j < TN / 2; ++j) {
        const int64_t n = n0 + wn * 32 + j * 16 + nq, at = m * No + n;
        const f32x4 u = acc[i][j], v = acc[i][j + TN / 2];
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = gate_act(u[e], g.act) * v[e];
        if (n + 4 <= No) {
          store4(h + at, x);
          if (keep) {
            store4(su + at, u);
            store4(sv + at, v);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < No) {
              h[at + e] = (T)x[e];
              if (keep) {
                su[at + e] = (T)u[e];
                sv[at + e] = (T)v[e];
              }
            }
        }
      }
    }
  } else if constexpr (MODE == kHiddenGrad) {
    const T *pu = (const T *)g.u, *pv = (const T *)g.v;
    T *du = (T *)g.out[0], *dv = (T *)g.out[1], *h = (T *)g.out[2];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = mrow + i * 16;
      if (m >= Mo) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int64_t n = n0 + wn * TN * 16 + j * 16 + nq, at = m * No + n;
        const f32x4 d = acc[i][j];
        f32x4 u, v, xu, xv, xh;
        if (n + 4 <= No) {
          u = load4(pu + at);
          v = load4(pv + at);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            u[e] = n + e < No ? load1(pu + at + e) : 0.0f;
            v[e] = n + e < No ? load1(pv + at + e) : 0.0f;
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float a, da;
          gate_act_grad(u[e], g.act, a, da);
          xu[e] = d[e] * v[e] * da;
          xv[e] = d[e] * a;
          xh[e] = a * v[e];
        }
        if (n + 4 <= No) {
          store4(du + at, xu);
          store4(dv + at, xv);
          store4(h + at, xh);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < No) {
              du[at + e] = (T)xu[e];
              dv[at + e] = (T)xv[e];
              h[at + e] = (T)xh[e];
            }
        }
      }
    }
  } else {
    float *part = nullptr;
    if constexpr (MODE == kDown || MODE == kInputGrad)
      if (g.splits > 1) part = g.partial + (int64_t)prob * Mo * No;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t m = mrow + i * 16;
      if (m >= Mo) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int64_t n = n0 + wn * TN * 16 + j * 16 + nq, at = m * No + n;
        const f32x4 x = acc[i][j];
        if (part) {
          if (n + 4 <= No)
            store4(part + at, x);
          else
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (n + e < No) part[at + e] = x[e];
        } else if (n + 4 <= No) {
          store4(out + at, x);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < No) out[at + e] = (T)x[e];
        }
      }
    }
  }
}

}  // namespace bkmoo
