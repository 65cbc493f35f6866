// Norms before and after a block, fused with its gate and residual scale.
//
//   forward   r' = r + c g p y / rms(y),  n = w r' / rms(r')   (rms(x)^2 = mean(x^2) + eps)
//   backward  with z = y / rms(y), x = r' / rms(r'), a = w dn:
//             dr = dR + (a - x mean(x a)) / rms(r')
//             e = c g p dr,  dy = (e - z mean(z e)) / rms(y)
//             dw = sum dn x,  dp = g s,  dg = p s,  s = sum c dr z  over a task's rows
//
// Everything is a sum over a row or a column of M x D elements that are read
// once: memory-bound.  A row stays in registers as it was read (16-byte vectors,
// at any alignment) between its statistics and its results, so each input is
// read once and each output written once; sums are fp32.  Backward passes over rows of more than 8192
// elements read a row again, out of the caches, in each of its three phases, and in part hold the column sums in scratch
// memory.  A workgroup goes
// through rows with as many waves on a row as it has vectors of 64 lanes (and several
// rows side by side where that is few), the next row's loads on their way.  The weight gradients'
// column sums run over chunks of rows in fp32 registers (the p and g gradients
// share one), go to a workspace per chunk and are added chunk by chunk in
// order: the result does not depend on the launch.
//
// Measured, bf16 with both norms and the gate: 16384 x 4096 forward 102 us (537 MB at 5.3 TB/s),
// backward 168 (806 MB at 4.8), 65536 x 1024 102 and 166; fp32 16384 x 4096 207 and 324.
// One row of 4096 2.8 us, which is a kernel's start and end, and 4.8 + 3.4.  Narrow rows lose to their
// reductions: 30000 x 300 19 (3.7 TB/s) and 63 (1.7).  Rows off 16 bytes lose a fifth forward and a third
// backward (8192 x 8191 bf16 128 and 229, x 8192 95 and 153); long ones to registers: bf16 4096 x 16384 107 (5.0
// TB/s) and 253 (3.2), x 16383 146 and 608, 2048 x 32768 252 (2.1) and 871 (0.9); fp32 4096 x 16384 194 (5.6) and
// 1035 (1.6).
#include "elem.h"
#include "layer_common.h"

namespace bkmoo {

namespace {

// Sum over a wave, in every lane: neighbours, then the halves of 16 lanes, then rows of 16.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float x) {
  x = add_dpp<0xB1>(x);   // lanes 1 0 3 2
  x = add_dpp<0x4E>(x);   // lanes 2 3 0 1
  x = add_dpp<0x141>(x);  // half rows of 16 mirrored
  x = add_dpp<0x140>(x);  // rows mirrored
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// Sums of N values over the WAVES waves of a row; every thread gets them.  One barrier:
// `lds` must not be what an earlier call used unless a barrier lies between.
template <int WAVES, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float *lds, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
  if constexpr (WAVES > 1) {
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[i * WAVES + wave] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = lds[i * WAVES];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s += lds[i * WAVES + w];
      x[i] = s;
    }
  }
}

struct NormArgs {
  const void *r, *y, *w, *p, *g;  // forward: r; backward: r' in r
  const void *dn, *dup;
  void *out0, *out1;              // forward: r', n; backward: dr, dy
  int64_t M, D;
  float c, eps;
  float *partial;                 // backward: [chunks][2][D]
  int chunk_rows, tasks;
  int chunks[kMaxK + 1];          // first chunk of each task
  int64_t rows[kMaxK + 1];
};

// How a workgroup holds rows: a row on WAVES waves with VPT vectors a thread, GROUPS rows side by
// side.
template <typename T, int WAVES, int VPT, int GROUPS>
struct Rows {
  static constexpr int V = Vec<T>::kN, kThreads = 64 * WAVES * GROUPS;
  static constexpr bool kAhead = VPT * V <= 8;  // registers for the next row's vectors
  static constexpr bool kHold = VPT * V <= 16;  // ... and for a row's at all (backward pass)
};

template <int VPT>
struct Raw {
  u32x4 v[VPT];
};
// A thread's vector i of a row; zeros past its end.  WHOLE: rows are whole vectors.
template <typename T, int WAVES, bool WHOLE>
__device__ __forceinline__ u32x4 vec_load(const T *row, int i, int at, int64_t D, bool there) {
  const int64_t c = (int64_t)(i * WAVES * 64 + at) * Vec<T>::kN;
  if (!there || c >= D) return u32x4{0, 0, 0, 0};
  return WHOLE ? *(const u32x4_any *)(row + c) : guarded_chunk(row, c, D);
}
template <typename T, int WAVES, int VPT, bool WHOLE>
__device__ __forceinline__ Raw<VPT> row_load(const T *row, int at, int64_t D, bool there) {
  Raw<VPT> x;
#pragma unroll
  for (int i = 0; i < VPT; ++i) x.v[i] = vec_load<T, WAVES, WHOLE>(row, i, at, D, there);
  return x;
}
template <typename T, int WAVES, bool WHOLE>
__device__ __forceinline__ void row_store(T *row, int i, int at, int64_t D, bool there, u32x4 v) {
  const int64_t c = (int64_t)(i * WAVES * 64 + at) * Vec<T>::kN;
  if (!there || c >= D) return;
  if constexpr (WHOLE)
    *(u32x4_any *)(row + c) = v;
  else
    guarded_store(row, c, D, v);
}
// One vector of a weight, or ones.
template <typename T>
__device__ __forceinline__ void weight_of(bool given, u32x4 v, float (&x)[Vec<T>::kN]) {
  unpack(v, x);
  if (!given)
#pragma unroll
    for (int e = 0; e < Vec<T>::kN; ++e) x[e] = 1.0f;
}

template <typename T, int WAVES, int VPT, int GROUPS, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES *GROUPS) void norm_forward_kernel(const NormArgs a) {
  using R = Rows<T, WAVES, VPT, GROUPS>;
  constexpr int V = R::V;
  __shared__ float lds[2][2][GROUPS * WAVES];
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % WAVES, grp = (threadIdx.x >> 6) / WAVES;
  const int at = wave * 64 + lane;
  const int64_t D = a.D, step = (int64_t)gridDim.x * GROUPS;
  const T *w = (const T *)a.w, *p = (const T *)a.p, *g = (const T *)a.g;
  const T *r = (const T *)a.r, *y = (const T *)a.y;
  const Raw<VPT> vw = row_load<T, WAVES, VPT, WHOLE>(w, at, D, true);
  const Raw<VPT> vp = row_load<T, WAVES, VPT, WHOLE>(p, at, D, p != nullptr);
  const Raw<VPT> vg = row_load<T, WAVES, VPT, WHOLE>(g, at, D, g != nullptr);
  int64_t row = (int64_t)blockIdx.x * GROUPS + grp;
  Raw<VPT> nr = row_load<T, WAVES, VPT, WHOLE>(r + row * D, at, D, row < a.M);
  Raw<VPT> ny = row_load<T, WAVES, VPT, WHOLE>(y + row * D, at, D, row < a.M);
  int turn = 0;
  // (every group goes round as often as the first: the barriers are the workgroup's)
  for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < a.M; first += step, row += step, turn ^= 1) {
    const bool there = row < a.M;
    const Raw<VPT> vr = nr, vy = ny;
    if constexpr (R::kAhead) {
      nr = row_load<T, WAVES, VPT, WHOLE>(r + (row + step) * D, at, D, row + step < a.M);
      ny = row_load<T, WAVES, VPT, WHOLE>(y + (row + step) * D, at, D, row + step < a.M);
    }
    float inv[1] = {1.0f};
    if (p) {
      inv[0] = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float x[V];
        unpack(vy.v[i], x);
#pragma unroll
        for (int e = 0; e < V; ++e) inv[0] += x[e] * x[e];
      }
      row_sums<WAVES>(inv, &lds[0][turn][grp * WAVES], wave, lane);
      inv[0] = 1.0f / sqrtf(inv[0] / (float)D + a.eps);
    }
    float rn[VPT][V], sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float x[V], kp[V], kg[V];
      unpack(vy.v[i], x);
      unpack(vr.v[i], rn[i]);
      weight_of<T>(p != nullptr, vp.v[i], kp);
      weight_of<T>(g != nullptr, vg.v[i], kg);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        rn[i][e] += a.c * (x[e] * inv[0] * kp[e] * kg[e]);
        sum[0] += rn[i][e] * rn[i][e];
      }
      row_store<T, WAVES, WHOLE>((T *)a.out0 + row * D, i, at, D, there, pack(rn[i]));
    }
    row_sums<WAVES>(sum, &lds[1][turn][grp * WAVES], wave, lane);
    const float rho = 1.0f / sqrtf(sum[0] / (float)D + a.eps);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float k[V], x[V];
      unpack(vw.v[i], k);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = rn[i][e] * rho * k[e];
      row_store<T, WAVES, WHOLE>((T *)a.out1 + row * D, i, at, D, there, pack(x));
    }
    if constexpr (!R::kAhead) {
      nr = row_load<T, WAVES, VPT, WHOLE>(r + (row + step) * D, at, D, row + step < a.M);
      ny = row_load<T, WAVES, VPT, WHOLE>(y + (row + step) * D, at, D, row + step < a.M);
    }
  }
}

// A workgroup takes one chunk of rows of one task.
template <typename T, int WAVES, int VPT, int GROUPS, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES *GROUPS, 2) void norm_backward_kernel(const NormArgs a) {
  using R = Rows<T, WAVES, VPT, GROUPS>;
  constexpr int V = R::V, kRow = WAVES * VPT * 64 * V;
  __shared__ float lds[2][4][GROUPS * WAVES];  // [][0] to [][2]: three sums
  __shared__ float cols[GROUPS > 1 ? 2 * kRow : 1];
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % WAVES, grp = (threadIdx.x >> 6) / WAVES;
  const int at = wave * 64 + lane;
  const int64_t D = a.D;
  int task = 0;
  while (task + 1 < a.tasks && (int)blockIdx.x >= a.chunks[task + 1]) ++task;
  const int64_t lo = a.rows[task] + (int64_t)((int)blockIdx.x - a.chunks[task]) * a.chunk_rows;
  const int64_t hi = lo + a.chunk_rows < a.rows[task + 1] ? lo + a.chunk_rows : a.rows[task + 1];
  const T *w = (const T *)a.w, *p = (const T *)a.p, *g = (const T *)a.g;
  const T *r = (const T *)a.r, *y = (const T *)a.y, *dn = (const T *)a.dn, *up = (const T *)a.dup;
  float sw[VPT][V], ss[VPT][V];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) sw[i][e] = ss[i][e] = 0.0f;
  int64_t row = lo + grp;
  // Short rows: the weights, this row and the next in registers.  Long ones: read again, from
  // the L2, in each of the three phases of a row.
  Raw<R::kHold ? VPT : 1> vw, vp, vg, vr, vn, vy, vu, nr, nn, ny, nu;
  auto ask = [&](int64_t q) {
    if constexpr (R::kHold) {
      nr = row_load<T, WAVES, VPT, WHOLE>(r + q * D, at, D, q < hi);
      nn = row_load<T, WAVES, VPT, WHOLE>(dn + q * D, at, D, q < hi);
      ny = row_load<T, WAVES, VPT, WHOLE>(y + q * D, at, D, q < hi);
      nu = row_load<T, WAVES, VPT, WHOLE>(up + q * D, at, D, up && q < hi);
    }
  };
  if constexpr (R::kHold) {
    vw = row_load<T, WAVES, VPT, WHOLE>(w, at, D, true);
    vp = row_load<T, WAVES, VPT, WHOLE>(p, at, D, p != nullptr);
    vg = row_load<T, WAVES, VPT, WHOLE>(g, at, D, g != nullptr);
  }
  ask(row);
  auto get = [&](int i, const Raw<R::kHold ? VPT : 1> &held, const T *from, bool there, float (&x)[V]) {
    if constexpr (R::kHold) {
      unpack(held.v[i], x);
    } else {
      unpack(vec_load<T, WAVES, WHOLE>(from, i, at, D, there), x);
    }
  };
  auto ones = [&](bool given, float (&x)[V]) {
    if (!given)
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = 1.0f;
  };
  int turn = 0;
  for (int64_t first = lo; first < hi; first += GROUPS, row += GROUPS, turn ^= 1) {
    const bool there = row < hi;
    vr = nr;
    vn = nn;
    vy = ny;
    vu = nu;
    const T *qr = r + row * D, *qn = dn + row * D, *qy = y + row * D, *qu = up ? up + row * D : nullptr;
    if constexpr (R::kAhead) ask(row + GROUPS);
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float xr[V], xn[V], xy[V], k[V];
      get(i, vr, qr, there, xr);
      get(i, vn, qn, there, xn);
      get(i, vy, qy, there, xy);
      get(i, vw, w, true, k);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[0] += xr[e] * xr[e];
        s[1] += xn[e] * k[e] * xr[e];
        s[2] += xy[e] * xy[e];
      }
    }
    row_sums<WAVES>(s, &lds[turn][0][grp * WAVES * 3], wave, lane);
    const float rho = 1.0f / sqrtf(s[0] / (float)D + a.eps);
    const float q = rho * rho * (s[1] / (float)D);  // mean(x a) / rms, with one r' left out
    const float sig = p ? 1.0f / sqrtf(s[2] / (float)D + a.eps) : 1.0f;
    // dr and, of it, e = c g p dr
    auto gradients = [&](int i, float (&xr)[V], float (&xn)[V], float (&dr)[V], float (&e_)[V]) {
      float k[V], kp[V], kg[V];
      get(i, vr, qr, there, xr);
      get(i, vn, qn, there, xn);
      get(i, vu, qu, there && up, dr);
      get(i, vw, w, true, k);
      get(i, vp, p, p != nullptr, kp);
      get(i, vg, g, g != nullptr, kg);
      ones(p != nullptr, kp);
      ones(g != nullptr, kg);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dr[e] += rho * (xn[e] * k[e] - xr[e] * q);
        e_[e] = a.c * dr[e] * kp[e] * kg[e];
      }
    };
    float m = 0.0f;
    if (p) {
      float t[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float xr[V], xn[V], dr[V], e_[V], xy[V];
        gradients(i, xr, xn, dr, e_);
        get(i, vy, qy, there, xy);
#pragma unroll
        for (int e = 0; e < V; ++e) t[0] += e_[e] * xy[e];
      }
      row_sums<WAVES>(t, &lds[turn][3][grp * WAVES], wave, lane);
      m = sig * sig * sig * (t[0] / (float)D);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float xr[V], xn[V], dr[V], e_[V], xy[V], x[V];
      gradients(i, xr, xn, dr, e_);
      get(i, vy, qy, there, xy);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if (there) {  // (one that is not has the statistics of zeros)
          sw[i][e] += xn[e] * (xr[e] * rho);
          ss[i][e] += a.c * dr[e] * (xy[e] * sig);
        }
        x[e] = sig * e_[e] - xy[e] * m;
      }
      row_store<T, WAVES, WHOLE>((T *)a.out0 + row * D, i, at, D, there, pack(dr));
      row_store<T, WAVES, WHOLE>((T *)a.out1 + row * D, i, at, D, there, pack(x));
    }
    if constexpr (!R::kAhead) ask(row + GROUPS);
  }
  // the groups' column sums, added in order
  if constexpr (GROUPS > 1) {
    for (int q = 0; q < GROUPS; ++q) {
      __syncthreads();
      if (grp == q)
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            float *c = cols + (i * WAVES * 64 + at) * V + e;
            c[0] = q ? c[0] + sw[i][e] : sw[i][e];
            c[kRow] = q ? c[kRow] + ss[i][e] : ss[i][e];
          }
    }
    __syncthreads();
    float *part = a.partial + (int64_t)blockIdx.x * 2 * D;
    for (int c = threadIdx.x; c < (int)D; c += R::kThreads) {
      part[c] = cols[c];
      part[D + c] = cols[kRow + c];
    }
  } else {
    float *part = a.partial + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = (int64_t)(i * WAVES * 64 + at) * V;
      if (c + V <= D) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
          *(u32x4_any *)(part + c + e) = pack(*(const float(*)[4]) & sw[i][e]);
          *(u32x4_any *)(part + D + c + e) = pack(*(const float(*)[4]) & ss[i][e]);
        }
        continue;
      }
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (c + e < D) {
          part[c + e] = sw[i][e];
          part[D + c + e] = ss[i][e];
        }
    }
  }
}

struct NormSumArgs {
  const float *partial;
  const void *p, *g;
  void *dw, *dp, *dg;
  int64_t D, task_stride;
  int chunks[kMaxK + 1];
};

constexpr int kSumCols = 16, kSumGroups = 64;

// Column sums over a task's chunks: 64 interleaved runs of chunks side by side,
// then these in order.
template <typename T>
__global__ __launch_bounds__(kSumCols *kSumGroups) void norm_sum_kernel(const NormSumArgs a) {
  __shared__ float lds[2][kSumGroups][kSumCols];
  const int col = threadIdx.x % kSumCols, grp = threadIdx.x / kSumCols, task = blockIdx.y;
  const int64_t c = (int64_t)blockIdx.x * kSumCols + col;
  float sw = 0.0f, ss = 0.0f;
  if (c < a.D)
    for (int k = a.chunks[task] + grp; k < a.chunks[task + 1]; k += kSumGroups) {
      sw += a.partial[(int64_t)k * 2 * a.D + c];
      ss += a.partial[(int64_t)k * 2 * a.D + a.D + c];
    }
  lds[0][grp][col] = sw;
  lds[1][grp][col] = ss;
  __syncthreads();
  if (grp != 0 || c >= a.D) return;
  for (int k = 1; k < kSumGroups; ++k) {
    sw += lds[0][k][col];
    ss += lds[1][k][col];
  }
  const int64_t at = task * a.task_stride + c;
  ((T *)a.dw)[at] = (T)sw;
  if (a.dp) ((T *)a.dp)[at] = (T)(a.g ? ss * load1((const T *)a.g + c) : ss);
  if (a.dg) ((T *)a.dg)[at] = (T)(a.p ? ss * load1((const T *)a.p + c) : ss);
}

constexpr int64_t kMaxRowBytes = 64 << 10;  // sixteen waves of four vectors
constexpr int64_t kMaxRows = 0x7fffffff;
// Workgroups of the backward pass (not the device's count: the workspace's size and the sums' order
// hang on it), about one of 512 threads a CU (bf16's registers leave no room
// for a second): a few more would take as long as all the others, and each writes sums of its
// own.  Of rows of 300 bf16 three of 256 threads instead take 73 us, these 59.
constexpr int kTargetChunks = 256;

int chunk_rows_for(int64_t M, int K) {
  const int64_t target = kTargetChunks - K, n = (M + target - 1) / target;
  return (int)(n < 1 ? 1 : n);
}

// A row's waves and vectors by its length: as many waves as it has vectors of 64 lanes, up to eight
// (a thread of sixteen waves has half the registers).
template <typename T, template <typename, int, int, int> class Launch, typename... Args>
hipError_t by_row(int64_t D, Args... args) {
  const int64_t nv = (D + Vec<T>::kN - 1) / Vec<T>::kN;
  if (nv <= 64) return Launch<T, 1, 1, 8>::run(args...);
  if (nv <= 128) return Launch<T, 2, 1, 4>::run(args...);
  if (nv <= 256) return Launch<T, 4, 1, 2>::run(args...);
  if (nv <= 512) return Launch<T, 8, 1, 1>::run(args...);
  if (nv <= 1024) return Launch<T, 8, 2, 1>::run(args...);
  if (nv <= 2048) return Launch<T, 8, 4, 1>::run(args...);
  return Launch<T, 16, 4, 1>::run(args...);
}
template <typename T, int WAVES, int VPT, int GROUPS>
struct Forward {
  static hipError_t run(const NormArgs &a, hipStream_t s) {
    // eight workgroups a CU go through the rows (launching one costs more than a short row)
    const int64_t n = (a.M + GROUPS - 1) / GROUPS, most = 8 * device_cu_count();
    const dim3 grid((unsigned)(n < most ? n : most)), block(64 * WAVES * GROUPS);
    if (a.D % Vec<T>::kN == 0)
      norm_forward_kernel<T, WAVES, VPT, GROUPS, true><<<grid, block, 0, s>>>(a);
    else
      norm_forward_kernel<T, WAVES, VPT, GROUPS, false><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
  }
};
template <typename T, int WAVES, int VPT, int GROUPS>
struct Backward {
  static hipError_t run(const NormArgs &a, int chunks, hipStream_t s) {
    const dim3 grid((unsigned)chunks), block(64 * WAVES * GROUPS);
    if (a.D % Vec<T>::kN == 0)
      norm_backward_kernel<T, WAVES, VPT, GROUPS, true><<<grid, block, 0, s>>>(a);
    else
      norm_backward_kernel<T, WAVES, VPT, GROUPS, false><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
  }
};

template <typename T>
hipError_t backward(const NormArgs &a, const NormSumArgs &sum, int chunks, hipStream_t s) {
  if (chunks > 0) {
    const hipError_t e = by_row<T, Backward>(a.D, a, chunks, s);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)((a.D + kSumCols - 1) / kSumCols), (unsigned)a.tasks);
  norm_sum_kernel<T><<<grid, kSumCols * kSumGroups, 0, s>>>(sum);
  return hipGetLastError();
}

bkmoo_status check_norm(int64_t M, int64_t D, int dt, double scale, double eps) {
  // (in the kernels' 32 bits: eps may be zero, but not become it)
  if (M < 0 || D < 1 || !valid_elem(dt) || !(eps >= 0.0) || !__builtin_isfinite((float)eps) ||
      (eps > 0.0 && (float)eps == 0.0f) || !__builtin_isfinite((float)scale))
    return BKMOO_EINVAL;
  if (D > kMaxRowBytes / elem_bytes(dt) || M > kMaxRows) return BKMOO_EUNSUPPORTED;
  return BKMOO_OK;
}

}  // namespace

}  // namespace bkmoo

using namespace bkmoo;

extern "C" bkmoo_status bkmoo_residual_norm_forward(int64_t M, int64_t D, bkmoo_dtype dt, const void *resid,
                                                    const void *y, const void *weight, const void *post_weight,
                                                    const void *gate, double scale, double eps, void *resid_out,
                                                    void *normed, hipStream_t stream) {
  const bkmoo_status st = check_norm(M, D, dt, scale, eps);
  if (st != BKMOO_OK) return st;
  const void *all[] = {resid, y, weight, post_weight, gate, resid_out, normed};
  for (const void *p : all)
    if (!natural(p, dt)) return BKMOO_EINVAL;
  if (!weight || (M > 0 && (!resid || !y || !resid_out || !normed))) return BKMOO_EINVAL;
  const size_t md = (size_t)M * D * elem_bytes(dt), d = (size_t)D * elem_bytes(dt);
  // r' may take r's place: a row is read before it is written
  const Range in[] = {{resid == resid_out ? nullptr : resid, md}, {y, md}, {weight, d}, {post_weight, d}, {gate, d}};
  const Range out[] = {{resid_out, md}, {normed, md}};
  if (any_overlap(in, out)) return BKMOO_EINVAL;
  if (M == 0) return BKMOO_OK;
  NormArgs a = {};
  a.r = resid;
  a.y = y;
  a.w = weight;
  a.p = post_weight;
  a.g = gate;
  a.out0 = resid_out;
  a.out1 = normed;
  a.M = M;
  a.D = D;
  a.c = (float)scale;
  a.eps = (float)eps;
  return status_of(dt == BKMOO_F32 ? by_row<float, Forward>(D, a, stream) : by_row<__bf16, Forward>(D, a, stream));
}

extern "C" bkmoo_status bkmoo_residual_norm_workspace_size(int64_t M, int64_t D, int32_t K, size_t *bytes) {
  if (M < 0 || D < 1 || K < 1 || !bytes) return BKMOO_EINVAL;
  if (K > kMaxK || M > kMaxRows || D > kMaxRowBytes / elem_bytes(BF16)) return BKMOO_EUNSUPPORTED;
  const int rows = chunk_rows_for(M, K);
  *bytes = align256((size_t)((M + rows - 1) / rows + K) * 2 * (size_t)D * sizeof(float));
  return BKMOO_OK;
}

extern "C" bkmoo_status bkmoo_residual_norm_backward(int64_t M, int64_t D, bkmoo_dtype dt, int32_t K,
                                                     const int64_t *task_rows, const void *dresid_out,
                                                     const void *dnormed, const void *resid_out, const void *y,
                                                     const void *weight, const void *post_weight, const void *gate,
                                                     double scale, double eps, void *dresid, void *dy, void *dweight,
                                                     void *dpost_weight, void *dgate, int64_t task_stride,
                                                     void *workspace, size_t ws_bytes, hipStream_t stream) {
  const bkmoo_status st = check_norm(M, D, dt, scale, eps);
  if (st != BKMOO_OK) return st;
  size_t need = 0;
  const bkmoo_status sw = bkmoo_residual_norm_workspace_size(M, D, K, &need);
  if (sw != BKMOO_OK) return sw;
  const void *all[] = {dresid_out, dnormed, resid_out, y, weight, post_weight, gate, dresid, dy, dweight, dpost_weight,
                       dgate};
  for (const void *p : all)
    if (!natural(p, dt)) return BKMOO_EINVAL;
  if (!weight || !dweight || (M > 0 && (!dnormed || !resid_out || !y || !dresid || !dy))) return BKMOO_EINVAL;
  if (!post_weight != !dpost_weight || !gate != !dgate) return BKMOO_EINVAL;
  if (!valid_task_rows(K, task_rows, M) || (K > 1 && task_stride < D)) return BKMOO_EINVAL;
  if (!workspace || (uintptr_t)workspace % 16 != 0) return BKMOO_EINVAL;
  if (ws_bytes < need) return BKMOO_EWORKSPACE;
  const size_t es = elem_bytes(dt), md = (size_t)M * D * es, d = (size_t)D * es;
  const Range in[] = {{dresid_out == dresid ? nullptr : dresid_out, md}, {dnormed, md}, {resid_out, md}, {y, md},
                      {weight, d}, {post_weight, d}, {gate, d}};
  const Range out[] = {{dresid, md}, {dy, md}, {workspace, need}};
  if (any_overlap(in, out)) return BKMOO_EINVAL;
  NormArgs a = {};
  a.r = resid_out;
  a.y = y;
  a.w = weight;
  a.p = post_weight;
  a.g = gate;
  a.dn = dnormed;
  a.dup = dresid_out;
  a.out0 = dresid;
  a.out1 = dy;
  a.M = M;
  a.D = D;
  a.c = (float)scale;
  a.eps = (float)eps;
  a.partial = (float *)workspace;
  a.chunk_rows = chunk_rows_for(M, K);
  a.tasks = K;
  NormSumArgs sum = {};
  sum.partial = a.partial;
  sum.p = post_weight;
  sum.g = gate;
  sum.dw = dweight;
  sum.dp = dpost_weight;
  sum.dg = dgate;
  sum.D = D;
  sum.task_stride = task_stride;
  int chunks = 0;
  for (int k = 0; k < K; ++k) {
    a.chunks[k] = sum.chunks[k] = chunks;
    a.rows[k] = task_rows[k];
    chunks += (int)((task_rows[k + 1] - task_rows[k] + a.chunk_rows - 1) / a.chunk_rows);
  }
  a.chunks[K] = sum.chunks[K] = chunks;
  a.rows[K] = M;
  return status_of(dt == BKMOO_F32 ? backward<float>(a, sum, chunks, stream)
                                   : backward<__bf16>(a, sum, chunks, stream));
}
