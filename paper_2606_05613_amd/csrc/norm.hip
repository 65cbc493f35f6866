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
// read once and each output written once; sums are fp32.  The weight gradients'
// column sums run over chunks of rows in fp32 registers (the p and g gradients
// share one), go to a workspace per chunk and are added chunk by chunk in
// order: the result does not depend on the launch.
#include "elem.h"
#include "layer_common.h"

namespace bkmoo {

namespace {

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// Sums of N values over the WAVES waves of a row; every thread gets them.
template <int WAVES, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float *lds, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
  if constexpr (WAVES > 1) {
    __syncthreads();
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

// ROWS rows a workgroup, a row on WAVES waves, VPT vectors a thread.
template <typename T, int WAVES, int VPT>
__global__ __launch_bounds__(WAVES > 4 ? 64 * WAVES : 256) void norm_forward_kernel(const NormArgs a) {
  constexpr int V = Vec<T>::kN, kRows = WAVES >= 4 ? 1 : 4 / WAVES;
  __shared__ float lds[2 * WAVES * kRows];
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % WAVES, sub = (threadIdx.x >> 6) / WAVES;
  const int64_t row = (int64_t)blockIdx.x * kRows + sub;
  if (row >= a.M) return;  // WAVES > 1 and kRows > 1 do not meet
  const int64_t D = a.D;
  const T *r = (const T *)a.r + row * D, *y = (const T *)a.y + row * D;
  const T *w = (const T *)a.w, *p = (const T *)a.p, *g = (const T *)a.g;
  u32x4 vr[VPT], vy[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
    vy[i] = vr[i] = u32x4{0, 0, 0, 0};
    if (c < D) {
      vy[i] = guarded_chunk(y, c, D);
      vr[i] = guarded_chunk(r, c, D);
    }
  }
  float inv[1] = {0.0f};
  if (p) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float x[V];
      unpack(vy[i], x);
#pragma unroll
      for (int e = 0; e < V; ++e) inv[0] += x[e] * x[e];
    }
    row_sums<WAVES>(inv, lds, wave, lane);
    inv[0] = 1.0f / sqrtf(inv[0] / (float)D + a.eps);
  }
  float rn[VPT][V], sum[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
    float x[V], k[V];
    unpack(vy[i], x);
    unpack(vr[i], rn[i]);
    if (c < D) {
      if (p) {
        unpack(guarded_chunk(p, c, D), k);
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = x[e] * inv[0] * k[e];
      }
      if (g) {
        unpack(guarded_chunk(g, c, D), k);
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] *= k[e];
      }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      rn[i][e] += a.c * x[e];
      sum[0] += rn[i][e] * rn[i][e];
    }
    if (c < D) guarded_store((T *)a.out0 + row * D, c, D, pack(rn[i]));
  }
  row_sums<WAVES>(sum, lds + WAVES * kRows, wave, lane);
  const float rho = 1.0f / sqrtf(sum[0] / (float)D + a.eps);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
    if (c >= D) continue;
    float k[V], x[V];
    unpack(guarded_chunk(w, c, D), k);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = rn[i][e] * rho * k[e];
    guarded_store((T *)a.out1 + row * D, c, D, pack(x));
  }
}

// A workgroup takes one chunk of rows of one task.
template <typename T, int WAVES, int VPT>
__global__ __launch_bounds__(64 * WAVES) void norm_backward_kernel(const NormArgs a) {
  constexpr int V = Vec<T>::kN;
  __shared__ float lds[4 * WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t D = a.D;
  int task = 0;
  while (task + 1 < a.tasks && (int)blockIdx.x >= a.chunks[task + 1]) ++task;
  const int64_t lo = a.rows[task] + (int64_t)((int)blockIdx.x - a.chunks[task]) * a.chunk_rows;
  const int64_t hi = lo + a.chunk_rows < a.rows[task + 1] ? lo + a.chunk_rows : a.rows[task + 1];
  const T *w = (const T *)a.w, *p = (const T *)a.p, *g = (const T *)a.g;
  float sw[VPT][V], ss[VPT][V];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) sw[i][e] = ss[i][e] = 0.0f;
  for (int64_t row = lo; row < hi; ++row) {
    const T *r = (const T *)a.r + row * D, *y = (const T *)a.y + row * D;
    const T *dn = (const T *)a.dn + row * D;
    const T *up = a.dup ? (const T *)a.dup + row * D : nullptr;
    u32x4 vr[VPT], vy[VPT], vn[VPT], vu[VPT];
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
      vr[i] = vy[i] = vn[i] = vu[i] = u32x4{0, 0, 0, 0};
      if (c < D) {
        vr[i] = guarded_chunk(r, c, D);
        vn[i] = guarded_chunk(dn, c, D);
        vy[i] = guarded_chunk(y, c, D);
        if (up) vu[i] = guarded_chunk(up, c, D);
      }
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
      float xr[V], xn[V], xy[V], k[V];
      unpack(vr[i], xr);
      unpack(vn[i], xn);
      unpack(vy[i], xy);
      unpack(c < D ? guarded_chunk(w, c, D) : u32x4{0, 0, 0, 0}, k);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[0] += xr[e] * xr[e];
        s[1] += xn[e] * k[e] * xr[e];
        s[2] += xy[e] * xy[e];
      }
    }
    row_sums<WAVES>(s, lds, wave, lane);
    const float rho = 1.0f / sqrtf(s[0] / (float)D + a.eps);
    const float q = rho * rho * (s[1] / (float)D);  // mean(x a) / rms, with one r' left out
    const float sig = p ? 1.0f / sqrtf(s[2] / (float)D + a.eps) : 1.0f;
    float dr[VPT][V], t[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
      float xr[V], xn[V], xy[V], k[V], kp[V], kg[V];
      unpack(vr[i], xr);
      unpack(vn[i], xn);
      unpack(vy[i], xy);
      unpack(vu[i], dr[i]);
      unpack(c < D ? guarded_chunk(w, c, D) : u32x4{0, 0, 0, 0}, k);
#pragma unroll
      for (int e = 0; e < V; ++e) kp[e] = kg[e] = 1.0f;
      if (p && c < D) unpack(guarded_chunk(p, c, D), kp);
      if (g && c < D) unpack(guarded_chunk(g, c, D), kg);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float x = xr[e] * rho;
        dr[i][e] += rho * (xn[e] * k[e] - xr[e] * q);
        sw[i][e] += xn[e] * x;
        const float d = a.c * dr[i][e];
        ss[i][e] += d * (xy[e] * sig);
        t[0] += d * kp[e] * kg[e] * xy[e];
      }
      if (c < D) guarded_store((T *)a.out0 + row * D, c, D, pack(dr[i]));
    }
    float m = 0.0f;
    if (p) {
      row_sums<WAVES>(t, lds + 3 * WAVES, wave, lane);
      m = sig * sig * sig * (t[0] / (float)D);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
      if (c >= D) continue;
      float xy[V], kp[V], kg[V], x[V];
      unpack(vy[i], xy);
#pragma unroll
      for (int e = 0; e < V; ++e) kp[e] = kg[e] = 1.0f;
      if (p) unpack(guarded_chunk(p, c, D), kp);
      if (g) unpack(guarded_chunk(g, c, D), kg);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = sig * (a.c * dr[i][e] * kp[e] * kg[e]) - xy[e] * m;
      guarded_store((T *)a.out1 + row * D, c, D, pack(x));
    }
  }
  float *part = a.partial + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t c = (int64_t)(i * WAVES * 64 + wave * 64 + lane) * V;
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (c + e < D) {
        part[c + e] = sw[i][e];
        part[D + c + e] = ss[i][e];
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

constexpr int kSumCols = 64, kSumGroups = 16;

// Column sums over a task's chunks: 16 interleaved runs of chunks side by side,
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
constexpr int kTargetChunks = 512;

int chunk_rows_for(int64_t M) {
  const int64_t n = (M + kTargetChunks - 1) / kTargetChunks;
  return (int)(n < 1 ? 1 : n);
}

template <typename T>
hipError_t forward(const NormArgs &a, hipStream_t s) {
  const int64_t nv = (a.D + Vec<T>::kN - 1) / Vec<T>::kN;
  const unsigned by4 = (unsigned)((a.M + 3) / 4), by1 = (unsigned)a.M;
  if (nv <= 64)
    norm_forward_kernel<T, 1, 1><<<by4, 256, 0, s>>>(a);
  else if (nv <= 128)
    norm_forward_kernel<T, 1, 2><<<by4, 256, 0, s>>>(a);
  else if (nv <= 256)
    norm_forward_kernel<T, 4, 1><<<by1, 256, 0, s>>>(a);
  else if (nv <= 512)
    norm_forward_kernel<T, 4, 2><<<by1, 256, 0, s>>>(a);
  else if (nv <= 1024)
    norm_forward_kernel<T, 4, 4><<<by1, 256, 0, s>>>(a);
  else if (nv <= 2048)
    norm_forward_kernel<T, 16, 2><<<by1, 1024, 0, s>>>(a);
  else
    norm_forward_kernel<T, 16, 4><<<by1, 1024, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const NormArgs &a, const NormSumArgs &sum, int chunks, hipStream_t s) {
  const int64_t nv = (a.D + Vec<T>::kN - 1) / Vec<T>::kN;
  if (chunks > 0) {
    const unsigned n = (unsigned)chunks;
    if (nv <= 64)
      norm_backward_kernel<T, 1, 1><<<n, 64, 0, s>>>(a);
    else if (nv <= 256)
      norm_backward_kernel<T, 4, 1><<<n, 256, 0, s>>>(a);
    else if (nv <= 512)
      norm_backward_kernel<T, 4, 2><<<n, 256, 0, s>>>(a);
    else if (nv <= 1024)
      norm_backward_kernel<T, 8, 2><<<n, 512, 0, s>>>(a);
    else if (nv <= 2048)
      norm_backward_kernel<T, 16, 2><<<n, 1024, 0, s>>>(a);
    else
      norm_backward_kernel<T, 16, 4><<<n, 1024, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)((a.D + kSumCols - 1) / kSumCols), (unsigned)a.tasks);
  norm_sum_kernel<T><<<grid, kSumCols * kSumGroups, 0, s>>>(sum);
  return hipGetLastError();
}

bkmoo_status check_norm(int64_t M, int64_t D, int dt, double scale, double eps) {
  if (M < 0 || D < 1 || !valid_elem(dt) || !(eps >= 0.0) || !__builtin_isfinite(eps) || !__builtin_isfinite(scale))
    return BKMOO_EINVAL;
  if (D * elem_bytes(dt) > kMaxRowBytes || M > 0x7fffffff) return BKMOO_EUNSUPPORTED;
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
  return status_of(dt == BKMOO_F32 ? forward<float>(a, stream) : forward<__bf16>(a, stream));
}

extern "C" bkmoo_status bkmoo_residual_norm_workspace_size(int64_t M, int64_t D, int32_t K, size_t *bytes) {
  if (M < 0 || D < 1 || K < 1 || !bytes) return BKMOO_EINVAL;
  if (K > kMaxK) return BKMOO_EUNSUPPORTED;
  const int rows = chunk_rows_for(M);
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
  a.chunk_rows = chunk_rows_for(M);
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
