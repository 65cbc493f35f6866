// The gated feed-forward block's entry points: argument checks, workspaces and
// the choice of kernels.  The kernels are in ffn_tile.h.
#include <atomic>

#include "elem.h"
#include "ffn.h"
#include "layer_common.h"
#include "mfma.h"

namespace bkmoo {

namespace {

constexpr int64_t kMaxWidth = 1 << 20;
constexpr int kCus = 256;  // MI355X (not the device's count: the workspace's size and the sums' order hang on the plan)
constexpr int kMaxSplits = 16;

// How a product is cut: tiles of side x side, the sum over k in `splits` parts (partial sums in
// fp32, added in order by a kernel of their own).
struct Plan {
  int side, splits;
};
// bkmoo_set_ffn_tiles: 0 leaves the choice.
std::atomic<int> g_side{0}, g_splits{0}, g_workgroups{0};

// Estimated time of a product on `tiles` tiles of a CU, `steps` steps of 128 bytes along k each,
// from times on MI355X.  bf16: a step of a tile of 256 takes a CU 1.8 us; of tiles of 128 one
// 1.0 and two side by side 1.2, of 64 0.56 to 0.95 for one to four: small tiles lose to L2 and
// LDS traffic, large ones to CUs without one.  fp32 is bound by the matrix cores at every
// side.  The epilogue adds what its accesses take, the hidden gradient's the most (us at 128
// and 256: 3000 x 1024 x 3000 51 and 51, 4096 x 2048 x 6144 157 and 165, 6000 x 512 x 1500 43 and 46, 1500 x 2048 x 6144
// 84 and 90, 2000 x 1500 x 4500 76 and 68: priced so that the large side is taken from where it wins for
// certain).  (us at 64 / 128 / 256,
// M x D x F: gate and up 100 x 2048 x 6144 22 / 32 / 60, 1000 x 1024 x 3000 26 / 23 / 34, 512 x
// 4096 x 14336 240 / 153 / 115; fp32 weight gradients 777 x 500 x 1364 42 / 46 / 82.)
double product_us(int side, int dt, Mode mode, int64_t tiles, int64_t steps, bool aligned) {
  const int64_t t = (tiles + kCus - 1) / kCus;  // of the busiest CU
  static const double four[4] = {0.0, 0.56, 0.65, 0.8};
  double step;
  if (dt == F32)
    step = side == 256 ? 7.2 * t : side == 128 ? 1.9 * t : t == 1 ? 0.6 : 0.5 * t;
  else
    step = side == 256 ? 1.8 * t : side == 128 ? 1.2 * (t / 2) + 1.0 * (t % 2) : 0.95 * (t / 4) + four[t % 4];
  if (!aligned) step *= 1.5;
  const double end = mode != kHiddenGrad ? (side == 256 ? 8.0 : side == 128 ? 2.5 : 1.0)
                                         : (side == 256 ? 36.0 : side == 128 ? 7.5 : 3.0);
  return steps * step + t * end;
}

Plan plan(int dt, Mode mode, int64_t M, int64_t N, int64_t K, int64_t problems, bool aligned) {
  Plan best = {128, 1};
  double least = 0.0;
  const int64_t steps = (K * elem_bytes(dt) + 127) / 128;
  for (int side = aligned ? 256 : 128; side >= 64; side /= 2)
    for (int splits = 1; splits <= kMaxSplits && (splits == 1 || steps / splits >= 4); splits *= 2) {
      if (splits > 1 && (mode == kGateUp || mode == kWeightGrad)) break;
      const int64_t tiles = ((M + side - 1) / side) * ((N + side - 1) / side) * problems * splits;
      double us = product_us(side, dt, mode, tiles, (steps + splits - 1) / splits, aligned);
      if (splits > 1) us += 4.0 + 1.5e-6 * splits * M * N;  // written and read again, a launch
      if (least == 0.0 || us < least) {
        least = us;
        best = Plan{side, splits};
      }
    }
  const int side = g_side.load(), splits = g_splits.load();
  if (side) best.side = side == 256 && !aligned ? 128 : side;
  if (splits && mode != kGateUp && mode != kWeightGrad) best.splits = splits;
  return best;
}

// Element i of a split sum and the seven after it: the parts in order.  Those past n stay as they are.
__device__ __forceinline__ void add_parts(const float *part, int splits, int64_t n, int64_t i, float (&s)[8]) {
  if (i + 8 <= n) {
    float x[8];
    load8(part + i).get(s);
    for (int k = 1; k < splits; ++k) {
      load8(part + k * n + i).get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += x[e];
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (i + e < n) {
      s[e] = part[i + e];
      for (int k = 1; k < splits; ++k) s[e] += part[k * n + i + e];
    }
}

// Eight elements a thread, rounded once.
template <typename T>
__global__ __launch_bounds__(256) void split_sum_kernel(const float *part, int splits, int64_t n, T *out) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  float s[8];
  add_parts(part, splits, n, i, s);
  if (i + 8 <= n) {
    store8(out + i, s);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (i + e < n) out[i + e] = (T)s[e];
}

// The same for dh, and what the hidden gradient's epilogue makes of it, rounded to T as there.  (Few rows of a wide model: F / 64 tiles
// alone do not fill the chip.  The product whole / in parts with this kernel, us: 16 x 2048 x 6144 bf16 22.5 /
// 9.1 + 4.3, fp32 64 / 19.6 + 5.6; 16 x 4096 x 14336 bf16 61 / 37.5 + 4.3; 200 x 2048 x 6144 fp32 88 / 63 + 8.8.)
template <typename T>
__global__ __launch_bounds__(256) void split_hidden_kernel(const float *part, int splits, int64_t n, int act, const T *u,
                                                           const T *v, T *du, T *dv, T *h) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  const bool whole = i + 8 <= n;
  float d[8], xu[8], xv[8];
  if (whole) {
    load8(u + i).get(xu);
    load8(v + i).get(xv);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      d[e] = 0.0f;
      xu[e] = i + e < n ? load1(u + i + e) : 0.0f;
      xv[e] = i + e < n ? load1(v + i + e) : 0.0f;
    }
  }
  add_parts(part, splits, n, i, d);
  float yu[8], yv[8], yh[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float a, da;
    gate_act_grad<T>(xu[e], act, a, da);
    yu[e] = d[e] * xv[e] * da;
    yv[e] = d[e] * a;
    yh[e] = a * xv[e];
  }
  if (whole) {
    store8(du + i, yu);
    store8(dv + i, yv);
    store8(h + i, yh);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (i + e < n) {
      du[i + e] = (T)yu[e];
      dv[i + e] = (T)yv[e];
      h[i + e] = (T)yh[e];
    }
}

// What joins a split sum: the rounded result, or (kHiddenGrad) the gradients made of it.
template <typename T>
hipError_t join(Mode mode, const TileArgs &g, hipStream_t s) {
  const int64_t n = g.M * g.N;
  const unsigned grid = (unsigned)((n + 2047) / 2048);
  if (mode == kHiddenGrad)
    split_hidden_kernel<<<grid, 256, 0, s>>>(g.partial, g.splits, n, g.act, (const T *)g.u, (const T *)g.v,
                                             (T *)g.out[0], (T *)g.out[1], (T *)g.out[2]);
  else
    split_sum_kernel<<<grid, 256, 0, s>>>(g.partial, g.splits, n, (T *)g.out[0]);
  return hipGetLastError();
}

struct FfnLayout {
  size_t du, dv, h, partial, total;
};
FfnLayout ffn_layout(int64_t M, int64_t D, int64_t F, int dt, bool backward) {
  FfnLayout L;
  const bool two = !backward && dt == BF16 && M <= kFewExact;
  const size_t mf = align256((size_t)M * F * elem_bytes(dt) * (two ? 2 : 1));
  L.h = 0;
  L.du = mf;
  L.dv = L.du + (backward ? mf : 0);
  L.partial = L.dv + (backward ? mf : 0);
  size_t partial = 0;
  auto need = [&](Mode mode, int64_t N, int64_t K) {
    for (const bool aligned : {false, true}) {
      const int splits = plan(dt, mode, M, N, K, 1, aligned).splits;
      const size_t bytes = splits > 1 ? align256((size_t)splits * M * N * sizeof(float)) : 0;
      if (bytes > partial) partial = bytes;
    }
  };
  need(backward ? kInputGrad : kDown, D, backward ? 2 * F : F);
  if (backward) need(kHiddenGrad, F, D);
  L.total = L.partial + partial;
  return L;
}

bkmoo_status check_ffn(int64_t M, int64_t D, int64_t F, int dt, int act) {
  if (M < 0 || D < 1 || F < 1 || !valid_elem(dt) || (act != BKMOO_SILU && act != BKMOO_GELU)) return BKMOO_EINVAL;
  if (D > kMaxWidth || F > kMaxWidth || M > 0x7fffffff) return BKMOO_EUNSUPPORTED;
  return BKMOO_OK;
}

// A product of one matrix [M][N], the sum over K a segment (of kInputGrad's two) split where that fills the chip.
// (`room` bytes for the parts: the workspace was laid out by the same plan, unless bkmoo_set_ffn_tiles came between.)
hipError_t product(int dt, Mode mode, TileArgs g, int64_t M, int64_t N, int64_t K, float *partial, size_t room,
                   bool aligned, hipStream_t s) {
  Plan p = plan(dt, mode, M, N, mode == kInputGrad ? 2 * K : K, 1, aligned);
  if ((size_t)p.splits * M * N * sizeof(float) > room) p.splits = 1;
  g.workgroups = g_workgroups.load();
  g.M = M;
  g.N = N;
  g.K = K;
  g.splits = p.splits;
  g.partial = partial;
  const Mode kernel = mode == kHiddenGrad && g.splits > 1 ? kHiddenPart : mode;
  const hipError_t e = launch_ffn_tile(dt, kernel, g, 1, aligned, p.side, s);
  if (e != hipSuccess || g.splits == 1) return e;
  return dt == F32 ? join<float>(mode, g, s) : join<__bf16>(mode, g, s);
}

}  // namespace

hipError_t launch_ffn_tile(int dt, Mode mode, const TileArgs &g, int tasks, bool aligned, int side, hipStream_t s) {
  return dt == F32 ? launch_ffn_tile_f32(mode, g, tasks, aligned, side, s)
                   : launch_ffn_tile_bf16(mode, g, tasks, aligned, side, s);
}

}  // namespace bkmoo

using namespace bkmoo;

extern "C" bkmoo_status bkmoo_set_ffn_tiles(int32_t side, int32_t splits, int32_t workgroups) {
  if ((side != 0 && side != 64 && side != 128 && side != 256) || splits < 0 || splits > kMaxSplits || workgroups < 0)
    return BKMOO_EINVAL;
  g_side.store(side);
  g_splits.store(splits);
  g_workgroups.store(workgroups);
  return BKMOO_OK;
}

extern "C" bkmoo_status bkmoo_ffn_workspace_size(int64_t M, int64_t D, int64_t F, bkmoo_dtype dt, int32_t backward,
                                                 size_t *bytes) {
  const bkmoo_status st = check_ffn(M, D, F, dt, BKMOO_SILU);
  if (st != BKMOO_OK) return st;
  if (!bytes || (backward != 0 && backward != 1)) return BKMOO_EINVAL;
  *bytes = ffn_layout(M, D, F, dt, backward != 0).total;
  if (*bytes == 0) *bytes = 256;
  return BKMOO_OK;
}

extern "C" bkmoo_status bkmoo_ffn_forward(int64_t M, int64_t D, int64_t F, bkmoo_dtype dt, bkmoo_act act,
                                          const void *x, const void *w_gate, const void *w_up, const void *w_down,
                                          void *y, void *gate_out, void *up_out, void *workspace, size_t ws_bytes,
                                          hipStream_t stream) {
  const bkmoo_status st = check_ffn(M, D, F, dt, act);
  if (st != BKMOO_OK) return st;
  const void *all[] = {x, w_gate, w_up, w_down, y, gate_out, up_out};
  for (const void *p : all)
    if (!natural(p, dt)) return BKMOO_EINVAL;
  if (!w_gate || !w_up || !w_down || !workspace || (uintptr_t)workspace % 16 || (M > 0 && (!x || !y)) ||
      !gate_out != !up_out)
    return BKMOO_EINVAL;
  const FfnLayout L = ffn_layout(M, D, F, dt, false);
  if (ws_bytes < L.total) return BKMOO_EWORKSPACE;
  const size_t es = elem_bytes(dt), md = (size_t)M * D * es, mf = (size_t)M * F * es, df = (size_t)D * F * es;
  const Range in[] = {{x, md}, {w_gate, df}, {w_up, df}, {w_down, df}};
  const Range out[] = {{y, md}, {gate_out, mf}, {up_out, mf}, {workspace, L.total}};
  if (any_overlap(in, out)) return BKMOO_EINVAL;
  if (M == 0) return BKMOO_OK;
  char *ws = (char *)workspace;
  const bool aligned = D * es % 4 == 0 && F * es % 4 == 0 && at4(x) && at4(w_gate) && at4(w_up) && at4(w_down);
  if (M <= kFewRows)
    return status_of(launch_ffn_few(dt, x, w_gate, w_up, w_down, ws + L.h, y, gate_out, up_out, M, D, F,
                                    act == BKMOO_SILU ? kSilu : kGelu, aligned, stream));
  TileArgs g = {};
  g.a[0] = x;
  g.b[0] = w_gate;
  g.b[1] = w_up;
  g.out[0] = ws + L.h;
  g.out[1] = gate_out;
  g.out[2] = up_out;
  g.M = M;
  g.N = F;
  g.K = D;
  g.act = act == BKMOO_SILU ? kSilu : kGelu;
  g.splits = 1;
  g.workgroups = g_workgroups.load();
  hipError_t e = launch_ffn_tile(dt, kGateUp, g, 1, aligned, plan(dt, kGateUp, M, 2 * F, D, 1, aligned).side, stream);
  if (e != hipSuccess) return BKMOO_EHIP;
  TileArgs d = {};
  d.a[0] = ws + L.h;
  d.b[0] = w_down;
  d.out[0] = y;
  return status_of(product(dt, kDown, d, M, D, F, (float *)(ws + L.partial), L.total - L.partial, aligned, stream));
}

extern "C" bkmoo_status bkmoo_ffn_backward(int64_t M, int64_t D, int64_t F, bkmoo_dtype dt, bkmoo_act act, int32_t K,
                                           const int64_t *task_rows, const void *dy, const void *x,
                                           const void *gate_out, const void *up_out, const void *w_gate,
                                           const void *w_up, const void *w_down, void *dx, void *dw_gate, void *dw_up,
                                           void *dw_down, int64_t task_stride, void *workspace, size_t ws_bytes,
                                           hipStream_t stream) {
  const bkmoo_status st = check_ffn(M, D, F, dt, act);
  if (st != BKMOO_OK) return st;
  if (K < 1) return BKMOO_EINVAL;
  if (K > kMaxK) return BKMOO_EUNSUPPORTED;
  const void *all[] = {dy, x, gate_out, up_out, w_gate, w_up, w_down, dx, dw_gate, dw_up, dw_down};
  for (const void *p : all)
    if (!natural(p, dt)) return BKMOO_EINVAL;
  if (!w_gate || !w_up || !w_down || !dw_gate || !dw_up || !dw_down || !workspace || (uintptr_t)workspace % 16 ||
      (M > 0 && (!dy || !x || !gate_out || !up_out || !dx)))
    return BKMOO_EINVAL;
  if (!valid_task_rows(K, task_rows, M) || (K > 1 && task_stride < D * F)) return BKMOO_EINVAL;
  const FfnLayout L = ffn_layout(M, D, F, dt, true);
  if (ws_bytes < L.total) return BKMOO_EWORKSPACE;
  const size_t es = elem_bytes(dt), md = (size_t)M * D * es, mf = (size_t)M * F * es, df = (size_t)D * F * es;
  const Range in[] = {{dy, md}, {x, md}, {gate_out, mf}, {up_out, mf}, {w_gate, df}, {w_up, df}, {w_down, df}};
  const Range out[] = {{dx, md}, {workspace, L.total}};
  if (any_overlap(in, out)) return BKMOO_EINVAL;
  char *ws = (char *)workspace;
  void *du = ws + L.du, *dv = ws + L.dv, *h = ws + L.h;
  const bool aligned =
      D * es % 4 == 0 && F * es % 4 == 0 && at4(dy) && at4(x) && at4(w_gate) && at4(w_up) && at4(w_down);
  hipError_t e = hipSuccess;
  if (M > 0) {
    TileArgs g = {};
    g.a[0] = dy;
    g.b[0] = w_down;
    g.u = gate_out;
    g.v = up_out;
    g.out[0] = du;
    g.out[1] = dv;
    g.out[2] = h;
    g.act = act == BKMOO_SILU ? kSilu : kGelu;
    e = product(dt, kHiddenGrad, g, M, F, D, (float *)(ws + L.partial), L.total - L.partial, aligned, stream);
    if (e != hipSuccess) return BKMOO_EHIP;
    TileArgs d = {};
    d.a[0] = du;
    d.a[1] = dv;
    d.b[0] = w_gate;
    d.b[1] = w_up;
    d.out[0] = dx;
    e = product(dt, kInputGrad, d, M, D, F, (float *)(ws + L.partial), L.total - L.partial, aligned, stream);
    if (e != hipSuccess) return BKMOO_EHIP;
  }
  TileArgs w = {};
  w.a[0] = du;
  w.a[1] = dv;
  w.a[2] = dy;
  w.b[0] = x;
  w.b[1] = x;
  w.b[2] = h;
  w.out[0] = dw_gate;
  w.out[1] = dw_up;
  w.out[2] = dw_down;
  w.M = F;
  w.N = D;
  w.task_stride = task_stride;
  w.splits = 1;
  w.workgroups = g_workgroups.load();
  for (int k = 0; k <= K; ++k) w.rows[k] = task_rows[k];
  return status_of(launch_ffn_tile(dt, kWeightGrad, w, K, aligned,
                                   plan(dt, kWeightGrad, F, D, (M + K - 1) / K, 3 * K, aligned).side, stream));
}
