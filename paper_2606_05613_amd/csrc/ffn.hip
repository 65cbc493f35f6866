// The gated feed-forward block's entry points: argument checks, workspaces and
// the choice of kernels.  The kernels are in ffn_tile.h.
#include "elem.h"
#include "ffn.h"
#include "layer_common.h"

namespace bkmoo {

namespace {

constexpr int64_t kMaxWidth = 1 << 20;
constexpr int kCus = 256;        // MI355X
constexpr int kMaxSplits = 16;

// The parts that a product's sum over k is cut into where its tiles alone leave most
// of the chip idle: partial sums in fp32, added in order by split_sum_kernel.
int split_count(int64_t M, int64_t N, int64_t K, int dt, bool wide) {
  const int64_t side = wide ? 256 : 128, tiles = ((M + side - 1) / side) * ((N + side - 1) / side);
  const int64_t steps = (K * elem_bytes(dt) + 127) / 128;
  int64_t n = kCus / (tiles < 1 ? 1 : tiles);
  if (n > steps / 8) n = steps / 8;
  if (n > kMaxSplits) n = kMaxSplits;
  return n < 1 ? 1 : (int)n;
}

// Wide (256 x 256) tiles move half the bytes through LDS for a product, but
// leave CUs without one where there are few.
bool wide_tiles(int64_t M, int64_t N, int64_t problems) {
  return ((M + 255) / 256) * ((N + 255) / 256) * problems >= kCus;
}

__global__ __launch_bounds__(256) void split_sum_f32(const float *part, int splits, int64_t n, float *out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float s = part[i];
  for (int k = 1; k < splits; ++k) s += part[k * n + i];
  out[i] = s;
}
__global__ __launch_bounds__(256) void split_sum_bf16(const float *part, int splits, int64_t n, __bf16 *out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float s = part[i];
  for (int k = 1; k < splits; ++k) s += part[k * n + i];
  out[i] = (__bf16)s;
}

hipError_t split_sum(int dt, const float *part, int splits, int64_t n, void *out, hipStream_t s) {
  const unsigned grid = (unsigned)((n + 255) / 256);
  if (dt == F32)
    split_sum_f32<<<grid, 256, 0, s>>>(part, splits, n, (float *)out);
  else
    split_sum_bf16<<<grid, 256, 0, s>>>(part, splits, n, (__bf16 *)out);
  return hipGetLastError();
}

struct FfnLayout {
  size_t du, dv, h, partial, total;
};
FfnLayout ffn_layout(int64_t M, int64_t D, int64_t F, int dt, bool backward) {
  FfnLayout L;
  const size_t mf = align256((size_t)M * F * elem_bytes(dt));
  L.h = 0;
  L.du = mf;
  L.dv = L.du + (backward ? mf : 0);
  L.partial = L.dv + (backward ? mf : 0);
  const int a = split_count(M, D, backward ? 2 * F : F, dt, true), b = split_count(M, D, backward ? 2 * F : F, dt, false);
  const int splits = a > b ? a : b;
  L.total = L.partial + (splits > 1 ? align256((size_t)splits * M * D * sizeof(float)) : 0);
  return L;
}

bkmoo_status check_ffn(int64_t M, int64_t D, int64_t F, int dt, int act) {
  if (M < 0 || D < 1 || F < 1 || !valid_elem(dt) || (act != BKMOO_SILU && act != BKMOO_GELU)) return BKMOO_EINVAL;
  if (D > kMaxWidth || F > kMaxWidth || M > 0x7fffffff) return BKMOO_EUNSUPPORTED;
  return BKMOO_OK;
}

// y = h Wd^T or dx = du Wg + dv Wu, the sum split where that fills the chip.
hipError_t narrow_product(int dt, Mode mode, TileArgs g, int64_t M, int64_t D, int64_t F, void *out, float *partial,
                          bool aligned, hipStream_t s) {
  const bool wide = aligned && wide_tiles(M, D, 1);
  g.M = M;
  g.N = D;
  g.K = F;
  g.out[0] = out;
  g.splits = split_count(M, D, mode == kInputGrad ? 2 * F : F, dt, wide);
  g.partial = partial;
  hipError_t e = launch_ffn_tile(dt, mode, g, 1, aligned, wide, s);
  if (e == hipSuccess && g.splits > 1) e = split_sum(dt, partial, g.splits, M * D, out, s);
  return e;
}

}  // namespace

hipError_t launch_ffn_tile(int dt, Mode mode, const TileArgs &g, int tasks, bool aligned, bool wide, hipStream_t s) {
  return dt == F32 ? launch_ffn_tile_f32(mode, g, tasks, aligned, wide, s)
                   : launch_ffn_tile_bf16(mode, g, tasks, aligned, wide, s);
}

}  // namespace bkmoo

using namespace bkmoo;

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
  const int64_t v = 16 / (int64_t)es;
  const bool aligned = D % v == 0 && F % v == 0 && at16(x) && at16(w_gate) && at16(w_up) && at16(w_down);
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
  hipError_t e = launch_ffn_tile(dt, kGateUp, g, 1, aligned, aligned && wide_tiles(M, 2 * F, 1), stream);
  if (e != hipSuccess) return BKMOO_EHIP;
  TileArgs d = {};
  d.a[0] = ws + L.h;
  d.b[0] = w_down;
  return status_of(narrow_product(dt, kDown, d, M, D, F, y, (float *)(ws + L.partial), aligned, stream));
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
  const int64_t v = 16 / (int64_t)es;
  const bool aligned = D % v == 0 && F % v == 0 && at16(dy) && at16(x) && at16(w_gate) && at16(w_up) && at16(w_down);
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
    g.M = M;
    g.N = F;
    g.K = D;
    g.act = act == BKMOO_SILU ? kSilu : kGelu;
    g.splits = 1;
    e = launch_ffn_tile(dt, kHiddenGrad, g, 1, aligned, aligned && wide_tiles(M, F, 1), stream);
    if (e != hipSuccess) return BKMOO_EHIP;
    TileArgs d = {};
    d.a[0] = du;
    d.a[1] = dv;
    d.b[0] = w_gate;
    d.b[1] = w_up;
    e = narrow_product(dt, kInputGrad, d, M, D, F, dx, (float *)(ws + L.partial), aligned, stream);
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
  for (int k = 0; k <= K; ++k) w.rows[k] = task_rows[k];
  return status_of(launch_ffn_tile(dt, kWeightGrad, w, K, aligned, aligned && wide_tiles(F, D, 3 * K), stream));
}
