// AdamW over many tensors at once, moments in 32 bits or in 8.
//
//   g = scale * grad,  m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2
//   p' = p (1 - lr wd) - (lr / (1 - b1^t)) m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
//
// Elementwise and memory-bound: per element the gradient is read, parameter and
// moments are read and written once (bf16 gradient and parameter, fp32 copy and
// moments: 28 bytes).  The tensors' addresses travel as kernel arguments, kMaxTensors
// a launch, so that nothing is copied or kept on the device; a workgroup takes a chunk
// of one tensor.
//
// Moments in 8 bits hold m and the root q = sqrt(v) (half of v's range of exponents)
// as e4m3 values times one fp32 scale per 256 elements, counted from a
// tensor's start; 32 lanes hold a block, so its maximum is five exchanges.  They are
// rounded stochastically: between two values the upper one is taken with the
// probability that keeps the mean.  Rounding to nearest would hold v in place for good:
// with b2 = 0.999 a step changes v by a thousandth, e4m3's values are an eighth
// apart.  The random bits are a mix of the elements' numbers and the caller's seed, so a
// step can be repeated.  Eight bits a moment, one mix for two elements, resolve a 512th of
// the distance between values; a moment that a step moves by less would stay, so where
// a beta is above kFineBeta (a step moves a moment by at most a fiftieth of what it differs
// from its mean by) each element gets a mix of its own, sixteen bits a moment.  A root that is not zero
// stays so (the next step divides by it).  The parameter takes the step from the unrounded moments.
//
// Measured, 200 million elements: fp32 throughout 1067 us (5.2 TB/s), bf16 with fp32 copy and
// moments 1043 (5.4), with 8-bit moments 601-636 (5.0-5.3), these without the copy 419-445 (4.5-4.8: the random
// bits and the maxima are no longer hidden).  Sixteen bits a moment (beta2 = 0.999) cost nothing
// on top: 597 (5.4) and 439 (4.6).  168 tensors of 2048: 4.7 us in one launch.
//
// The unit is built without contraction: a moment one place off is now and then
// rounded to the other e4m3 value, so the expressions up to there round as written.
#include <math.h>

#include <algorithm>

#include "elem.h"
#include "layer_common.h"

namespace bkmoo {

namespace {

constexpr int kBlock = 256;             // elements that share a scale
constexpr int kChunk = 4096;            // elements of a workgroup
constexpr int kAdamThreads = 256;
constexpr int kLaneElems = 8;
constexpr int kMaxTensors = 192;
constexpr int64_t kMaxChunks = (1 << 24) - 1;  // a launch has fewer than 2^32 threads
constexpr int64_t kMaxElems = kMaxChunks * kChunk, kMaxTotal = (int64_t)1 << 48;  // of a tensor, of all
constexpr double kFineBeta = 0.98;
constexpr float kF8Max = 448.0f;
constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: a block below it holds zeros

struct AdamArgs {
  const void *grad;
  void *m, *v;
  float *scale_m, *scale_v, *master;
  const float *grad_scale;
  float b1, c1, b2, c2, keep, step, rootc, eps;  // c = 1 - b, keep = 1 - lr wd, step = lr / (1 - b1^t)
  uint32_t seed;
  int n;                         // tensors of this launch
  int64_t start0, block0, total; // its first element in the flat vectors and block of 256, its elements
  void *p[kMaxTensors];
  uint32_t start[kMaxTensors], block[kMaxTensors];  // of each tensor, from those on
  uint32_t chunk[kMaxTensors];   // first chunk, and whether weight decay applies (kDecay)
};
constexpr uint32_t kDecay = 0x80000000u;
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_byte __attribute__((aligned(1)));

// Eight elements from i on, of n (all of them there if ALL); zeros past the end.
template <bool ALL, typename T>
__device__ __forceinline__ void load8_of(const T *p, int64_t i, int64_t n, float (&x)[8]) {
  if (ALL || i + 8 <= n) {
    load8(p + i).get(x);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = i + e < n ? load1(p + i + e) : 0.0f;
}
template <bool ALL, typename T>
__device__ __forceinline__ void store8_of(T *p, int64_t i, int64_t n, const float (&x)[8]) {
  if (ALL || i + 8 <= n) {
    store8(p + i, x);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (i + e < n) p[i + e] = (T)x[e];
}

// Eight e4m3 values.
template <bool ALL>
__device__ __forceinline__ void load8_f8(const uint8_t *p, int64_t i, int64_t n, float (&x)[8]) {
  u32x2 w = {0, 0};
  if (ALL || i + 8 <= n) {
    w = *(const u32x2_byte *)(p + i);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e < n) w[e >> 2] |= (uint32_t)p[i + e] << (8 * (e & 3));
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
    x[4 * h] = lo[0];
    x[4 * h + 1] = lo[1];
    x[4 * h + 2] = hi[0];
    x[4 * h + 3] = hi[1];
  }
}
template <bool ALL>
__device__ __forceinline__ void store8_f8(uint8_t *p, int64_t i, int64_t n, const float (&x)[8]) {
  u32x2 w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int t = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h], x[4 * h + 1], 0, false);
    t = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2], x[4 * h + 3], t, true);
    w[h] = (uint32_t)t;
  }
  if (ALL || i + 8 <= n) {
    *(u32x2_byte *)(p + i) = w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (i + e < n) p[i + e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
}

// Maximum over the 32 lanes that hold a block: neighbours, then the halves of 16 lanes, then
// two rows of 16.
template <int CTRL>
__device__ __forceinline__ float max_dpp(float x) {
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float block_max(float x) {
  x = max_dpp<0xB1>(x);   // lanes 1 0 3 2
  x = max_dpp<0x4E>(x);   // lanes 2 3 0 1
  x = max_dpp<0x141>(x);  // half rows of 16 mirrored
  x = max_dpp<0x140>(x);  // rows mirrored
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// 32 random bits for the `number`-th element or pair of elements.
__device__ __forceinline__ uint32_t random_bits(uint32_t number, uint32_t seed) {
  constexpr uint32_t kGolden = 0x9E3779B1u;  // 2^32 over the golden ratio, odd
  uint32_t h = number * kGolden + seed;
  h = (h ^ (h >> 16)) * kGolden;
  h = (h ^ (h >> 15)) * kGolden;
  return h ^ (h >> 16);
}

// 0 <= y <= 448 (and a rounding) to one of the two e4m3 values around it: adding a random number to
// the 20 bits below e4m3's last place and cutting them off.  Below 2^-6 values are
// 2^-9 apart, as they are in [2^-6, 2^-5): shifted there and back.
__device__ __forceinline__ float round_f8(float y, uint32_t random20) {
  const float low = y < 0.015625f ? 0.015625f : 0.0f;
  const uint32_t b = (__float_as_uint(y + low) + random20) & 0xfff00000u;
  return __uint_as_float(b) - low;
}

// Eight elements of a lane, from i on.  T: parameter, G: gradient, S8: moments in 8 bits, FINE:
// sixteen random bits a moment, MASTER: a 32-bit copy takes the step, ALL: all eight are there (and,
// S8, all of the block's).
template <typename T, typename G, bool S8, bool FINE, bool MASTER, bool ALL>
__device__ __forceinline__ void step8(const AdamArgs &a, T *p, const G *grad, float *master, int64_t start,
                                      int64_t block, int64_t i, int64_t n, float gs, float keep) {
  float g[8], m[8], q[8], x[8];
  load8_of<ALL>(grad, i, n, g);
  if constexpr (MASTER)
    load8_of<ALL>(master, i, n, x);
  else
    load8_of<ALL>((const T *)p, i, n, x);
  if constexpr (S8) {
    uint8_t *m8 = (uint8_t *)a.m + start, *v8 = (uint8_t *)a.v + start;
    const int64_t blk = block + i / kBlock;
    load8_f8<ALL>(m8, i, n, m);
    load8_f8<ALL>(v8, i, n, q);
    const float om = ALL || i < n ? a.scale_m[blk] : 0.0f, oq = ALL || i < n ? a.scale_v[blk] : 0.0f;
    float tm = 0.0f, tq = 0.0f, odd = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float ge = g[e] * gs;
      m[e] = m[e] * om * a.b1 + a.c1 * ge;
      const float r = q[e] * oq;
      q[e] = sqrtf(r * r * a.b2 + a.c2 * ge * ge);
      tm = fmaxf(tm, fabsf(m[e]));
      tq = fmaxf(tq, q[e]);
      odd += m[e] + q[e];
    }
    tm = block_max(tm);
    tq = block_max(tq);
    const float im = tm >= kTiny ? 1.0f / tm * kF8Max : 0.0f, iq = tq >= kTiny ? 1.0f / tq * kF8Max : 0.0f;
    float wm[8], wq[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint32_t number = (uint32_t)blk * kBlock + ((uint32_t)i & (kBlock - 1)) + e;
      uint32_t rm[2], rr[2];
      if constexpr (FINE) {
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const uint32_t h = random_bits(number + f, a.seed);
          rm[f] = ((h & 0xffff) << 4) + 8;
          rr[f] = ((h >> 16) << 4) + 8;
        }
      } else {
        const uint32_t h = random_bits(number / 2, a.seed);
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          rm[f] = (((h >> (16 * f)) & 255) << 12) + 2048;
          rr[f] = (((h >> (16 * f + 8)) & 255) << 12) + 2048;
        }
      }
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const float xm = m[e + f] * im, xq = q[e + f] * iq;
        wm[e + f] = copysignf(round_f8(fabsf(xm), rm[f]), xm);
        wq[e + f] = fmaxf(round_f8(xq, rr[f]), xq > 0.0f ? 0.001953125f : 0.0f);
      }
    }
    // A NaN or an infinity among them (or an overflow of the sum: nothing changes then).  The maximum
    // passes over a NaN: its own values are NaN, the block's others and its scale as without it.  An
    // infinity is the maximum: the scale holds it, and zero times it is NaN for all.
    if (!(fabsf(odd) < __builtin_inff())) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xm = m[e] * im, xq = q[e] * iq;
        if (!(xm == xm)) wm[e] = xm;
        if (!(xq == xq)) wq[e] = xq;
      }
    }
    if (ALL || i < n) {
      store8_f8<ALL>(m8, i, n, wm);
      store8_f8<ALL>(v8, i, n, wq);
      if ((threadIdx.x & 31) == 0) {
        a.scale_m[blk] = tm >= kTiny ? tm * (1.0f / kF8Max) : 0.0f;
        a.scale_v[blk] = tq >= kTiny ? tq * (1.0f / kF8Max) : 0.0f;
      }
    }
  } else {
    float *m32 = (float *)a.m + start, *v32 = (float *)a.v + start;
    load8_of<ALL>(m32, i, n, m);
    load8_of<ALL>(v32, i, n, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float ge = g[e] * gs;
      m[e] = a.b1 * m[e] + a.c1 * ge;
      q[e] = a.b2 * q[e] + a.c2 * (ge * ge);
    }
    store8_of<ALL>(m32, i, n, m);
    store8_of<ALL>(v32, i, n, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = sqrtf(q[e]);
  }
  // (the reciprocal instruction is within an ulp, of a normal number, which eps sees to; the step it
  // scales is added to the parameter)
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = x[e] * keep - a.step * m[e] * __builtin_amdgcn_rcpf(q[e] * a.rootc + a.eps);
  if (ALL || i < n) {
    if constexpr (MASTER) store8_of<ALL>(master, i, n, x);
    store8_of<ALL>(p, i, n, x);
  }
}

// A workgroup: one chunk of one tensor.
template <typename T, typename G, bool S8, bool FINE, bool MASTER>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamArgs a) {
  int t = 0;
  {
    int hi = a.n;  // the chunks of t are at or before blockIdx.x, those of hi behind it
    while (hi - t > 1) {
      const int mid = (t + hi) >> 1;
      if ((a.chunk[mid] & ~kDecay) <= blockIdx.x) t = mid; else hi = mid;
    }
  }
  const int64_t first = (int64_t)(blockIdx.x - (a.chunk[t] & ~kDecay)) * kChunk;
  const int64_t start = a.start0 + a.start[t], n = (t + 1 < a.n ? (int64_t)a.start[t + 1] : a.total) - a.start[t];
  const int64_t end = first + kChunk < n ? first + kChunk : n, block = a.block0 + a.block[t];
  T *p = (T *)a.p[t];
  const G *grad = (const G *)a.grad + start;
  float *master = MASTER ? a.master + start : nullptr;
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const float keep = a.chunk[t] & kDecay ? a.keep : 1.0f;
  constexpr int kRound = kAdamThreads * kLaneElems;
  const int64_t lane = (int64_t)threadIdx.x * kLaneElems;
  int64_t base = first;
  for (; base + kRound <= end; base += kRound)
    step8<T, G, S8, FINE, MASTER, true>(a, p, grad, master, start, block, base + lane, n, gs, keep);
  if (base < end && (S8 || base + lane < n))  // (S8: a block's lanes stay together)
    step8<T, G, S8, FINE, MASTER, false>(a, p, grad, master, start, block, base + lane, n, gs, keep);
}

template <typename T, typename G, bool MASTER>
void launch_states(const AdamArgs &a, unsigned chunks, bool s8, bool fine, hipStream_t s) {
  if (!s8)
    adamw_kernel<T, G, false, false, MASTER><<<chunks, kAdamThreads, 0, s>>>(a);
  else if (fine)
    adamw_kernel<T, G, true, true, MASTER><<<chunks, kAdamThreads, 0, s>>>(a);
  else
    adamw_kernel<T, G, true, false, MASTER><<<chunks, kAdamThreads, 0, s>>>(a);
}
template <typename T, typename G>
hipError_t launch(const AdamArgs &a, int64_t chunks, bool s8, bool fine, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (a.master) {
      launch_states<T, G, true>(a, (unsigned)chunks, s8, fine, s);
      return hipGetLastError();
    }
  }
  launch_states<T, G, false>(a, (unsigned)chunks, s8, fine, s);
  return hipGetLastError();
}

int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

// Two of the tensors share a byte (they would be stepped by two workgroups at once).  Tensors in
// ascending order, as one buffer's views are, need one look each.  Else kSorted of them at a time are
// sorted, on the stack, and compared with each other and with all that come behind them: without an
// allocation, which could fail here.
bool tensors_overlap(int32_t T, const bkmoo_tensor *tensors, size_t es) {
  constexpr int kSorted = 1024;
  struct Span {
    uintptr_t lo, hi;
  };
  auto span = [&](int32_t t) {
    const uintptr_t p = (uintptr_t)tensors[t].data;
    return Span{p, p + (size_t)tensors[t].n * es};
  };
  uintptr_t end = 0;
  int32_t first = 0;
  for (; first < T; ++first) {
    if (tensors[first].n == 0) continue;
    const Span x = span(first);
    if (x.lo < end) break;
    end = x.hi;
  }
  if (first == T) return false;
  Span s[kSorted];
  for (int32_t t = 0; t < T;) {
    int n = 0;
    for (; t < T && n < kSorted; ++t)
      if (tensors[t].n > 0) s[n++] = span(t);
    if (n == 0) return false;
    std::sort(s, s + n, [](const Span &a, const Span &b) { return a.lo < b.lo; });
    for (int i = 1; i < n; ++i)
      if (s[i].lo < s[i - 1].hi) return true;
    for (int32_t q = t; q < T; ++q) {
      if (tensors[q].n == 0) continue;
      const Span x = span(q);
      // the first that starts behind x's start, and the one before it
      const int i = (int)(std::upper_bound(s, s + n, x.lo, [](uintptr_t p, const Span &a) { return p < a.lo; }) - s);
      if ((i < n && s[i].lo < x.hi) || (i > 0 && x.lo < s[i - 1].hi)) return true;
    }
  }
  return false;
}

}  // namespace

}  // namespace bkmoo

using namespace bkmoo;

extern "C" bkmoo_status bkmoo_adamw(int32_t T, const bkmoo_tensor *tensors, bkmoo_dtype dt, int64_t N,
                                    const void *grad, bkmoo_dtype grad_dt, bkmoo_state_dtype state_dt, void *moment1,
                                    void *moment2, float *scales, int64_t blocks, float *master,
                                    const bkmoo_adamw_hparams *hp, const float *grad_scale, hipStream_t stream) {
  if (T < 1 || !tensors || !hp || N < 0 || !valid_elem(dt) || !valid_elem(grad_dt)) return BKMOO_EINVAL;
  if (state_dt != BKMOO_STATE_F32 && state_dt != BKMOO_STATE_F8) return BKMOO_EINVAL;
  if (master && dt != BKMOO_BF16) return BKMOO_EINVAL;
  if (!(hp->lr >= 0.0) || !__builtin_isfinite(hp->lr) || !(hp->beta1 >= 0.0 && hp->beta1 < 1.0) ||
      !(hp->beta2 >= 0.0 && hp->beta2 < 1.0) || !(hp->eps > 0.0) || !__builtin_isfinite(hp->eps) ||
      !(hp->weight_decay >= 0.0) || !__builtin_isfinite(hp->weight_decay) || hp->step < 1)
    return BKMOO_EINVAL;
  if ((float)hp->eps < __FLT_MIN__) return BKMOO_EINVAL;  // the reciprocal instruction takes such a number for zero
  const bool s8 = state_dt == BKMOO_STATE_F8;
  int64_t total = 0, blks = 0;
  for (int t = 0; t < T; ++t) {
    const int64_t n = tensors[t].n;
    if (n < 0 || n > N - total || (n > 0 && !tensors[t].data) || !natural(tensors[t].data, dt)) return BKMOO_EINVAL;
    if (n > kMaxElems) return BKMOO_EUNSUPPORTED;
    total += n;
    blks += blocks_of(n);
  }
  if (total != N) return BKMOO_EINVAL;
  if (N > kMaxTotal) return BKMOO_EUNSUPPORTED;
  if (s8 ? blocks != blks || (N > 0 && !scales) : scales != nullptr) return BKMOO_EINVAL;
  if (N > 0 && (!grad || !moment1 || !moment2)) return BKMOO_EINVAL;
  if (!natural(grad, grad_dt) || (uintptr_t)master % 4 || (uintptr_t)scales % 4 || (uintptr_t)grad_scale % 4 ||
      (!s8 && ((uintptr_t)moment1 % 4 || (uintptr_t)moment2 % 4)))
    return BKMOO_EINVAL;
  const size_t sb = (size_t)N * (s8 ? 1 : 4);
  const Range in[] = {{grad, (size_t)N * elem_bytes(grad_dt)}, {grad_scale, sizeof(float)}};
  const Range out[] = {{moment1, sb}, {moment2, sb}, {scales, s8 ? (size_t)blks * 2 * sizeof(float) : 0},
                       {master, (size_t)N * sizeof(float)}};
  if (any_overlap(in, out)) return BKMOO_EINVAL;
  for (int t = 0; t < T; ++t) {
    const Range p[] = {{tensors[t].data, (size_t)tensors[t].n * elem_bytes(dt)}};
    if (any_overlap(p, out) || any_overlap(in, p)) return BKMOO_EINVAL;
  }
  if (tensors_overlap(T, tensors, elem_bytes(dt))) return BKMOO_EINVAL;
  AdamArgs a;
  a.grad = grad;
  a.m = moment1;
  a.v = moment2;
  a.scale_m = scales;
  a.scale_v = scales ? scales + blks : nullptr;
  a.master = master;
  a.grad_scale = grad_scale;
  a.b1 = (float)hp->beta1;
  a.c1 = (float)(1.0 - hp->beta1);
  a.b2 = (float)hp->beta2;
  a.c2 = (float)(1.0 - hp->beta2);
  a.keep = (float)(1.0 - hp->lr * hp->weight_decay);
  a.step = (float)(hp->lr / (1.0 - pow(hp->beta1, (double)hp->step)));
  a.rootc = (float)(1.0 / sqrt(1.0 - pow(hp->beta2, (double)hp->step)));
  a.eps = (float)hp->eps;
  if (!__builtin_isfinite(a.keep) || !__builtin_isfinite(a.step) || !__builtin_isfinite(a.eps)) return BKMOO_EINVAL;
  a.seed = hp->seed;
  const bool fine = hp->beta1 > kFineBeta || hp->beta2 > kFineBeta;
  int64_t at = 0, blk = 0;
  for (int t = 0; t < T;) {
    a.n = 0;
    a.start0 = at;
    a.block0 = blk;
    int64_t chunks = 0;
    for (; t < T && a.n < kMaxTensors; ++t) {
      const int64_t n = tensors[t].n, c = (n + kChunk - 1) / kChunk;
      if (n == 0) continue;
      if (a.n > 0 && (chunks + c > kMaxChunks || at + n - a.start0 > 0xffffffffll)) break;
      a.p[a.n] = tensors[t].data;
      a.start[a.n] = (uint32_t)(at - a.start0);
      a.block[a.n] = (uint32_t)(blk - a.block0);
      a.chunk[a.n] = (uint32_t)chunks | (tensors[t].decay != 0 ? kDecay : 0);
      at += n;
      blk += blocks_of(n);
      chunks += c;
      ++a.n;
    }
    if (a.n == 0) continue;
    a.total = at - a.start0;
    hipError_t e;
    if (dt == BKMOO_F32)
      e = grad_dt == BKMOO_F32 ? launch<float, float>(a, chunks, s8, fine, stream) : launch<float, __bf16>(a, chunks, s8, fine, stream);
    else
      e = grad_dt == BKMOO_F32 ? launch<__bf16, float>(a, chunks, s8, fine, stream) : launch<__bf16, __bf16>(a, chunks, s8, fine, stream);
    if (e != hipSuccess) return BKMOO_EHIP;
  }
  return BKMOO_OK;
}

extern "C" bkmoo_status bkmoo_adamw_blocks(int32_t T, const bkmoo_tensor *tensors, int64_t *blocks) {
  if (T < 1 || !tensors || !blocks) return BKMOO_EINVAL;
  int64_t n = 0;
  for (int t = 0; t < T; ++t) {
    if (tensors[t].n < 0) return BKMOO_EINVAL;
    if (tensors[t].n > kMaxElems) return BKMOO_EUNSUPPORTED;
    n += blocks_of(tensors[t].n);
  }
  *blocks = n;
  return BKMOO_OK;
}
