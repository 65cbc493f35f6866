// The feed-forward block for few rows (tokens being generated): every weight is read
// once for up to 64 tokens, so the time is the weights' bytes, and at the smallest sizes two
// kernels' start and end (about 4 us each).
//
// A workgroup computes 16 or 32 output columns (of the gate and of the up product, or of
// the result) for all tokens; its four waves split the sum over k, each on a ring of steps in
// LDS of its own that loads fill ahead: no wave waits for another before the sums meet, in
// wave order.
//
// us, gate and up / down: D=2048 F=6144, one token 9.9 / 7.8 (75 MB at 4.3 TB/s), 24 tokens
// 10.4 / 8.4; D=4096 F=14336, one 41.9 / 21.7 (352 MB at 5.5 TB/s), 24 44.9 / 27.9, 64
// 51.9 / 42.7.  fp32, both: D=2048 F=6144 1, 24 and 64 tokens 36.5, 48.0 and 79.0 (151 MB at 4.1 TB/s for one), D=4096
// F=14336 133, 154 and 250 (5.3): at 64 the matrix cores, a tenth as fast as bf16's, take more than half of it.  Loads straight into the matrix layout instead of LDS, which ask for 16
// bytes of 16 rows in turn, four times the look-ups of lines: 46.3 / 22.2 and, with 24 tokens, 58.7
// / 36.7.
#include "elem.h"
#include "ffn.h"
#include "mfma.h"

namespace bkmoo {

namespace {

constexpr float kBf16Max = 0x1.fep127f;

struct FewArgs {
  const void *x, *w0, *w1;     // [M][K]; [N][K] (w1: the up product's)
  void *out, *u, *v;           // [M][N]; u, v: may be null
  void *lo;                    // [M][F] or null: what rounding h to T leaves out, rounded to T
  int64_t M, N, K;
  int act;
};

// h is what the two kernels pass on, rounded to T: the operand type of the second product's matrix
// instructions.  Up to eight tokens of bf16 pass it on as two bf16, the second
// what rounding leaves out of the first (2^-17 of it is lost then): a token's errors come from a
// few large elements of h and do not average out.  The second product takes both as the 16 tokens
// of a tile (SPLIT), at no cost.  Where the first part's sum is not finite (an infinite weight, an
// infinity or NaN in h) it is the result: the second part's may be an infinity of the other
// sign, or NaN.

// The waves' sums, added in wave order, and what becomes of them.
template <typename T, bool PAIR, int R, int NT, int WAVES, bool SPLIT>
__device__ __forceinline__ void finish(const FewArgs &a, const f32x4 (*sums)[(PAIR ? 2 : 1) * R][NT][64], int64_t n0,
                                       int wave, int lane) {
  const int g = lane >> 4, r = lane & 15;
  // a wave for each tile of columns and tokens: lane (g, r) has columns 4 g .. + 3 of token r
  for (int p = wave; p < R * NT; p += WAVES) {
    const int c = p % R, t = p / R;
    f32x4 s[2];
#pragma unroll
    for (int i = 0; i < (PAIR ? 2 : 1); ++i) {
      s[i] = sums[0][i * R + c][t][lane];
#pragma unroll
      for (int q = 1; q < WAVES; ++q) s[i] += sums[q][i * R + c][t][lane];
      if constexpr (SPLIT) {
        f32x4 both = s[i];
#pragma unroll
        for (int q = 0; q < WAVES; ++q) both += sums[q][i * R + c][t][lane ^ 8];  // (token r + 8)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (__builtin_isfinite(s[i][e])) s[i][e] = both[e];
      }
    }
    const int64_t m = t * 16 + r, n = n0 + c * 16 + 4 * g;
    if (m >= a.M) continue;
    const int64_t at = m * a.N + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) {
        if constexpr (PAIR) {
          const float h = gate_act<T>(s[0][e], a.act) * s[1][e];
          T hi = (T)h;
          if (a.lo) {
            // (a finite h that rounds to infinity: the largest bf16, the rest in the second)
            const bool fine = __builtin_isfinite(h);
            if (fine && !__builtin_isfinite((float)hi)) hi = (T)copysignf(kBf16Max, h);
            ((T *)a.lo)[at + e] = (T)(fine ? h - (float)hi : 0.0f);
          }
          ((T *)a.out)[at + e] = hi;
          if (a.u) {
            ((T *)a.u)[at + e] = (T)s[0][e];
            ((T *)a.v)[at + e] = (T)s[1][e];
          }
        } else {
          ((T *)a.out)[at + e] = (T)s[0][e];
        }
      }
  }
}

// PAIR: both projections and the gate; else one product.  R: tiles of 16 columns, NT: tiles of 16
// tokens.  Rows that do not start at four bytes: loads straight into the matrix instruction's
// layout, at any alignment.  Lane l holds 16 bytes of weight row l mod 16, and the same bytes of
// token l mod 16.  A step of a wave is 128 bytes of every row, in two loads that take turns
// in the line (the order of k is the same for weights and tokens, and free).  U steps make a
// batch; one batch travels while the one before is multiplied.
template <typename T, bool PAIR, int R, int NT, int WAVES, int U, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, 2) void ffn_few_any_kernel(const FewArgs a) {
  constexpr int V = 16 / sizeof(T), BK = 8 * V, W = (PAIR ? 2 : 1) * R;
  __shared__ f32x4 sums[WAVES][W][NT][64];
  // (the wave's number in a scalar register: matrix instructions heed no lane mask, so what
  // depends on it must branch, not mask)
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int64_t K = a.K, n0 = (int64_t)blockIdx.x * (16 * R);
  const T *w[W], *x[NT];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const int64_t n = n0 + (i % R) * 16 + r, row = n < a.N ? n : a.N - 1;
    w[i] = (const T *)(i < R ? a.w0 : a.w1) + row * K + g * 2 * V;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t mt = SPLIT ? r & 7 : t * 16 + r, m = mt < a.M ? mt : a.M - 1;
    x[t] = (const T *)(SPLIT && r >= 8 ? a.lo : a.x) + m * K + g * 2 * V;
  }
  f32x4 acc[W][NT];
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0, 0, 0, 0};

  const int full = (int)(K / BK);  // whole steps; a last short one goes to the last wave
  const int s0 = full * wave / WAVES, s1 = full * (wave + 1) / WAVES;
  u32x4 fw[2][U][2][W], fx[2][U][2][NT];
  auto ask = [&](int set, int s) {
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (s + q < s1)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t at = (int64_t)(s + q) * BK + h * V;
#pragma unroll
          for (int i = 0; i < W; ++i) fw[set][q][h][i] = *(const u32x4_any *)(w[i] + at);
#pragma unroll
          for (int t = 0; t < NT; ++t) fx[set][q][h][t] = *(const u32x4_any *)(x[t] + at);
        }
  };
  auto products = [&](int set, int s) {
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (s + q < s1)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < W; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t)
              acc[i][t] = multiply(as_frag<T>(fw[set][q][h][i]), as_frag<T>(fx[set][q][h][t]), acc[i][t]);
  };
  ask(0, s0);
  for (int s = s0; s < s1; s += 2 * U) {
    ask(1, s + U);
    products(0, s);
    ask(0, s + 2 * U);
    products(1, s + U);
  }
  if (wave == WAVES - 1 && (int64_t)full * BK < K) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = (int64_t)full * BK + h * V, k = at + g * 2 * V, left = k < K ? K - k : 0;  // of this chunk
      Frag<T> f[W];
#pragma unroll
      for (int i = 0; i < W; ++i) f[i] = as_frag<T>(guarded_chunk(w[i] + at, (int64_t)0, left));
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const Frag<T> y = as_frag<T>(guarded_chunk(x[t] + at, (int64_t)0, left));
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i][t] = multiply(f[i], y, acc[i][t]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][i][t][lane] = acc[i][t];
  __syncthreads();
  finish<T, PAIR, R, NT, WAVES, SPLIT>(a, sums, n0, wave, lane);
}

// The same through LDS: a wave's loads cover whole lines of eight rows, into a ring of DEPTH
// steps of its own.
template <typename T, bool PAIR, int R, int NT, int WAVES, int DEPTH, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES) void ffn_few_kernel(const FewArgs a) {
  constexpr int ES = sizeof(T), V = 16 / ES, BK = 8 * V, W = (PAIR ? 2 : 1) * R;
  constexpr int kSlot = (W + NT) * 2048, kLoads = 2 * (W + NT), kSums = WAVES * W * NT * 1024;
  constexpr int kRing = WAVES * DEPTH * kSlot;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kRing > kSums ? kRing : kSums];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int64_t K = a.K, n0 = (int64_t)blockIdx.x * (16 * R);
  const int steps = (int)((K + BK - 1) / BK);
  const int s0 = steps * wave / WAVES, s1 = steps * (wave + 1) / WAVES;
  const uint32_t ring = (uint32_t)(uintptr_t)(BKMOO_LDS unsigned char *)lds + wave * DEPTH * kSlot;

  // loads: rows lane / 8 and 8 + lane / 8 of a tile, chunk c at place c ^ (row / 2 mod 8)
  const int row = lane >> 3, chunk0 = (lane & 7) ^ (row >> 1), chunk1 = (lane & 7) ^ ((row >> 1) + 4);
  const uint32_t ld = (uint32_t)(K * ES);
  const uint32_t off0 = row * ld + chunk0 * 16, off1 = (row + 8) * ld + chunk1 * 16;
  const char *pw[2] = {(const char *)a.w0 + (n0 * K + (int64_t)s0 * BK) * ES,
                       PAIR ? (const char *)a.w1 + (n0 * K + (int64_t)s0 * BK) * ES : nullptr};
  const char *px = (const char *)a.x + (int64_t)s0 * 128, *pl = SPLIT ? (const char *)a.lo + (int64_t)s0 * 128 : px;
  int64_t wbytes = ((a.N - n0) * K - (int64_t)s0 * BK) * ES, xbytes = a.M * K * ES - (int64_t)s0 * 128;
  int left = (int)K - s0 * BK, asked = s0;
  auto ask = [&](int slot) {
    const bool any = asked < s1;  // else zeros, so that every step has its loads to count
    const i32x4 d0 = make_desc(pw[0], any ? wbytes : 0), d1 = make_desc(pw[PAIR ? 1 : 0], any ? wbytes : 0);
    const i32x4 dx = make_desc(px, any ? xbytes : 0), dl = SPLIT ? make_desc(pl, any ? xbytes : 0) : dx;
    const uint32_t o0 = chunk0 * V < left ? off0 : kNowhere, o1 = chunk1 * V < left ? off1 : kNowhere;
    const uint32_t to = ring + slot * kSlot;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const uint32_t down = (i % R) * 16 * ld;
      load_to_lds(to + i * 2048, i < R ? d0 : d1, o0 + down);
      load_to_lds(to + i * 2048 + 1024, i < R ? d0 : d1, o1 + down);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      load_to_lds(to + (W + t) * 2048, dx, o0 + t * 16 * ld);
      // (SPLIT: the second eight rows are the first of the other matrix)
      load_to_lds(to + (W + t) * 2048 + 1024, dl, SPLIT && o1 != kNowhere ? o1 - 8 * ld : o1 + t * 16 * ld);
    }
    pw[0] += 128;
    pw[1] += 128;
    px += 128;
    pl += 128;
    wbytes -= 128;
    xbytes -= 128;
    left -= BK;
    ++asked;
  };
  f32x4 acc[W][NT];
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0, 0, 0, 0};
  const int place = r * 128 + 16 * (g ^ ((r >> 1) & 7));
#pragma unroll
  for (int q = 0; q < DEPTH - 1; ++q) ask(q);
  int slot = 0;
  for (int s = s0; s < s1; ++s) {
    // the step before has been read from LDS: its place is free
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    ask(slot == 0 ? DEPTH - 1 : slot - 1);
    wait_loads<(DEPTH - 1) * kLoads>();
    if (const int rest = (int)K - s * BK; rest < BK && rest % V != 0) {
      // the row ends inside a chunk: what was loaded of the next one is cleared
#pragma unroll
      for (int i = 0; i < W + NT; ++i) {
        const uint32_t at = ring + slot * kSlot + i * 2048 + lane * 16;
        const int keep0 = (rest - chunk0 * V) * ES, keep1 = (rest - chunk1 * V) * ES;
        if (keep0 > 0 && keep0 < 16) keep_bytes(at, keep0);
        if (keep1 > 0 && keep1 < 16) keep_bytes(at + 1024, keep1);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    const BKMOO_LDS char *from = (const BKMOO_LDS char *)(uintptr_t)(ring + slot * kSlot);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = place ^ (h * 64);
      Frag<T> fw[W], fx[NT];
#pragma unroll
      for (int i = 0; i < W; ++i) fw[i] = as_frag<T>(*(const BKMOO_LDS u32x4 *)(from + at + i * 2048));
#pragma unroll
      for (int t = 0; t < NT; ++t) fx[t] = as_frag<T>(*(const BKMOO_LDS u32x4 *)(from + at + (W + t) * 2048));
#pragma unroll
      for (int i = 0; i < W; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = multiply(fw[i], fx[t], acc[i][t]);
    }
    slot = slot + 1 == DEPTH ? 0 : slot + 1;
  }
  wait_loads<0>();
  __syncthreads();  // every ring is done: the sums take their place
  f32x4(*sums)[W][NT][64] = reinterpret_cast<f32x4(*)[W][NT][64]>(lds);
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][i][t][lane] = acc[i][t];
  __syncthreads();
  finish<T, PAIR, R, NT, WAVES, SPLIT>(a, sums, n0, wave, lane);
}

// Steps of the ring that fit into KB kilobytes of LDS, at most eight.
template <bool PAIR, int R, int NT, int WAVES, int KB>
constexpr int kDepth = [] {
  const int n = KB / (WAVES * ((PAIR ? 2 : 1) * R + NT) * 2);
  return n > 8 ? 8 : n;
}();

template <typename T, bool PAIR, int R, int NT, int WAVES, int KB, bool SPLIT = false>
hipError_t launch_tiles(const FewArgs &a, hipStream_t s) {
  static_assert(kDepth<PAIR, R, NT, WAVES, KB> >= 2, "a step travels while another is multiplied");
  ffn_few_kernel<T, PAIR, R, NT, WAVES, kDepth<PAIR, R, NT, WAVES, KB>, SPLIT>
      <<<dim3((unsigned)((a.N + 16 * R - 1) / (16 * R))), dim3(64 * WAVES), 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, bool PAIR, int R, int WAVES, int KB>
hipError_t launch(const FewArgs &a, hipStream_t s) {
  if constexpr (!PAIR && sizeof(T) == 2)
    if (a.lo) return launch_tiles<T, PAIR, R, 1, WAVES, KB, true>(a, s);
  // KB is what two workgroups a CU leave each.  Gate and up of 33 to 64 tokens in 16 columns a
  // workgroup would have a ring of one step there, nothing on its way during the products: 96 give
  // two, and these widths (below 4096) have at most one workgroup a CU (us, one step / two / three in
  // 160 KB: 64 x 2048 x 4032 11.0 / 8.8 / 9.3, 64 x 1024 x 3584 6.5 / 6.0 / 6.4, 64 x 512 x 1408 4.6 / 4.9 / 5.1,
  // fp32 64 x 1024 x 2048 16.1 / 13.6 / 14.0).  The result's ring has two as it is (four: 64 x 4096 x
  // 14336 42.7 / 43.0).
  if (a.M <= 16) return launch_tiles<T, PAIR, R, 1, WAVES, KB>(a, s);
  if (a.M <= 32) return launch_tiles<T, PAIR, R, 2, WAVES, KB>(a, s);
  return launch_tiles<T, PAIR, R, 4, WAVES, (PAIR && R == 1 ? 96 : KB)>(a, s);
}

template <typename T, bool PAIR, int NT, int U, bool SPLIT = false>
hipError_t launch_any_tiles(const FewArgs &a, hipStream_t s) {
  ffn_few_any_kernel<T, PAIR, 1, NT, 4, U, SPLIT><<<dim3((unsigned)((a.N + 15) / 16)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, bool PAIR>
hipError_t launch_any(const FewArgs &a, hipStream_t s) {
  if constexpr (!PAIR && sizeof(T) == 2)
    if (a.lo) return launch_any_tiles<T, PAIR, 1, 2, true>(a, s);
  return a.M <= 16   ? launch_any_tiles<T, PAIR, 1, 2>(a, s)
         : a.M <= 32 ? launch_any_tiles<T, PAIR, 2, 1>(a, s)
                     : launch_any_tiles<T, PAIR, 4, 1>(a, s);
}

// Two tiles of columns a workgroup read the tokens half as often, but make half as many
// workgroups: for more than 16 tokens where these still reach half the CUs (gate and up, us,
// one / two tiles: D=4096 F=14336, 1 token 41.6 / 41.8, 24 47.0 / 45.1, 64 64.7 / 52.6; D=2048
// F=6144, 24 13.4 / 12.4, 64 19.2 / 15.5; D=1000 F=2600, 24 5.8 / 7.4, 64 7.8 / 8.7).  The result has
// too few columns for it (24 tokens, 4096 columns: 27.8 / 36.9).
template <typename T>
hipError_t few(const FewArgs &pair, const FewArgs &down, bool aligned, hipStream_t s) {
  if (!aligned) {
    const hipError_t e = launch_any<T, true>(pair, s);
    return e == hipSuccess ? launch_any<T, false>(down, s) : e;
  }
  const hipError_t e = pair.M > 16 && pair.N >= 32 * 128 ? launch<T, true, 2, 4, 160>(pair, s)
                                                         : launch<T, true, 1, 4, 80>(pair, s);
  return e == hipSuccess ? launch<T, false, 1, 4, 80>(down, s) : e;
}

}  // namespace

hipError_t launch_ffn_few(int dt, const void *x, const void *wg, const void *wu, const void *wd, void *h, void *y,
                          void *u, void *v, int64_t M, int64_t D, int64_t F, int act, bool aligned, hipStream_t s) {
  void *lo = dt == BF16 && M <= kFewExact ? (char *)h + (size_t)M * F * elem_bytes(dt) : nullptr;
  const FewArgs pair = {x, wg, wu, h, u, v, lo, M, F, D, act};
  const FewArgs down = {h, wd, nullptr, y, nullptr, nullptr, lo, M, D, F, act};
  return dt == F32 ? few<float>(pair, down, aligned, s) : few<__bf16>(pair, down, aligned, s);
}

}  // namespace bkmoo
