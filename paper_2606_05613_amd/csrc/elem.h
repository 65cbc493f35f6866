// Element access of the layer operators: fp32 and bf16 in memory, fp32 in registers.
#pragma once

#include "internal.h"

namespace bkmoo {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

__device__ __forceinline__ float load1(const float *p) { return *p; }
__device__ __forceinline__ float load1(const __bf16 *p) { return (float)*p; }

// The 16 bytes of a chunk that starts at element c of a row of `n` elements (any
// alignment), zeros past the row's end: a chunk that crosses it is the row's last 16 bytes,
// moved down.
template <typename T>
__device__ __forceinline__ u32x4 guarded_chunk(const T *row, int64_t c, int64_t n) {
  constexpr int V = 16 / sizeof(T);
  union {
    u32x4 v;
    uint64_t d[2];
    uint32_t w[4];
    uint16_t h[8];
  } x;
  if (n >= V) {
    const int64_t from = c + V <= n ? c : n - V;
    x.v = *(const u32x4_any *)(row + from);
    if (from != c) {
      const int64_t over = c - from;
      const int bits = over < V ? (int)over * (int)sizeof(T) * 8 : 128;
      const uint64_t lo = x.d[0], hi = x.d[1];
      x.d[0] = bits < 64 ? (lo >> bits) | (hi << 1 << (63 - bits)) : bits < 128 ? hi >> (bits - 64) : 0;
      x.d[1] = bits < 64 ? hi >> bits : 0;
    }
    return x.v;
  }
  x.v = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (c + e < n) {
      if (sizeof(T) == 2)
        x.h[e] = ((const uint16_t *)row)[c + e];
      else
        x.w[e] = ((const uint32_t *)row)[c + e];
    }
  return x.v;
}

// Vectors of 16 bytes as fp32 and back (rounded to nearest even).
template <typename T>
struct Vec {
  static constexpr int kN = 16 / sizeof(T);
};
__device__ __forceinline__ void unpack(u32x4 v, float (&x)[4]) {
  x[0] = __uint_as_float(v.x);
  x[1] = __uint_as_float(v.y);
  x[2] = __uint_as_float(v.z);
  x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack(u32x4 v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
  return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
  union {
    bf16x8 h;
    u32x4 v;
  } u;
#pragma unroll
  for (int i = 0; i < 8; ++i) u.h[i] = (__bf16)x[i];
  return u.v;
}
// Eight consecutive elements at any alignment.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
  u32x4 a, b;
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = __uint_as_float(a[e]);
      x[e + 4] = __uint_as_float(b[e]);
    }
  }
};
template <>
struct Eight<__bf16> {
  u32x4 v;
  __device__ __forceinline__ void get(float (&x)[8]) const { unpack(v, x); }
};
__device__ __forceinline__ Eight<float> load8(const float *p) {
  return {*(const u32x4_any *)p, *(const u32x4_any *)(p + 4)};
}
__device__ __forceinline__ Eight<__bf16> load8(const __bf16 *p) { return {*(const u32x4_any *)p}; }
// The eight elements from c on of a row of n, zeros past its end.
__device__ __forceinline__ Eight<float> guarded_load8(const float *row, int64_t c, int64_t n) {
  return {guarded_chunk(row, c, n), guarded_chunk(row, c + 4, n)};
}
__device__ __forceinline__ Eight<__bf16> guarded_load8(const __bf16 *row, int64_t c, int64_t n) {
  return {guarded_chunk(row, c, n)};
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
  u32x4 a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    a[e] = __float_as_uint(x[e]);
    b[e] = __float_as_uint(x[e + 4]);
  }
  *(u32x4_any *)p = a;
  *(u32x4_any *)(p + 4) = b;
}
__device__ __forceinline__ void store8(__bf16 *p, const float (&x)[8]) { *(u32x4_any *)p = pack(x); }

// The 16 bytes at element c of a row of n elements: what lies past its end stays as it is.
template <typename T>
__device__ __forceinline__ void guarded_store(T *row, int64_t c, int64_t n, u32x4 v) {
  constexpr int V = 16 / sizeof(T);
  if (c + V <= n) {
    *(u32x4_any *)(row + c) = v;
    return;
  }
  if (c >= n) return;
  // 8, 4 and 2 bytes, as the elements left make up
  typedef uint64_t u64_any __attribute__((aligned(2)));
  typedef uint32_t u32_any __attribute__((aligned(2)));
  char *p = (char *)(row + c);
  const int bytes = (int)(n - c) * (int)sizeof(T);
  uint64_t d = (uint64_t)v.y << 32 | v.x;
  if (bytes & 8) {
    *(u64_any *)p = d;
    p += 8;
    d = (uint64_t)v.w << 32 | v.z;
  }
  if (bytes & 4) {
    *(u32_any *)p = (uint32_t)d;
    p += 4;
    d >>= 32;
  }
  if (bytes & 2) *(uint16_t *)p = (uint16_t)d;
}

}  // namespace bkmoo
