// Loads from memory to LDS, products on the matrix cores and the gate's activation,
// shared by the feed-forward block's kernels.
#pragma once

#include "elem.h"
#include "ffn.h"

namespace bkmoo {

#define BKMOO_LDS __attribute__((address_space(3)))

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A buffer descriptor of the `bytes` (>= 0) from p on; its range ends at 2 GiB.
__device__ __forceinline__ i32x4 make_desc(const void *p, int64_t bytes) {
  const uint64_t a = (uint64_t)p;
  const uint32_t n = (uint32_t)((uint64_t)bytes >> 31) != 0 ? 0x7fffffffu : (uint32_t)bytes;
  i32x4 r;
  r.x = (int)(uint32_t)a;
  r.y = (int)((uint32_t)(a >> 32) & 0xffff);
  r.z = (int)n;
  r.w = 0x00020000;
  return r;
}

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane; beyond the descriptor's
// range zeros.  No register is written: what it leaves outstanding is waited for
// by wait_loads() alone.  (M0 holds the LDS address; nothing else here uses it.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, i32x4 d, uint32_t off) {
  const i32x4 desc = {__builtin_amdgcn_readfirstlane(d.x), __builtin_amdgcn_readfirstlane(d.y),
                      __builtin_amdgcn_readfirstlane(d.z), __builtin_amdgcn_readfirstlane(d.w)};
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(off), "s"(desc)
               : "memory");
}
// Until at most N of the wave's loads are outstanding.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Every wave's LDS reads have returned and its LDS writes are done.
__device__ __forceinline__ void barrier_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// A 16-byte chunk in LDS, loaded by this lane, of which only the first `keep` bytes belong to the
// row: the rest becomes zero.
__device__ __forceinline__ void keep_bytes(uint32_t lds, int keep) {
  BKMOO_LDS uint32_t *p = (BKMOO_LDS uint32_t *)(uintptr_t)lds;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = keep - 4 * i;
    if (b < 4) p[i] = b <= 0 ? 0 : p[i] & ((1u << (8 * b)) - 1);
  }
}
constexpr uint32_t kNowhere = 0x80000000u;  // beyond every descriptor's range

// Fragments: 16 rows (or columns) of an operand and 64 bytes of k; lane l holds 16 bytes of
// row l mod 16, from k = (l / 16) times the elements of 16 bytes on.
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

template <typename T>
__device__ __forceinline__ Frag<T> as_frag(u32x4 v) {
  return Frag<T>{__builtin_bit_cast(decltype(Frag<T>::v), v)};
}
__device__ __forceinline__ f32x4 multiply(const Frag<__bf16> &n, const Frag<__bf16> &m, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(n.v, m.v, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(const Frag<float> &n, const Frag<float> &m, f32x4 acc) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(n.v[e], m.v[e], acc, 0, 0, 0);
  return acc;
}

// Gate activation and its derivative: z s(z') with the logistic function s (GELU's tanh
// form is u times s of twice tanh's argument).  One exponential of a non-positive
// number gives s and 1 - s without cancellation.  bf16: the exponential and reciprocal
// instructions (an ulp or two of fp32) are far below the result's rounding.
template <typename T>
__device__ __forceinline__ void logistic(float z, float &s, float &r) {
  const float e = sizeof(T) == 2 ? __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(z)) : expf(-fabsf(z));
  const float p = sizeof(T) == 2 ? __builtin_amdgcn_rcpf(1.0f + e) : 1.0f / (1.0f + e);
  s = z >= 0.0f ? p : e * p;
  r = z >= 0.0f ? e * p : p;
  if (!(z == z)) s = r = z;
}
template <typename T>
__device__ __forceinline__ float gate_act(float u, int act) {
  float s, r;
  logistic<T>(act == kSilu ? u : 1.5957691216057308f * (u + 0.044715f * u * u * u), s, r);
  return u * s;
}
template <typename T>
__device__ __forceinline__ void gate_act_grad(float u, int act, float &a, float &da) {
  float z = u, dz = 1.0f, s, r;
  if (act != kSilu) {
    z = 1.5957691216057308f * (u + 0.044715f * u * u * u);
    dz = 1.5957691216057308f * (1.0f + 0.134145f * u * u);
  }
  logistic<T>(z, s, r);
  a = u * s;
  const float q = s * r;
  da = q == 0.0f ? s : s + u * q * dz;
}

}  // namespace bkmoo
