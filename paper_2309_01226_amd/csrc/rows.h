// Rows read and written eight elements at a time, at any alignment of their elements (the
// hardware takes 16-byte accesses at odd addresses), and sums over a wave.
#pragma once

#include "common.h"

typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef floatx4 floatx4_any __attribute__((aligned(4)));

// Eight elements as they lie in memory.
template <class T>
struct Raw8;
template <>
struct Raw8<bf16> {
  u32x4 w;
};
template <>
struct Raw8<float> {
  floatx4 w[2];
};

// STREAM: past the caches.  n: elements of the row from p on; all eight for n >= 8, none for n <= 0; what is
// behind the row reads as 0.
template <bool STREAM>
__device__ __forceinline__ Raw8<bf16> load8(const bf16* p, int n) {
  Raw8<bf16> r;
  if (n >= 8) {
    const u32x4_any* q = reinterpret_cast<const u32x4_any*>(p);
    r.w = STREAM ? __builtin_nontemporal_load(q) : *q;
    return r;
  }
  bf16 x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = e < n ? p[e] : (bf16)0.f;
  __builtin_memcpy(&r.w, x, 16);
  return r;
}
template <bool STREAM>
__device__ __forceinline__ Raw8<float> load8(const float* p, int n) {
  Raw8<float> r;
  if (n >= 8) {
    const floatx4_any* q = reinterpret_cast<const floatx4_any*>(p);
    r.w[0] = STREAM ? __builtin_nontemporal_load(q) : q[0];
    r.w[1] = STREAM ? __builtin_nontemporal_load(q + 1) : q[1];
    return r;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) r.w[e >> 2][e & 3] = e < n ? p[e] : 0.f;
  return r;
}

__device__ __forceinline__ void widen8(const Raw8<bf16>& r, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(r.w[e] << 16);
    x[2 * e + 1] = __uint_as_float(r.w[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = r.w[e >> 2][e & 3];
}

template <bool STREAM>
__device__ __forceinline__ void store8(bf16* p, int n, const float (&x)[8]) {
  bf16 y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = f2bf(x[e]);
  if (n >= 8) {
    u32x4 w;
    __builtin_memcpy(&w, y, 16);
    u32x4_any* q = reinterpret_cast<u32x4_any*>(p);
    if (STREAM) __builtin_nontemporal_store(w, q);
    else *q = w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) p[e] = y[e];
}
template <bool STREAM>
__device__ __forceinline__ void store8(float* p, int n, const float (&x)[8]) {
  if (n >= 8) {
    floatx4_any* q = reinterpret_cast<floatx4_any*>(p);
    const floatx4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
    if (STREAM) {
      __builtin_nontemporal_store(a, q);
      __builtin_nontemporal_store(b, q + 1);
    } else {
      q[0] = a;
      q[1] = b;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) p[e] = x[e];
}

// Sum over each group of L lanes (8, 16, 32 or 64) on the vector unit, in every lane: lanes 1 and 2 away, the mirror images
// in 8 and 16, then the rows of 16 and the halves.
__device__ __forceinline__ float group_total(float v, int L) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 15, 15, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 15, 15, true));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 15, 15, true));
  if (L >= 16) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 15, 15, true));
  if (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (L >= 64) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(h[0]) + __uint_as_float(h[1]);
  }
  return v;
}
__device__ __forceinline__ float wave_total(float v) { return group_total(v, 64); }
