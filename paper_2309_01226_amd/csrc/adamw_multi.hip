// One AdamW step over many tensors in few launches, moments in 32 or in 8 bits.
//
//   p <- p - lr wd p;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2;
//   p <- p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit moments: the 256 elements of a block share a power of two.  The root
// r = sqrt(v) is an unsigned number (1 + f / 16) 2^(e - 15), e and f of 4 bits,
// and m a sign and (1 + f / 8) 2^(e - 15), f of 3 bits; code 0 is zero.  A
// number of this kind is a float's own bits, cut off behind f and with another
// exponent bias, so coding and decoding are an addition and a shift.  Rounding:
//  * v is held as its root: half the exponent range, and the root is what the
//    update divides by.
//  * A moving average changes by (1 - b) (x - avg), for v a thousandth of it;
//    the nearest code would stay where it is for ever.  So the bits that are cut
//    off are rounded up with the probability that they stand for: the sum of bits
//    and a hash of (key of tensor and step, element) carries or does not.  The
//    mean over steps is right, and the same seed gives the same result.
//  * A root over zero never becomes zero (the update would divide by eps).
// All arithmetic is fp32; what is cut to 8 bits enters the next step only, the
// update of p takes m and v as they were formed.
//
// Bound by HBM: 30 bytes per element with 32-bit moments and an fp32 gradient (28
// without the bf16 copy), 18 with 8-bit ones, 16 with a bf16 gradient also.  A
// workgroup takes 4096 consecutive elements of one tensor, found from the launch's table
// of tensors in the kernel arguments (nothing is copied to the device, so the
// call needs no workspace and can be captured); a wave takes whole blocks, four
// consecutive elements per lane, and has the loads of all its blocks in flight first.
#include "adamw_math.h"
#include "common.h"
#include "kernels.h"

namespace {

constexpr int CHUNK = 4096;   // elements of a workgroup
constexpr int NB = 4;         // 256-element blocks of a wave
typedef uint8_t u8x4 __attribute__((ext_vector_type(4)));

// The tensor of the launch whose chunks include workgroup `wg`: every lane looks at one entry.
__device__ __forceinline__ int entry_of(const int* first, int count, int wg) {
  const int lane = threadIdx.x & 63;
  const bool at = lane < count && first[lane] <= wg;
  return __builtin_amdgcn_readfirstlane((int)__popcll(__builtin_amdgcn_ballot_w64(at)) - 1);
}

template <class V, class T>
__device__ __forceinline__ void load4(const T* p, long i, long n, bool vec, T (&x)[4]) {
  if (vec && i + 4 <= n) {
    const V v = __builtin_nontemporal_load(reinterpret_cast<const V*>(p + i));
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? p[i + e] : T(0);
  }
}
template <class V, class T>
__device__ __forceinline__ void store4(T* p, long i, long n, bool vec, const T (&x)[4]) {
  if (vec && i + 4 <= n) {
    V v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = x[e];
    __builtin_nontemporal_store(v, reinterpret_cast<V*>(p + i));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[i + e] = x[e];
  }
}

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, SAT_WAVE));
  return v;
}

// Exponent byte of a block whose largest magnitude has the bits `top`: the power of two
// under which it is at most the largest code, 2 - 2^-MANT.
template <int MANT>
__device__ __forceinline__ int block_exp(uint32_t top) {
  return min(max((int)((top + ((1u << (23 - MANT)) - 1)) >> 23), 16), 254);
}
// Code of the magnitude with bits `b` under the exponent byte `e`, rounded up by `dither`.
template <int MANT>
__device__ __forceinline__ int encode(uint32_t b, uint32_t dither, int e) {
  return (int)((b + dither) >> (23 - MANT)) - ((e - 15) << MANT);
}
template <int MANT>
__device__ __forceinline__ float decode(uint32_t code, int e) {
  return code ? __uint_as_float((code << (23 - MANT)) + ((uint32_t)(e - 15) << 23)) : 0.f;
}
__device__ __forceinline__ float decode_m(uint32_t code, int e) {
  return __uint_as_float(__float_as_uint(decode<3>(code & 127, e)) | (code >> 7) << 31);
}

template <class G>
struct Vec4;
template <>
struct Vec4<float> { using type = floatx4; };
template <>
struct Vec4<bf16> { using type = bf16x4; };

template <class G>
__global__ __launch_bounds__(256) void adamw_multi32_kernel(AdamWMulti a) {
  const int k = entry_of(a.first, a.count, blockIdx.x);
  const AdamWEntry& t = a.t[k];
  AdamWConsts c = a.c;
  c.lr_wd = t.lr_wd;
  const long n = t.n, base = (long)((int)blockIdx.x - a.first[k]) * CHUNK + 4 * threadIdx.x;
  const bool vec = t.vec;
  const G* g = (const G*)t.g;
  float* m = (float*)t.m;
  float* v = (float*)t.v;
  float pp[NB][4], mm[NB][4], vv[NB][4];
  G gg[NB][4];
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    const long i = base + u * 1024;
    load4<floatx4>((const float*)t.p, i, n, vec, pp[u]);
    load4<typename Vec4<G>::type>(g, i, n, vec, gg[u]);
    load4<floatx4>((const float*)m, i, n, vec, mm[u]);
    load4<floatx4>((const float*)v, i, n, vec, vv[u]);
  }
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    const long i = base + u * 1024;
    bf16 sh[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      adamw_one(pp[u][e], (float)gg[u][e], mm[u][e], vv[u][e], c);
      sh[e] = f2bf(pp[u][e]);
    }
    store4<floatx4>(t.p, i, n, vec, pp[u]);
    store4<floatx4>(m, i, n, vec, mm[u]);
    store4<floatx4>(v, i, n, vec, vv[u]);
    if (t.shadow != nullptr) store4<bf16x4>(t.shadow, i, n, vec, sh);
  }
}

template <class G>
__global__ __launch_bounds__(256) void adamw_multi8_kernel(AdamWMulti a) {
  const int k = entry_of(a.first, a.count, blockIdx.x);
  const AdamWEntry& t = a.t[k];
  AdamWConsts c = a.c;
  c.lr_wd = t.lr_wd;
  const int lane = threadIdx.x & 63;
  const long n = t.n;
  const long b0 = (long)((int)blockIdx.x - a.first[k]) * (CHUNK / 256) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * NB;
  const bool vec = t.vec;
  const G* g = (const G*)t.g;
  uint8_t* m = (uint8_t*)t.m;
  uint8_t* v = (uint8_t*)t.v;
  float pp[NB][4];
  G gg[NB][4];
  uint8_t mc[NB][4], vc[NB][4];
  int me[NB], ve[NB];
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    const long i = (b0 + u) * 256 + 4 * lane;
    load4<floatx4>((const float*)t.p, i, n, vec, pp[u]);
    load4<typename Vec4<G>::type>(g, i, n, vec, gg[u]);
    load4<u8x4>((const uint8_t*)m, i, n, vec, mc[u]);
    load4<u8x4>((const uint8_t*)v, i, n, vec, vc[u]);
    const bool live = (b0 + u) * 256 < n;
    me[u] = live ? t.m_exp[b0 + u] : 0;
    ve[u] = live ? t.v_exp[b0 + u] : 0;
  }
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    if ((b0 + u) * 256 >= n) break;
    const long i = (b0 + u) * 256 + 4 * lane;
    float mm[4], rr[4];
    bf16 sh[4];
    uint32_t mtop = 0, rtop = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
      mm[e] = decode_m(mc[u][e], me[u]);
      const float r = decode<4>(vc[u][e], ve[u]);
      float vv = r * r;
      adamw_one(pp[u][e], (float)gg[u][e], mm[e], vv, c);
      rr[e] = sqrtf(vv);
      sh[e] = f2bf(pp[u][e]);
      mtop = max(mtop, __float_as_uint(mm[e]) & 0x7FFFFFFFu);
      rtop = max(rtop, __float_as_uint(rr[e]));
    }
    store4<floatx4>(t.p, i, n, vec, pp[u]);
    if (t.shadow != nullptr) store4<bf16x4>(t.shadow, i, n, vec, sh);
    const int em = block_exp<3>(wave_umax(mtop)), er = block_exp<4>(wave_umax(rtop));
    const uint32_t h0 = ((uint32_t)i + t.key) * 0x9E3779B1u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t h = h0 + e * 0x9E3779B1u;
      h = (h ^ h >> 15) * 0x85EBCA6Bu;
      h ^= h >> 13;
      const uint32_t mb = __float_as_uint(mm[e]), rb = __float_as_uint(rr[e]);
      const int qm = min(max(encode<3>(mb & 0x7FFFFFFFu, h & 0xFFFFFu, em), 0), 127);
      const int qr = min(max(encode<4>(rb, h >> 13, er), 1), 255);
      mc[u][e] = (uint8_t)(qm | (int)(mb >> 31) << 7);
      vc[u][e] = (uint8_t)(rr[e] > 0.f ? qr : 0);
    }
    store4<u8x4>(m, i, n, vec, mc[u]);
    store4<u8x4>(v, i, n, vec, vc[u]);
    if (lane == 0) {
      t.m_exp[b0 + u] = (uint8_t)em;
      t.v_exp[b0 + u] = (uint8_t)er;
    }
  }
}

// The values that 8-bit moments stand for: m and v = r^2 (both exact in fp32; m also in bf16).
template <class O>
__global__ __launch_bounds__(256) void adamw_state_kernel(AdamWMulti a) {
  const int k = entry_of(a.first, a.count, blockIdx.x);
  const AdamWEntry& t = a.t[k];
  const int lane = threadIdx.x & 63;
  const long n = t.n;
  const long b0 = (long)((int)blockIdx.x - a.first[k]) * (CHUNK / 256) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * NB;
  const bool vec = t.vec;
  uint8_t mc[NB][4], vc[NB][4];
  int me[NB], ve[NB];
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    const long i = (b0 + u) * 256 + 4 * lane;
    load4<u8x4>((const uint8_t*)t.m, i, n, vec, mc[u]);
    load4<u8x4>((const uint8_t*)t.v, i, n, vec, vc[u]);
    const bool live = (b0 + u) * 256 < n;
    me[u] = live ? t.m_exp[b0 + u] : 0;
    ve[u] = live ? t.v_exp[b0 + u] : 0;
  }
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    const long i = (b0 + u) * 256 + 4 * lane;
    O mo[4], vo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float r = decode<4>(vc[u][e], ve[u]);
      mo[e] = (O)decode_m(mc[u][e], me[u]);
      vo[e] = (O)(r * r);
    }
    store4<typename Vec4<O>::type>((O*)t.m_out, i, n, vec, mo);
    store4<typename Vec4<O>::type>((O*)t.v_out, i, n, vec, vo);
  }
}

}  // namespace

long adamw_chunks(long n) { return (n + CHUNK - 1) / CHUNK; }

hipError_t launch_adamw_multi(const AdamWMulti& a, int chunks, int bits, bool grad_bf16, hipStream_t s) {
  const dim3 grid((unsigned)chunks), block(256);
  if (bits == 32 && grad_bf16) hipLaunchKernelGGL(adamw_multi32_kernel<bf16>, grid, block, 0, s, a);
  else if (bits == 32) hipLaunchKernelGGL(adamw_multi32_kernel<float>, grid, block, 0, s, a);
  else if (grad_bf16) hipLaunchKernelGGL(adamw_multi8_kernel<bf16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(adamw_multi8_kernel<float>, grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_adamw_state(const AdamWMulti& a, int chunks, bool out_bf16, hipStream_t s) {
  const dim3 grid((unsigned)chunks), block(256);
  if (out_bf16) hipLaunchKernelGGL(adamw_state_kernel<bf16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(adamw_state_kernel<float>, grid, block, 0, s, a);
  return hipGetLastError();
}
