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
// update of p takes m and v as they were formed.  The 8-bit step takes the hardware's
// root and reciprocal, 1 ulp off each and 0 for a v below 2^-126 (p stays within 16 ulp of the step's
// terms); the 32-bit one is the single tensor's arithmetic, bit for bit.
//
// Bound by HBM: 30 bytes per element with 32-bit moments and an fp32 gradient (28
// without the bf16 copy), 18 with 8-bit ones, 16 with a bf16 gradient also.  A
// workgroup takes consecutive elements of one tensor, found from the launch's table of tensors in the
// kernel arguments (nothing is copied to the device, so the call needs no workspace and can be
// captured); a wave takes whole blocks, four consecutive elements per lane, and has the loads of all its blocks
// in flight first.  4096 elements a workgroup; 1024 where the whole table would give 256 CUs fewer than four
// workgroups each: 0.17 M elements 9.0 -> 4.2 us, large tables the same within 1 %.  Such a table (up to 126 MB)
// stays in the last-level cache from step to step, a larger one goes past the caches: 2 M elements 8.1 us, past them
// 10.5; 4 M 19.8 and 21.3; 160 M with 32-bit moments 883 us through the caches, 799 past them.  Whole aligned runs take a
// straight-line path (8 bits: 1891 -> 1197 us), the others go element by element.
// 160 M values with 32-bit moments: 4.80 GB in 809 us, 5.9 TB/s; 444 M with 8-bit ones: 7.1 GB in 1199 us, 5.9;
// reading their values back as bf16, 6 bytes each: 513 us, 5.2 (another card: 752, 1102 and 471 us).  A copy of 4 GiB
// moves 4.8 TB/s, torch's product in place 5.9, its fill 6.8.
#include "adamw_math.h"
#include "common.h"
#include "kernels.h"

namespace {

typedef uint8_t u8x4 __attribute__((ext_vector_type(4)));
typedef uint8_t u8x8 __attribute__((ext_vector_type(8)));

// The tensor of the launch whose chunks include workgroup `wg`: every lane looks at one entry.
__device__ __forceinline__ int entry_of(const int* first, int count, int wg) {
  const int lane = threadIdx.x & 63;
  const bool at = lane < count && first[lane] <= wg;
  return __builtin_amdgcn_readfirstlane((int)__popcll(__builtin_amdgcn_ballot_w64(at)) - 1);
}

// N elements from i on.  FULL: all below n and aligned; otherwise one by one.  STREAM: past the caches.
template <bool FULL, class V, bool STREAM, class T, int N>
__device__ __forceinline__ void load(const T* p, long i, long n, T (&x)[N]) {
  if constexpr (FULL) {
    const V* q = reinterpret_cast<const V*>(p + i);
    const V v = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = v[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = i + e < n ? p[i + e] : T(0);
  }
}
template <bool FULL, class V, bool STREAM, class T, int N>
__device__ __forceinline__ void store(T* p, long i, long n, const T (&x)[N]) {
  if constexpr (FULL) {
    V v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = x[e];
    V* q = reinterpret_cast<V*>(p + i);
    if (STREAM) __builtin_nontemporal_store(v, q);
    else *q = v;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (i + e < n) p[i + e] = x[e];
  }
}

// Maximum over the wave, on the vector unit: lanes 1 and 2 away, 4 and 8 around the row of 16, then
// the rows and halves.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 15, 15, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 15, 15, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 15, 15, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 15, 15, true));
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(r[0], r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(h[0], h[1]);
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
// Of 16 bytes of values, and their codes.
template <class O>
struct Store;
template <>
struct Store<float> { using type = floatx4; using codes = u8x4; };
template <>
struct Store<bf16> { using type = bf16x8; using codes = u8x8; };

// A wave's NB runs of 256 elements from `b0` (in runs) on.
template <class G, int NB, bool FULL>
__device__ __forceinline__ void step32(const AdamWEntry& t, const AdamWConsts& c, long b0) {
  constexpr bool STREAM = NB > 1;
  using GV = typename Vec4<G>::type;
  const long n = t.n, i0 = b0 * 256 + 4 * (threadIdx.x & 63);
  float* m = (float*)t.m;
  float* v = (float*)t.v;
  float pp[NB][4], mm[NB][4], vv[NB][4];
  G gg[NB][4];
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    load<FULL, floatx4, STREAM>((const float*)t.p, i0 + u * 256, n, pp[u]);
    load<FULL, GV, STREAM>((const G*)t.g, i0 + u * 256, n, gg[u]);
    load<FULL, floatx4, STREAM>((const float*)m, i0 + u * 256, n, mm[u]);
    load<FULL, floatx4, STREAM>((const float*)v, i0 + u * 256, n, vv[u]);
  }
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    const long i = i0 + u * 256;
    bf16 sh[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      adamw_one(pp[u][e], (float)gg[u][e], mm[u][e], vv[u][e], c);
      sh[e] = f2bf(pp[u][e]);
    }
    store<FULL, floatx4, STREAM>(t.p, i, n, pp[u]);
    store<FULL, floatx4, STREAM>(m, i, n, mm[u]);
    store<FULL, floatx4, STREAM>(v, i, n, vv[u]);
    if (t.shadow != nullptr) store<FULL, bf16x4, STREAM>(t.shadow, i, n, sh);
  }
}

// A wave's NB blocks from b0 on.
template <class G, int NB, bool FULL>
__device__ __forceinline__ void step8(const AdamWEntry& t, const AdamWConsts& c, long b0) {
  constexpr bool STREAM = NB > 1;
  using GV = typename Vec4<G>::type;
  const int lane = threadIdx.x & 63;
  const long n = t.n, i0 = b0 * 256 + 4 * lane;
  uint8_t* m = (uint8_t*)t.m;
  uint8_t* v = (uint8_t*)t.v;
  const float ibc = 1.f / c.bc2s;
  float pp[NB][4];
  G gg[NB][4];
  uint8_t mc[NB][4], vc[NB][4];
  int me[NB], ve[NB];
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    const bool live = FULL || (b0 + u) * 256 < n;
    me[u] = live ? t.m_exp[b0 + u] : 0;
    ve[u] = live ? t.v_exp[b0 + u] : 0;
    load<FULL, u8x4, STREAM>((const uint8_t*)m, i0 + u * 256, n, mc[u]);
    load<FULL, u8x4, STREAM>((const uint8_t*)v, i0 + u * 256, n, vc[u]);
    load<FULL, GV, STREAM>((const G*)t.g, i0 + u * 256, n, gg[u]);
    load<FULL, floatx4, STREAM>((const float*)t.p, i0 + u * 256, n, pp[u]);
  }
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    if (!FULL && (b0 + u) * 256 >= n) break;
    const long i = i0 + u * 256;
    float mm[4], rr[4];
    bf16 sh[4];
    uint32_t mtop = 0, rtop = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
      const float g = (float)gg[u][e];
      const float r = decode<4>(vc[u][e], ve[u]);
      mm[e] = c.b1 * decode_m(mc[u][e], me[u]) + c.omb1 * g;
      rr[e] = __builtin_amdgcn_sqrtf(c.b2 * (r * r) + c.omb2 * g * g);
      float p = pp[u][e];
      p = p - c.lr_wd * p;
      p = p - c.step * mm[e] * __builtin_amdgcn_rcpf(rr[e] * ibc + c.eps);
      pp[u][e] = p;
      sh[e] = f2bf(p);
      mtop = max(mtop, __float_as_uint(mm[e]) & 0x7FFFFFFFu);
      rtop = max(rtop, __float_as_uint(rr[e]));
    }
    store<FULL, floatx4, STREAM>(t.p, i, n, pp[u]);
    if (t.shadow != nullptr) store<FULL, bf16x4, STREAM>(t.shadow, i, n, sh);
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
    store<FULL, u8x4, STREAM>(m, i, n, mc[u]);
    store<FULL, u8x4, STREAM>(v, i, n, vc[u]);
    if (lane == 0) {
      t.m_exp[b0 + u] = (uint8_t)em;
      t.v_exp[b0 + u] = (uint8_t)er;
    }
  }
}

template <class G, int BITS, int NB>
__global__ __launch_bounds__(256) void adamw_multi_kernel(AdamWMulti a) {
  const int k = entry_of(a.first, a.count, blockIdx.x);
  const AdamWEntry& t = a.t[k];
  AdamWConsts c = a.c;
  c.lr_wd = t.lr_wd;
  const long b0 = ((long)((int)blockIdx.x - a.first[k]) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * NB;
  const bool full = t.vec && (b0 + NB) * 256 <= t.n;
  if constexpr (BITS == 32) {
    if (full) step32<G, NB, true>(t, c, b0);
    else step32<G, NB, false>(t, c, b0);
  } else {
    if (full) step8<G, NB, true>(t, c, b0);
    else step8<G, NB, false>(t, c, b0);
  }
}

// The values that 8-bit moments stand for: m and v = r^2 (both exact in fp32; m also in bf16).  A
// lane takes as many elements as fill a store of 16 bytes, so that a wave's stores are whole lines (fp32, 210 M
// elements: eight a lane 450 us, four 377).
template <class O, int NB, bool FULL>
__device__ __forceinline__ void values(const AdamWEntry& t, long b0) {
  using OV = typename Store<O>::type;
  using CV = typename Store<O>::codes;
  constexpr int E = 16 / sizeof(O), R = NB * 4 / E;  // elements of a lane, rounds of a wave
  const int lane = threadIdx.x & 63;
  const long n = t.n, i0 = b0 * 256 + E * lane;
  uint8_t mc[R][E], vc[R][E];
  int me[R], ve[R];
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const long b = (i0 + u * 64 * E) >> 8;
    const bool live = FULL || b * 256 < n;
    me[u] = live ? t.m_exp[b] : 0;
    ve[u] = live ? t.v_exp[b] : 0;
    load<FULL, CV, true>((const uint8_t*)t.m, i0 + u * 64 * E, n, mc[u]);
    load<FULL, CV, true>((const uint8_t*)t.v, i0 + u * 64 * E, n, vc[u]);
  }
#pragma unroll
  for (int u = 0; u < R; ++u) {
    O mo[E], vo[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float r = decode<4>(vc[u][e], ve[u]);
      mo[e] = (O)decode_m(mc[u][e], me[u]);
      vo[e] = (O)(r * r);
    }
    store<FULL, OV, true>((O*)t.m_out, i0 + u * 64 * E, n, mo);
    store<FULL, OV, true>((O*)t.v_out, i0 + u * 64 * E, n, vo);
  }
}

template <class O, int NB>
__global__ __launch_bounds__(256) void adamw_state_kernel(AdamWMulti a) {
  const int k = entry_of(a.first, a.count, blockIdx.x);
  const AdamWEntry& t = a.t[k];
  const long b0 = ((long)((int)blockIdx.x - a.first[k]) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * NB;
  if (t.vec && (b0 + NB) * 256 <= t.n) values<O, NB, true>(t, b0);
  else values<O, NB, false>(t, b0);
}

}  // namespace

template <class G, int BITS>
static void step(const AdamWMulti& a, dim3 grid, int chunk, hipStream_t s) {
  if (chunk == kAdamWMultiChunk) hipLaunchKernelGGL((adamw_multi_kernel<G, BITS, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((adamw_multi_kernel<G, BITS, 1>), grid, dim3(256), 0, s, a);
}

hipError_t launch_adamw_multi(const AdamWMulti& a, int chunks, int chunk, int bits, bool grad_bf16, hipStream_t s) {
  const dim3 grid((unsigned)chunks);
  if (bits == 32 && grad_bf16) step<bf16, 32>(a, grid, chunk, s);
  else if (bits == 32) step<float, 32>(a, grid, chunk, s);
  else if (grad_bf16) step<bf16, 8>(a, grid, chunk, s);
  else step<float, 8>(a, grid, chunk, s);
  return hipGetLastError();
}

hipError_t launch_adamw_state(const AdamWMulti& a, int chunks, bool out_bf16, hipStream_t s) {
  const dim3 grid((unsigned)chunks);
  if (out_bf16) hipLaunchKernelGGL((adamw_state_kernel<bf16, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((adamw_state_kernel<float, 4>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
