// Dropout from a counter-based generator: y = x / (1 - p) where the generator's 16 bits of an
// element are at or above 65536 p, else 0.  Nothing is stored for the backward, which is the
// same call on the gradient.
//
// Eight columns of a row are one item: one counter, one Philox of 10 rounds (20 products of 32 x 32 bits, the
// costliest part), 16 bits for each element.  With 32 bits for each there would be two Philox to an item, about the
// time of the item's way through memory.  Bound by HBM: 8192 x 16384 bf16, 1.07 GB in 85 us, 6.3 TB/s (a copy of 1
// GiB: 5.0); 32768 x 4096 fp32, 1.07 GB in 185 us, 5.8 TB/s.  257 x 1280: 7 us, the call's host side.
#include <algorithm>

#include "kernels.h"
#include "philox.h"
#include "rows.h"

namespace {

constexpr int NT = 256;
constexpr int U = 1;  // items of a thread (8192 x 16384: 91.5 us; two 101.5, four 103.6, cached stores)
// Elements from which on bf16 results go past the caches: what is read and written then nearly fills the last-level one
// of 256 MB (8192 x 16384: 91.5 -> 85 us; in turn with other operands, 16384 x 4096: 46.7 -> 45.2).  Not fp32, whose
// lanes store two 16-byte halves of lines apart (32768 x 4096: 185 -> 197 us).
constexpr int64_t kStream = 60000000;

// x / n for inv = 2^32 / n + 1 (0 for n = 1): exact while x n < 2^32.
__device__ __forceinline__ int div_by(int x, uint32_t inv) { return inv ? (int)__umulhi((uint32_t)x, inv) : x; }

template <class T, bool STREAM>
__global__ __launch_bounds__(NT) void dropout_kernel(DropoutArgs a) {
  const DropConsts c = {(uint32_t)a.seed, (uint32_t)(a.seed >> 32), a.limit, a.up, a.step};
  const uint64_t step = drop_step(c);
  // items of this workgroup: NT * U from `first` on, numbered row by row
  const int64_t first = (int64_t)blockIdx.x * (NT * U);
  const int row0 = (int)(first / a.n8), at0 = (int)(first - (int64_t)row0 * a.n8);
  const T* x = (const T*)a.x;
  T* y = (T*)a.y;
  Raw8<T> raw[U];
  int row[U], c8[U], n[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = at0 + u * NT + threadIdx.x, q = div_by(i, a.inv);
    row[u] = row0 + q;
    c8[u] = i - q * a.n8;
    n[u] = row[u] < a.rows ? a.cols - 8 * c8[u] : 0;
    if (n[u] > 0) raw[u] = load8<false>(x + (int64_t)row[u] * a.ldx + 8 * c8[u], n[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (n[u] <= 0) continue;
    const DropRow r = drop_bits(c, step, (uint32_t)row[u], (uint32_t)c8[u]);
    float v[8];
    widen8(raw[u], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = drop_keeps(c, r, e) ? v[e] * c.up : 0.f;
    store8<STREAM>(y + (int64_t)row[u] * a.ldy + 8 * c8[u], n[u], v);
  }
}

}  // namespace

hipError_t launch_dropout(DropoutArgs a, bool f32, hipStream_t s) {
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  a.n8 = (a.cols + 7) / 8;
  a.inv = a.n8 > 1 ? (uint32_t)((1ull << 32) / a.n8 + 1) : 0;
  const int64_t groups = ((int64_t)a.rows * a.n8 + NT * U - 1) / (NT * U);
  const bool stream = !f32 && (int64_t)a.rows * a.cols >= kStream;
  const auto kernel = f32 ? dropout_kernel<float, false> : stream ? dropout_kernel<bf16, true> : dropout_kernel<bf16, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(NT), 0, s, a);
  return hipGetLastError();
}
