// Dropout from a counter-based generator: y = x / (1 - p) where the generator's 16 bits of an
// element are at or above 65536 p, else 0.  Nothing is stored for the backward, which is the
// same call on the gradient.
//
// Eight columns of a row are one item: one counter, one Philox of 10 rounds (20 multiplications of
// 32 x 32 bits, the costliest part), 16 bits for each element.  Words of 32 bits for each would double
// the generator's work, which then is no longer hidden behind memory.
#include <algorithm>

#include "kernels.h"
#include "philox.h"
#include "rows.h"

namespace {

constexpr int NT = 256;
constexpr int U = 2;  // items of a thread in flight

// x / n for inv = 2^32 / n + 1 (0 for n = 1): exact while x n < 2^32.
__device__ __forceinline__ int div_by(int x, uint32_t inv) { return inv ? (int)__umulhi((uint32_t)x, inv) : x; }

template <class T>
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
    store8<false>(y + (int64_t)row[u] * a.ldy + 8 * c8[u], n[u], v);
  }
}

}  // namespace

hipError_t launch_dropout(DropoutArgs a, bool f32, hipStream_t s) {
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  a.n8 = (a.cols + 7) / 8;
  a.inv = a.n8 > 1 ? (uint32_t)((1ull << 32) / a.n8 + 1) : 0;
  const int64_t groups = ((int64_t)a.rows * a.n8 + NT * U - 1) / (NT * U);
  if (f32) hipLaunchKernelGGL(dropout_kernel<float>, dim3((unsigned)groups), dim3(NT), 0, s, a);
  else hipLaunchKernelGGL(dropout_kernel<bf16>, dim3((unsigned)groups), dim3(NT), 0, s, a);
  return hipGetLastError();
}
