// Rotary positions with one to four axes (time, height, width, ...) on packed rows.
//
// Pair i of a head's rd / 2 belongs to one axis; its angle is pos[row, axis] times a
// frequency of the pair, and (u, w) -> (u cos - w sin, u sin + w cos).  The
// transpose (inverse) is the backward.  Pairs are (2 i, 2 i + 1) or (i, i + rd / 2).
//
// Angles: the frequencies are in turns, 64 bits, from the host; the row's turns
// are one 64-bit product, of which only the part within half a turn is kept
// (exact), so that far positions lose nothing, and cos / sin of that part are fp32.
//
// Bound by HBM for many heads: read and write of every rotated element (and, into
// another buffer, of the others).  cos and sin of a row serve all its heads: a
// workgroup takes up to 16 rows, starts the loads of its elements, forms the rows'
// cos and sin in LDS meanwhile, then rotates.  32749 rows of 20 heads of 128, bf16 in place: 335 MB
// in 58 us, 5.8 TB/s; 5003 rows of 32 fp32 heads of 256, a quarter of the dims rotated, into another
// buffer: 328 MB in 57 us, 5.7 TB/s (a copy of 4 GiB: 4.7).  257 rows of 32 heads of 80: 4.1 us, the launch and
// one way to memory; a call among others takes its host side, 7.8 us.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace {

constexpr int NT = 256;
constexpr int U = 2;        // items of a thread in flight (168 MB in place: 66.7 us, four 74.0, of streams 57.9 and 62.2)
constexpr int MAX_CS = 2048;  // (cos, sin) pairs in LDS: rows of a workgroup x pairs

template <class T, int V>
struct Item {
  T a[V], b[V];  // pairs apart: first and second halves; interleaved: a only
};

// STREAM: past the caches.
template <bool STREAM, class T, int V>
__device__ __forceinline__ void ld(const T* p, T (&x)[V]) {
  if constexpr (V * sizeof(T) == 16) {
    const u32x4* q = reinterpret_cast<const u32x4*>(p);
    const u32x4 w = STREAM ? __builtin_nontemporal_load(q) : *q;
    __builtin_memcpy(x, &w, 16);
  } else if constexpr (V * sizeof(T) == 8 && V > 2) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    __builtin_memcpy(x, &w, 8);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = p[e];
  }
}
template <bool STREAM, class T, int V>
__device__ __forceinline__ void st(T* p, const T (&x)[V]) {
  if constexpr (V * sizeof(T) == 16) {
    u32x4 w;
    __builtin_memcpy(&w, x, 16);
    u32x4* q = reinterpret_cast<u32x4*>(p);
    if (STREAM) __builtin_nontemporal_store(w, q);
    else *q = w;
  } else if constexpr (V * sizeof(T) == 8 && V > 2) {
    u32x2 w;
    __builtin_memcpy(&w, x, 8);
    *reinterpret_cast<u32x2*>(p) = w;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = x[e];
  }
}

// x / d for inv = 2^32 / d + 1 (0 for d = 1): exact while x d < 2^32 (of a row, x < H dh and d <= dh).
__device__ __forceinline__ int div_by(int x, uint32_t inv) { return inv ? (int)__umulhi((uint32_t)x, inv) : x; }

// V: elements of one load.  INTER: pairs (2 i, 2 i + 1), V of them = V / 2 pairs per
// item; otherwise an item is V pairs, V elements of each half.  Items of a row: for each head its
// rotated items, then (copy) its unrotated ones, V elements each.
template <class T, int V, bool INTER, bool STREAM>
__global__ __launch_bounds__(NT) void rotary_axes_kernel(RotaryAxes a) {
  __shared__ float2 cs[MAX_CS];
  const int t0 = blockIdx.x * a.rows_wg;
  const int rows = min(a.rows_wg, a.T - t0);
  const int total = rows * a.items;
  const T* x = (const T*)a.x + (long)t0 * a.ldx;
  T* y = (T*)a.y + (long)t0 * a.ldy;
  const int half = a.half;
  const int rot = INTER ? 2 * half / V : half / V;  // rotated items of a head

  auto place = [&](int i, int& row, int& off, int& pair) {
    row = a.rows_wg == 1 ? 0 : div_by(i, a.inv_items);
    const int r = i - row * a.items;
    const int h = div_by(r, a.inv_head_items);
    const int c = r - h * a.head_items;
    if (c < rot) {
      pair = INTER ? c * (V / 2) : c * V;
      off = h * a.dh + c * V;
    } else {
      pair = -1;
      off = h * a.dh + 2 * half + (c - rot) * V;
    }
  };
  auto load = [&](int i, Item<T, V>& it) {
    int row, off, pair;
    place(i, row, off, pair);
    const T* p = x + (long)row * a.ldx + off;
    ld<STREAM, T, V>(p, it.a);
    if (!INTER && pair >= 0) ld<STREAM, T, V>(p + half, it.b);
  };
  auto rotate = [&](int i, Item<T, V>& it) {
    int row, off, pair;
    place(i, row, off, pair);
    T* p = y + (long)row * a.ldy + off;
    if (pair >= 0) {
      const float2* q = cs + row * half + pair;
      if (INTER) {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          const float c = q[e].x, s = q[e].y;
          const float u = (float)it.a[2 * e], w = (float)it.a[2 * e + 1];
          it.a[2 * e] = (T)(u * c - w * s);
          it.a[2 * e + 1] = (T)(u * s + w * c);
        }
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float c = q[e].x, s = q[e].y;
          const float u = (float)it.a[e], w = (float)it.b[e];
          it.a[e] = (T)(u * c - w * s);
          it.b[e] = (T)(u * s + w * c);
        }
        st<STREAM, T, V>(p + half, it.b);
      }
    }
    st<STREAM, T, V>(p, it.a);
  };

  Item<T, V> it[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + u * NT;
    if (i < total) load(i, it[u]);
  }
  for (int i = threadIdx.x; i < rows * half; i += NT) {
    const int row = div_by(i, a.inv_half), pair = i - row * half;
    const double turns = (double)a.pos[(long)(t0 + row) * a.ldp + a.axis[pair]] * a.freq[pair];
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = make_float2(c, a.inverse ? -s : s);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + u * NT;
    if (i < total) rotate(i, it[u]);
  }
  for (int i = threadIdx.x + U * NT; i < total; i += NT) {
    load(i, it[0]);
    rotate(i, it[0]);
  }
}

uint32_t inv_of(int d) { return d == 1 ? 0u : (uint32_t)((1ull << 32) / d + 1); }

template <class T, int V>
hipError_t launch(RotaryAxes a, bool inter, bool copy, hipStream_t s) {
  const int rot = inter ? 2 * a.half / V : a.half / V;
  a.head_items = rot + (copy ? (a.dh - 2 * a.half) / V : 0);
  a.items = a.H * a.head_items;
  // Rows of a workgroup: about U items a thread, fewer while that leaves fewer than
  // four workgroups for each of the 256 CUs.
  int rows = std::max(1, std::min(std::min(16, U * NT / std::max(1, a.items)), MAX_CS / a.half));
  while (rows > 1 && sat_cdiv(a.T, rows) < 1024) --rows;
  a.rows_wg = rows;
  a.inv_items = inv_of(a.items);
  a.inv_head_items = inv_of(a.head_items);
  a.inv_half = inv_of(a.half);
  const dim3 grid((unsigned)sat_cdiv(a.T, rows));
  // What does not stay in the last-level cache (256 MB) for the next operator goes past the caches: 2 x 168 MB 57.9
  // us against 66.7, 2 x 96 MB from memory 34.2 against 39.5 (from the cache 33.5 against 31.5); 2 x 64 MB
  // would be 24.1 against 22.0.
  const bool stream = V * sizeof(T) == 16 && (double)a.T * a.H * (copy ? 2 * a.dh : 2 * a.half) * sizeof(T) >= 80e6;
  auto go = [&](auto inter_, auto stream_) {
    hipLaunchKernelGGL((rotary_axes_kernel<T, V, decltype(inter_)::value, decltype(stream_)::value>), grid, dim3(NT), 0, s, a);
    return hipGetLastError();
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if constexpr (V * sizeof(T) == 16)
    if (stream) return inter ? go(Yes(), Yes()) : go(No(), Yes());
  if constexpr (V > 1)
    if (inter) return go(Yes(), No());
  return go(No(), No());
}

}  // namespace

hipError_t launch_rotary_axes(const RotaryAxes& a, bool f32, bool inter, hipStream_t s) {
  if (a.T == 0 || a.H == 0) return hipSuccess;
  const bool copy = a.x != a.y;
  // widest load that divides every stretch of a row and is aligned in both buffers; two
  // elements or one are loaded one by one (dh is even)
  const int size = f32 ? 4 : 2;
  const auto fits = [&](int v) {
    const long bytes = (long)v * size;
    return (inter ? 2 * a.half : a.half) % v == 0 && a.dh % v == 0 && a.ldx % v == 0 && a.ldy % v == 0 &&
           reinterpret_cast<uintptr_t>(a.x) % bytes == 0 && reinterpret_cast<uintptr_t>(a.y) % bytes == 0;
  };
  const bool two = inter || a.half % 2 == 0;
  if (f32 && fits(4)) return launch<float, 4>(a, inter, copy, s);
  if (f32) return two ? launch<float, 2>(a, inter, copy, s) : launch<float, 1>(a, inter, copy, s);
  if (fits(8)) return launch<bf16, 8>(a, inter, copy, s);
  if (fits(4)) return launch<bf16, 4>(a, inter, copy, s);
  return two ? launch<bf16, 2>(a, inter, copy, s) : launch<bf16, 1>(a, inter, copy, s);
}
