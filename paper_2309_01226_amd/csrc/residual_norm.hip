// The boundary of two sublayers in one pass over the rows, forward and backward:
//
//   u = N_post(f)                    norm of the branch's rows, or f itself
//   y = alpha x + beta gate m u      m: dropout's 0 or 1 / (1 - p); y is rounded to the stream's type
//   h = N_pre(y)                     the next sublayer's input, from y as it is stored
//
//   t  = dy + N_pre'(dh)             the gradient at y
//   dx = alpha t                     du = beta gate m t       df = N_post'(du)
//   dgate = sum beta m u t           dg = sum g xh, db = sum g for each norm, over the rows
//   N'(g) = rs (a - mean(a) - xh mean(a xh)), a = gain g, xh the normalised row; RMS norms
//   subtract no mean.
//
// Bound by HBM: every array is read or written once (fp32 stream, 12 bytes an element forward and 18
// backward).  16384 x 4096, fp32, both norms: forward 146 us, 5.5 TB/s, backward 213 us, 5.7 TB/s (a copy of 1 GiB:
// 5.0); 16448 x 1280, bf16, backward 50 us, 5.0 TB/s; one row of 4096 9 us, the call's host side.
//
// A row belongs to d / 512 waves, or to 8, 16 or 32 lanes of one, eight columns a thread, so that a thread's
// columns stay the same from row to row: gains and the sums of their gradients live in its registers, and the next
// row's loads are in flight while a row is worked on.  A mean or a variance is formed inside each
// wave and joined by the pairwise formula of Chan, Golub and LeVeque (one barrier where a second pass
// over the row would take two).  The sums over rows go to one row of partial sums for each
// workgroup, added in order by a second kernel: the same bits on every call.
#include <algorithm>

#include "kernels.h"
#include "philox.h"
#include "rows.h"

namespace {

constexpr int CUS = 256;
constexpr int64_t kStream = 240000000;  // bytes of a call

// NARROW: rows of up to 256 columns, on 8, 16 or 32 lanes; else a row's place is the same for a whole wave.
template <bool NARROW>
struct RowPlace {
  int wpr;    // waves of a row
  int L;      // lanes of a row in each of them
  int rw;     // this thread's row among those of the workgroup
  int at;     // this wave's pair in the row's part of Shared
  int wave;   // this wave among its row's
  int col, n; // first column of the thread, and columns of the row from there on
  __device__ __forceinline__ RowPlace(int waves, int lanes, int d) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    wpr = NARROW ? 1 : waves;
    L = NARROW ? lanes : 64;
    const int q = w / wpr;
    wave = w - q * wpr;
    at = q * wpr;
    rw = NARROW ? q * (64 / L) + lane / L : q;
    col = 8 * (wave * 64 + lane % L);
    n = d - col;
  }
};

// Pairs of sums of up to 16 waves, two sets of them by turns: between a set's reads and its next
// writes every wave passes the other set's barrier.
struct Shared {
  float2 part[2][16];
};

// What a wave wrote to LDS is there for all; the next row's loads stay in flight.
__device__ __forceinline__ void share() {
  wait_lgkm0();
  cta_barrier();
}

// Sums of a and b over the row.
template <bool NARROW>
__device__ __forceinline__ float2 row_sums(const RowPlace<NARROW>& p, Shared& sh, int& turn, float a, float b) {
  float2 s = make_float2(group_total(a, p.L), group_total(b, p.L));
  if (p.wpr == 1) return s;
  float2* part = sh.part[turn];
  turn ^= 1;
  if ((threadIdx.x & 63) == 0) part[p.at + p.wave] = s;
  share();
  s = make_float2(0.f, 0.f);
  for (int i = 0; i < p.wpr; ++i) {
    const float2 q = part[p.at + i];
    s.x += q.x;
    s.y += q.y;
  }
  return s;
}

// Mean (0 for RMS) and reciprocal deviation of a row whose elements are v (0 behind its end).
template <bool NARROW>
__device__ __forceinline__ float2 row_stats(const RowPlace<NARROW>& p, Shared& sh, int& turn, const float (&v)[8], int kind,
                                            int d, float eps) {
  float s = 0.f;
  if (kind == kNormRms) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e] * v[e];
    return make_float2(0.f, rsqrtf(row_sums(p, sh, turn, s, 0.f).x / d + eps));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s += v[e];
  // columns of the row's i-th wave
  const auto width = [&](int i) { return (float)min(512, d - 512 * i); };
  float mean = group_total(s, p.L) / width(p.wave), m2 = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m2 += e < p.n ? (v[e] - mean) * (v[e] - mean) : 0.f;
  m2 = group_total(m2, p.L);
  if (p.wpr > 1) {
    float2* part = sh.part[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) part[p.at + p.wave] = make_float2(mean, m2);
    share();
    mean = m2 = 0.f;
    for (int i = 0; i < p.wpr; ++i) mean += part[p.at + i].x * width(i);
    mean /= d;
    for (int i = 0; i < p.wpr; ++i) {
      const float2 q = part[p.at + i];
      m2 += q.y + width(i) * (q.x - mean) * (q.x - mean);
    }
  }
  return make_float2(mean, rsqrtf(m2 / d + eps));
}

// Rows of a matrix that begin at row r0 for the workgroup, this thread's eight columns of its row; nothing where `on` is
// false or the row is not there.  FAST: rows are whole 16-byte pieces, and an access that is not wanted has an
// offset past the end of the buffer, for which the hardware reads zeros and writes nothing.  So no access
// stands behind a branch and the compiler's waits count exactly: the next row's loads stay in flight over the
// whole row (with branches it has to wait for them at once: 16384 rows of 4096, backward, 280 us instead of 229).
// FAST 2: bf16 past the caches.  Not fp32, whose lanes take halves of lines apart (16384 x 4096, backward with both
// norms: 219 us with the fp32 loads past them too, 214 without).
constexpr uint32_t NOWHERE = 0x80000000u;
constexpr int NONTEMPORAL = 2;
template <class T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const T* p) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, 0x7FFFFFFF, 0x00020000);
}
template <bool NARROW, class T>
__device__ __forceinline__ uint32_t place(const RowPlace<NARROW>& p, int64_t ld, int n) {
  return n > 0 ? (uint32_t)(((NARROW ? p.rw * (int)ld : 0) + p.col) * (int)sizeof(T)) : NOWHERE;
}
template <int FAST, bool NARROW, class T>
__device__ __forceinline__ Raw8<T> get(const RowPlace<NARROW>& p, const T* m, int64_t ld, int r0, int rows, bool on) {
  const int row = r0 + p.rw, n = on && row < rows ? p.n : 0;
  if constexpr (!FAST) return load8<false>(m + (int64_t)row * ld + p.col, n);
  const __amdgpu_buffer_rsrc_t b = buffer(m + (int64_t)(NARROW ? r0 : row) * ld);
  const uint32_t o = place<NARROW, T>(p, ld, n);
  constexpr int AUX = FAST == 2 ? NONTEMPORAL : 0;
  Raw8<T> r;
  if constexpr (sizeof(T) == 2) {
    r.w = __builtin_amdgcn_raw_buffer_load_b128(b, o, 0, AUX);
  } else {
    r.w[0] = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(b, o, 0, 0));
    r.w[1] = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(b, o, 16, 0));
  }
  return r;
}
template <int FAST, bool NARROW, class T>
__device__ __forceinline__ void put(const RowPlace<NARROW>& p, T* m, int64_t ld, int r0, int rows, bool on, const float (&x)[8]) {
  const int row = r0 + p.rw, n = on && row < rows ? p.n : 0;
  if constexpr (!FAST) {
    store8<false>(m + (int64_t)row * ld + p.col, n, x);
    return;
  }
  const __amdgpu_buffer_rsrc_t b = buffer(m + (int64_t)(NARROW ? r0 : row) * ld);
  const uint32_t o = place<NARROW, T>(p, ld, n);
  constexpr int AUX = FAST == 2 ? NONTEMPORAL : 0;
  if constexpr (sizeof(T) == 2) {
    bf16x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = f2bf(x[e]);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, y), b, o, 0, AUX);
  } else {
    const floatx4 lo = {x[0], x[1], x[2], x[3]}, hi = {x[4], x[5], x[6], x[7]};
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, lo), b, o, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, hi), b, o, 16, 0);
  }
}
// The row's pair of statistics, 0 for the branch's norm and 2 for the next one's.
template <int FAST, bool NARROW>
__device__ __forceinline__ float2 get_stats(const RowPlace<NARROW>& p, const float* stats, int which, int r0, int rows, bool on) {
  const int row = r0 + p.rw;
  const float* s = stats + (int64_t)which * rows + r0;
  if constexpr (!FAST) return on && row < rows ? make_float2(s[p.rw], s[rows + p.rw]) : make_float2(0.f, 0.f);
  const uint32_t o = on && row < rows ? (uint32_t)p.rw * 4 : NOWHERE;
  return make_float2(__uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer(s), o, 0, 0)),
                     __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer(s + rows), o, 0, 0)));
}
template <int FAST, bool NARROW>
__device__ __forceinline__ void put_stats(const RowPlace<NARROW>& p, float* stats, int which, int r0, int rows, bool on, float2 v) {
  const bool me = on && p.col == 0 && r0 + p.rw < rows;
  float* s = stats + (int64_t)which * rows + r0;
  if constexpr (!FAST) {
    if (me) s[p.rw] = v.x, s[rows + p.rw] = v.y;
    return;
  }
  const uint32_t o = me ? (uint32_t)p.rw * 4 : NOWHERE;
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v.x), buffer(s), o, 0, 0);
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v.y), buffer(s + rows), o, 0, 0);
}

// Columns of a vector for each channel, or `none` without one.
template <class P>
__device__ __forceinline__ void channels(const float* g, const P& p, float none, float (&x)[8]) {
  if (g != nullptr && p.n > 0) {
    widen8(load8<false>(g + p.col, p.n), x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = none;
  }
}

// beta gate m of eight columns of a row; exactly 0 where dropped.
template <class P>
__device__ __forceinline__ void branch_factors(const ResidualNormArgs& a, const DropConsts& c, uint64_t step, int row,
                                               const P& p, float scale, float (&m)[8]) {
  if (c.limit == 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = scale;
    return;
  }
  const DropRow r = drop_bits(c, step, (uint32_t)row, (uint32_t)p.col / 8);
#pragma unroll
  for (int e = 0; e < 8; ++e) m[e] = drop_keeps(c, r, e) ? scale : 0.f;
}

template <class XT, int MAXT, int FAST, bool NARROW = false>
__global__ __launch_bounds__(MAXT) void residual_norm_fwd_kernel(ResidualNormArgs a) {
  __shared__ Shared sh;
  int turn = 0;
  const RowPlace<NARROW> p(a.wpr, a.L, a.d);
  const DropConsts c = {(uint32_t)a.seed, (uint32_t)(a.seed >> 32), a.limit, a.up, a.step};
  const uint64_t step = drop_step(c);
  const float scale = a.beta * (c.limit ? c.up : 1.f);
  const int rows_wg = a.rows_wg, stride = gridDim.x * rows_wg, T = a.T;
  const XT* x = (const XT*)a.x;
  XT* y = (XT*)a.y;
  const bool pre = a.pre != 0, post = a.post != 0;
  float g_pre[8], b_pre[8], g_post[8], b_post[8], gate[8];
  channels(a.g_pre, p, 1.f, g_pre);
  channels(a.b_pre, p, 0.f, b_pre);
  channels(a.g_post, p, 1.f, g_post);
  channels(a.b_post, p, 0.f, b_post);
  channels(a.gate, p, 1.f, gate);
  Raw8<XT> nx;
  Raw8<bf16> nf;
  auto load = [&](int r0) {
    nx = get<FAST>(p, x, a.ldx, r0, T, true);
    nf = get<FAST>(p, a.f, a.ldf, r0, T, true);
  };
  // a row's outputs, in the order of the loop below; before the loop for no row, so that as many accesses follow
  // the first loads as the others
  const float none[8] = {};
  load(blockIdx.x * rows_wg);
  if (FAST) {
    put_stats<FAST>(p, a.stats, 0, 0, 0, false, make_float2(0.f, 0.f));
    put<FAST>(p, y, a.ldy, 0, 0, false, none);
    put<FAST>(p, a.h, a.ldh, 0, 0, false, none);
    put_stats<FAST>(p, a.stats, 2, 0, 0, false, make_float2(0.f, 0.f));
  }
  for (int r0 = blockIdx.x * rows_wg; r0 < T; r0 += stride) {
    const int row = r0 + p.rw;
    const int n = row < T ? p.n : 0;
    float v[8], u[8];
    widen8(nx, v);
    widen8(nf, u);
    load(r0 + stride);
    float2 st = make_float2(0.f, 0.f);
    if (post) {
      st = row_stats(p, sh, turn, u, a.post, a.d, a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = (u[e] - st.x) * st.y * g_post[e] + b_post[e];
    }
    put_stats<FAST>(p, a.stats, 0, r0, T, post, st);
    float m[8];
    branch_factors(a, c, step, row, p, scale, m);
    // a dropped element adds nothing, whatever the branch holds there
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = a.alpha * v[e] + (m[e] != 0.f ? m[e] * gate[e] * u[e] : 0.f);
    put<FAST>(p, y, a.ldy, r0, T, true, v);
    if (pre) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < n ? (float)(XT)v[e] : 0.f;
      st = row_stats(p, sh, turn, v, a.pre, a.d, a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (v[e] - st.x) * st.y * g_pre[e] + b_pre[e];
    }
    put<FAST>(p, a.h, a.ldh, r0, T, pre, v);
    put_stats<FAST>(p, a.stats, 2, r0, T, pre, st);
  }
}

// The workgroup's sums for its columns, of the rows it holds at once, to its row of partial sums.
template <class P>
__device__ __forceinline__ void put_sums(const ResidualNormArgs& a, const P& p, float* join, float* part,
                                         const float (&s)[8]) {
  if (a.rows_wg == 1) {
    store8<false>(part + p.col, p.n, s);
    return;
  }
  __syncthreads();
  const int w = 8 * p.L * p.wpr;
#pragma unroll
  for (int e = 0; e < 8; ++e) join[p.rw * w + p.col + e] = s[e];
  __syncthreads();
  for (int i = threadIdx.x; i < a.d; i += blockDim.x) {
    float t = 0.f;
    for (int r = 0; r < a.rows_wg; ++r) t += join[r * w + i];
    part[i] = t;
  }
}

// POST: with a norm of the branch.  Without one its sums' registers are free, and four waves fit a SIMD; with
// one, three, or two of rows of eight waves.  The widest rows take all 16 waves of a workgroup: there nothing is loaded
// ahead and gains are read again for each row (KEEP false).
template <class XT, int MAXT, bool POST, int FAST, bool NARROW = false>
__global__ __launch_bounds__(MAXT, MAXT > 768 ? 4 : MAXT > 512 ? 3 : 2) void residual_norm_bwd_kernel(ResidualNormArgs a) {
  __shared__ Shared sh;
  __shared__ float join[MAXT * 8];
  constexpr bool KEEP = FAST && MAXT <= 768;
  int turn = 0;
  const RowPlace<NARROW> p(a.wpr, a.L, a.d);
  const DropConsts c = {(uint32_t)a.seed, (uint32_t)(a.seed >> 32), a.limit, a.up, a.step};
  const uint64_t step = drop_step(c);
  const float scale = a.beta * (c.limit ? c.up : 1.f), inv_d = 1.f / a.d;
  const int rows_wg = a.rows_wg, stride = gridDim.x * rows_wg, T = a.T;
  const bool pre = a.pre != 0, branch = POST || a.dgate;  // whether the branch's rows are needed
  const XT* y = (const XT*)a.y;
  const XT* dy = (const XT*)a.dy;
  XT* dx = (XT*)a.dx;
  float g_pre[8], g_post[8], b_post[8], gate[8];
  const auto vectors = [&]() {
    if (POST) {
      channels(a.g_post, p, 1.f, g_post);
      channels(a.b_post, p, 0.f, b_post);
    }
    channels(a.gate, p, 1.f, gate);
  };
  if (KEEP) {
    channels(a.g_pre, p, 1.f, g_pre);
    vectors();
  }
  Raw8<XT> ny, ndy;
  Raw8<bf16> nf, ndh;
  float2 nst, npost;
  auto load = [&](int r0) {
    ny = get<FAST>(p, y, a.ldy, r0, T, pre);
    ndh = get<FAST>(p, a.dh, a.lddh, r0, T, pre);
    nst = get_stats<FAST>(p, a.stats, 2, r0, T, pre);
    ndy = get<FAST>(p, dy, a.lddy, r0, T, dy != nullptr);
    nf = get<FAST>(p, a.f, a.ldf, r0, T, branch);
    npost = get_stats<FAST>(p, a.stats, 0, r0, T, POST);
  };
  if (KEEP) {
    load(blockIdx.x * rows_wg);
    // as many accesses after the first loads as after the others
    const float none[8] = {};
    put<FAST>(p, dx, a.lddx, 0, 0, false, none);
    put<FAST>(p, a.df, a.lddf, 0, 0, false, none);
  }
  float s_gpre[8], s_bpre[8], s_gpost[8], s_bpost[8], s_gate[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s_gpre[e] = s_bpre[e] = s_gpost[e] = s_bpost[e] = s_gate[e] = 0.f;
  for (int r0 = blockIdx.x * rows_wg; r0 < T; r0 += stride) {
    const int row = r0 + p.rw;
    const int n = row < T ? p.n : 0;
    if (!KEEP) load(r0);
    float t[8], yh[8], g[8], f[8];
    widen8(ndy, t);
    widen8(ny, yh);
    widen8(ndh, g);
    widen8(nf, f);
    const float2 st = nst, pst = npost;
    if (KEEP) load(r0 + stride);
    if (pre) {
      if (!KEEP) channels(a.g_pre, p, 1.f, g_pre);
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        yh[e] = e < n ? (yh[e] - st.x) * st.y : 0.f;
        s_gpre[e] += g[e] * yh[e];
        s_bpre[e] += g[e];
        g[e] *= g_pre[e];
        s0 += g[e];
        s1 += g[e] * yh[e];
      }
      const float2 s = row_sums(p, sh, turn, s0, s1);
      const float m0 = a.pre == kNormRms ? 0.f : s.x * inv_d, m1 = s.y * inv_d;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] += st.y * (g[e] - m0 - yh[e] * m1);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = a.alpha * t[e];
    put<FAST>(p, dx, a.lddx, r0, T, true, g);
    float m[8];
    branch_factors(a, c, step, row, p, scale, m);
    if (POST) {
      if (!KEEP) vectors();
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[e] = e < n ? (f[e] - pst.x) * pst.y : 0.f;
        const float tm = e < n && m[e] != 0.f ? t[e] * m[e] : 0.f;
        if (m[e] != 0.f) s_gate[e] += tm * (f[e] * g_post[e] + b_post[e]);
        const float du = tm * gate[e];
        s_gpost[e] += du * f[e];
        s_bpost[e] += du;
        t[e] = du * g_post[e];
        s0 += t[e];
        s1 += t[e] * f[e];
      }
      const float2 s = row_sums(p, sh, turn, s0, s1);
      const float m0 = a.post == kNormRms ? 0.f : s.x * inv_d, m1 = s.y * inv_d;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = pst.y * (t[e] - m0 - f[e] * m1);
    } else {
      if (!KEEP) vectors();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float tm = e < n && m[e] != 0.f ? t[e] * m[e] : 0.f;
        if (m[e] != 0.f) s_gate[e] += tm * f[e];
        t[e] = tm * gate[e];
      }
    }
    put<FAST>(p, a.df, a.lddf, r0, T, true, t);
  }
  float* part = a.ws + (int64_t)blockIdx.x * a.sums * a.d;
  if (a.dg_pre) put_sums(a, p, join, part, s_gpre), part += a.d;
  if (a.db_pre) put_sums(a, p, join, part, s_bpre), part += a.d;
  if (POST && a.dg_post) put_sums(a, p, join, part, s_gpost), part += a.d;
  if (POST && a.db_post) put_sums(a, p, join, part, s_bpost), part += a.d;
  if (a.dgate) put_sums(a, p, join, part, s_gate);
}

// Partial sums of G workgroups, added in order: 64 columns of one sum for each workgroup, 16 slices of the
// partial rows.
struct SumOut {
  float* out[5];
};
__global__ __launch_bounds__(1024) void residual_norm_sums_kernel(const float* __restrict__ ws, int G, int sums, int d,
                                                                  SumOut o) {
  __shared__ float part[16][64];
  const int k = blockIdx.y, lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  const int per = (G + 15) / 16, g1 = min(G, (slice + 1) * per);
  float s = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int g = slice * per; g < g1; ++g) s += ws[((int64_t)g * sums + k) * d + col];
  }
  part[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && col < d) {
    for (int i = 1; i < 16; ++i) s += part[i][lane];
    o.out[k][col] = s;
  }
}

int waves_of_row(int d) { return (d + 511) / 512; }
int lanes_of_row(int d) { return d > 256 ? 64 : d > 128 ? 32 : d > 64 ? 16 : 8; }

// A backward workgroup, one on a CU: its most threads by the kernel's registers, and rows of waves in it.
struct BwdShape {
  int most, lines;
};
BwdShape bwd_shape(int d, bool fast) {
  const int w = waves_of_row(d);
  if (d <= 256) return {768, 12};
  if (!fast || w > 12) return {1024, std::max(1, 16 / w)};
  return w == 7 || w == 8 ? BwdShape{512, 1} : BwdShape{768, 12 / w};
}
int bwd_rows_wg(int d, const BwdShape& b) { return b.lines * (64 / lanes_of_row(d)); }
int bwd_groups(int T, int d, const BwdShape& b) { return std::min(CUS, sat_cdiv(T, bwd_rows_wg(d, b))); }

using Kernel = void (*)(ResidualNormArgs);
template <class XT>
Kernel fwd_kernel(int L, int threads, int fast) {
  if (L < 64) return fast ? residual_norm_fwd_kernel<XT, 256, 1, true> : residual_norm_fwd_kernel<XT, 256, 0, true>;
  if (!fast) return residual_norm_fwd_kernel<XT, 1024, 0>;
  if (fast == 2)
    return threads <= 256   ? residual_norm_fwd_kernel<XT, 256, 2>
           : threads <= 512 ? residual_norm_fwd_kernel<XT, 512, 2>
                            : residual_norm_fwd_kernel<XT, 1024, 2>;
  return threads <= 256   ? residual_norm_fwd_kernel<XT, 256, 1>
         : threads <= 512 ? residual_norm_fwd_kernel<XT, 512, 1>
                          : residual_norm_fwd_kernel<XT, 1024, 1>;
}
template <class XT, bool POST>
Kernel bwd_kernel(int L, int most, int fast) {
  if (L < 64) return fast ? residual_norm_bwd_kernel<XT, 768, POST, 1, true> : residual_norm_bwd_kernel<XT, 768, POST, 0, true>;
  if (!fast) return residual_norm_bwd_kernel<XT, 1024, POST, 0>;
  if (fast == 2)
    return most == 512   ? residual_norm_bwd_kernel<XT, 512, POST, 2>
           : most == 768 ? residual_norm_bwd_kernel<XT, 768, POST, 2>
                         : residual_norm_bwd_kernel<XT, 1024, POST, 2>;
  return most == 512   ? residual_norm_bwd_kernel<XT, 512, POST, 1>
         : most == 768 ? residual_norm_bwd_kernel<XT, 768, POST, 1>
                       : residual_norm_bwd_kernel<XT, 1024, POST, 1>;
}

int sum_outputs(const ResidualNormArgs& a, SumOut* o) {
  int n = 0;
  for (float* q : {a.dg_pre, a.db_pre, a.dg_post, a.db_post, a.dgate})
    if (q) o->out[n++] = q;
  return n;
}

}  // namespace

// (the same for either way of access, so that alignment does not matter to the caller)
int64_t residual_norm_ws(int T, int d, int sums) {
  return (int64_t)std::max(bwd_groups(T, d, bwd_shape(d, true)), bwd_groups(T, d, bwd_shape(d, false))) * sums * d;
}

// How rows are accessed: 1 where they are whole 16-byte pieces, of every array that is there; 2 with bf16 past the caches
// as well, where all arrays together nearly fill the last-level one (256 MB), so that the next kernel would not find the
// results there.  us with and without, operands in turn, rows of 4096: a backward of 300 MB, bf16, 57 and 63; of
// 1.2 GB, fp32, both norms 213 and 219; a forward of 0.8 GB, fp32, both norms 146 and 152.  A bf16 forward and a copy of h:
// 200 MB in all 57 and 56, 250 MB 70 and 73, 300 MB 83 and 91.
// 0, by elements, where they are not: dearest backward, where nothing is loaded ahead and the kernel with a norm of the branch
// spills.  Both norms, gate, all sums, fp32: 16384 x 4095 forward 204 us, backward 401 (4096: 178 and 229), 16448 x 1283
// 82 and 150 (1280: 72 and 90).
static int fast_rows(const ResidualNormArgs& a, bool f32, bool back) {
  bool ok = a.d % 8 == 0;
  const auto rows = [&](const void* p, int64_t ld, int size) {
    if (p != nullptr) ok = ok && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * size % 16 == 0 && ld < (1 << 21);
  };
  const int size = f32 ? 4 : 2;
  rows(a.y, a.ldy, size);
  rows(a.f, a.ldf, 2);
  if (back) {
    rows(a.dy, a.lddy, size);
    rows(a.dx, a.lddx, size);
    rows(a.dh, a.lddh, 2);
    rows(a.df, a.lddf, 2);
  } else {
    rows(a.x, a.ldx, size);
    rows(a.h, a.ldh, 2);
  }
  if (!ok) return 0;
  const int wide = back ? 2 + !!a.pre : 2, narrow = back ? 1 + !!a.pre + (a.post || a.dgate) : 1 + !!a.pre;  // arrays
  const int64_t bytes = (int64_t)a.T * a.d * (wide * size + narrow * 2);
  return bytes >= kStream ? 2 : 1;
}

hipError_t launch_residual_norm_fwd(ResidualNormArgs a, bool f32, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  a.wpr = waves_of_row(a.d);
  a.L = lanes_of_row(a.d);
  const int lines = std::max(1, 4 / a.wpr);  // of waves
  a.rows_wg = lines * (64 / a.L);
  const int threads = 64 * a.wpr * lines;
  const dim3 grid(std::min(sat_cdiv(a.T, a.rows_wg), CUS * std::max(1, 1024 / threads)));
  const int fast = fast_rows(a, f32, false);
  const Kernel kernel = f32 ? fwd_kernel<float>(a.L, threads, fast) : fwd_kernel<bf16>(a.L, threads, fast);
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_residual_norm_bwd(ResidualNormArgs a, bool f32, hipStream_t s) {
  SumOut o;
  a.sums = sum_outputs(a, &o);
  a.wpr = waves_of_row(a.d);
  a.L = lanes_of_row(a.d);
  const int fast = fast_rows(a, f32, true);
  const BwdShape shape = bwd_shape(a.d, fast);
  a.rows_wg = bwd_rows_wg(a.d, shape);
  const int threads = 64 * a.wpr * shape.lines, G = bwd_groups(a.T, a.d, shape);
  if (G > 0) {
    const auto pick = f32 ? (a.post ? bwd_kernel<float, true> : bwd_kernel<float, false>)
                          : (a.post ? bwd_kernel<bf16, true> : bwd_kernel<bf16, false>);
    const Kernel kernel = pick(a.L, shape.most, fast);
    hipLaunchKernelGGL(kernel, dim3(G), dim3(threads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.sums == 0) return hipSuccess;
  hipLaunchKernelGGL(residual_norm_sums_kernel, dim3(sat_cdiv(a.d, 64), a.sums), dim3(1024), 0, s, a.ws, G, a.sums, a.d, o);
  return hipGetLastError();
}
