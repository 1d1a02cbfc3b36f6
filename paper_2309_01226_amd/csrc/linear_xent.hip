// Softmax cross entropy of a linear head, with its gradients, without keeping the logits.
//
//   z = x w^T + b (rows t, vocabulary v)     lse_t = log sum_v exp z     loss_t = lse_t - z_label
//   dz = c_t (exp(z - lse_t) - [v = label])  dx = dz w     dw = dz^T x     db = sum_t dz
//
// Rows whose label is outside [0, V) take no part: the others are numbered in order (compact rows) and only
// they are worked on, as many as there are (known on the device alone).
//
// Three products carry it; there is no second product for the logits in the backward.  A 256 x 256 tile of
// the forward product stays in registers, where a token's logits of a piece of 128 vocabulary entries
// lie in two lanes: their maximum m and sum of exp(z - m) go out as the piece's statistics, and, for the
// gradients, (m - z) log2 e as a number of 16 bits, in steps of 2^-10 up to 32 and of 2^-8 up to 160.  Once all
// pieces give lse, dz is formed from those in place.  Half a step is 2^-11.5 of exp(z - m) (2^-9.5 of those below
// 2^-32), a small part of the rounding that a bf16 operand of the two other products takes, which exp(z - m)
// held as bf16 would double.  The label's entry, where 1 is subtracted, comes from the fp32 logit instead.  The numbers of a chunk of tokens are what is kept, at
// most 512 MiB, whatever N; several chunks add up dw in fp32.
//
// dz is an operand in bf16.  A chunk with no more rows than a tile has keeps what that rounding loses as a
// second operand: few roundings do not average out, and the products of so few rows are bound by the
// way of w and dw through memory.
//
// Bound by the matrix products (6 N V d operations), whose loop is the one of gemm256.hip.
#include <algorithm>

#include "gemm256_tile.h"
#include "rows.h"

namespace {

constexpr int PIECE = 128;   // vocabulary entries of one pair of statistics: the rows of a wave's part of a tile
constexpr int TB = 64;       // tokens of a workgroup of the scaling pass
constexpr int CUS = 256;
constexpr int EP = 136;      // fp32 pitch of a staging row
constexpr int QP = 68;       // its pitch in words of two 16-bit numbers
constexpr float LOG2E = 1.4426950408889634f;
constexpr float STEPS = 1024.f;   // of the fixed-point numbers; 65535 of them stand for 0
constexpr float INF = __builtin_inff();

__host__ __device__ inline int cdiv(int a, int b) { return (a + b - 1) / b; }

// K slices of a product of `tiles` tiles of `ktiles` 64-deep steps on 256 CUs.  Cost in steps of one tile:
// rounds of 256 workgroups, a step or two of start and end for each, and the partial products' way to
// memory and back (0.26 MB each way for a tile, about 0.064 steps).  At most 512 partial tiles (128 MB).
__host__ __device__ inline int pick_split(int tiles, int ktiles) {
  int best = 1;
  float cost = 0.f;
  for (int s = 1; s <= 16; ++s) {
    if (s > 1 && (tiles * s > 512 || ktiles < 8 * s)) break;
    const float c = (float)cdiv(tiles * s, CUS) * (cdiv(ktiles, s) + 2) + (s > 1 ? 0.064f * tiles * s : 0.f);
    if (s == 1 || c < cost) {
      best = s;
      cost = c;
    }
  }
  return best;
}

// The compact rows of the chunk that starts at `first`.
__device__ __forceinline__ int chunk_rows(const LinearXentArgs& a, int first) {
  return min(max(a.meta[0] - first, 0), a.chunk);
}

// Row c of the compact rows of x: x itself where every row takes part.
__device__ __forceinline__ const bf16* compact_x(const LinearXentArgs& a, long& ld) {
  const bool all = a.meta[0] == a.N;
  ld = all ? a.ldx : a.d;
  return all ? a.x : a.xc;
}

// Workgroup `bid` of `total`: the ids that an XCD is dealt are a contiguous range.
__device__ __forceinline__ int xcd_place(int bid, int total) {
  const int x = bid & 7, q = total >> 3, r = total & 7;
  return x * q + min(x, r) + (bid >> 3);
}

// ---------------------------------------------------------------- rows

// Numbers the rows that take part, in order, on one workgroup: idx, pos, lab of compact rows, their number; rows
// that do not get loss and lse 0.
__global__ __launch_bounds__(1024) void xent_rows_kernel(LinearXentArgs a) {
  __shared__ int sums[2][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0, turn = 0;
  int next = (int)threadIdx.x < a.N ? a.labels[threadIdx.x] : -1;
  for (int r0 = 0; r0 < a.N; r0 += 1024) {
    const int r = r0 + threadIdx.x, label = next;
    next = r + 1024 < a.N ? a.labels[r + 1024] : -1;
    const bool live = r < a.N && label >= 0 && label < a.V;
    const uint64_t mask = __builtin_amdgcn_ballot_w64(live);
    if (lane == 0) sums[turn][wave] = __popcll(mask);
    __syncthreads();
    int at = base + __popcll(mask & ((1ull << lane) - 1));
    for (int w = 0; w < 16; ++w) {
      const int n = sums[turn][w];
      if (w < wave) at += n;
      base += n;
    }
    turn ^= 1;
    if (live) {
      a.idx[at] = r;
      a.lab[at] = label;
    }
    if (r < a.N) {
      a.pos[r] = live ? at : -1;
      if (!live) a.row_loss[r] = a.lse[r] = 0.f;
    }
  }
  if (threadIdx.x == 0) {
    a.meta[0] = base;
    a.inv_n[0] = 1.f / max(base, 1);
  }
}

// One wave a row: x of rows that take part, to their compact place unless all do; zeros to dx of the others.
__global__ __launch_bounds__(256) void xent_copy_kernel(LinearXentArgs a) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.N || a.meta[0] == a.N) return;
  const int p = a.pos[r];
  const u32x4 zero = {0, 0, 0, 0};
  if (p >= 0) {
    for (int c = (threadIdx.x & 63) * 8; c < a.d; c += 512)
      *reinterpret_cast<u32x4*>(a.xc + (long)p * a.d + c) = *reinterpret_cast<const u32x4*>(a.x + r * a.ldx + c);
  } else if (a.dx != nullptr) {
    for (int c = (threadIdx.x & 63) * 8; c < a.d; c += 512)
      *reinterpret_cast<u32x4*>(a.dx + r * a.lddx + c) = zero;
  }
}

// ---------------------------------------------------------------- logits

template <int LAY>
struct Operand {
  const bf16* p;
  long ld;
  // from row0 on, at K-tile k0 of those from kb on
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(int row0, int kb, int k0) const {
    const bf16* q = p + (LAY == LAY_K ? (long)row0 * ld + kb : (long)(kb + k0) * ld + row0);
    return __builtin_amdgcn_make_buffer_rsrc((void*)q, (short)0, 0x7FFFFFFF, 0x00020000);
  }
};

// acc += A B over k in [kb, kb + K), and, where A2 is there, A2 B as well (A2's pitch is A's).
template <int AL, int BL>
__device__ __forceinline__ void tile_product(floatx16 (&acc)[4][4], bf16* smem, const Operand<AL>& A, const bf16* A2, const Operand<BL>& B,
                                             int m0, int M, int n0, int N, int kb, int K, int wave) {
  Loader<AL> la;
  Loader<BL> lb;
  la.init(A.ld, M - m0, wave);
  lb.init(B.ld, N - n0, wave);
  Frags<AL> FA;
  Frags<BL> FB;
  FA.init((wave >> 1) * 128);
  FB.init((wave & 1) * 128);
  const int n1 = cdiv(K, BK), nk = A2 != nullptr ? 2 * n1 : n1;
  gemm256_loop<AL, BL>(
      acc, smem, la, lb, FA, FB, [&](int t, int k0) { return Operand<AL>{t < n1 ? A.p : A2, A.ld}.at(m0, kb, k0); },
      [&](int, int k0) { return B.at(n0, kb, k0); }, nk, [&](int t) { return t < nk ? (t < n1 ? t : t - n1) * BK : K; }, K, wave);
}

// (m - z) log2 e >= 0, times 2^10, as 16 bits in the low half of a word: steps of 2^-10 up to 32, of 2^-8 from there to
// 160, 65535 for what is above.
__device__ __forceinline__ uint32_t to_steps(float s) {
  // 2^23 more: rounded to whole steps, which are the low bits
  return __float_as_uint(fminf(fminf(s, __builtin_fmaf(s, 0.25f, 24576.f)), 65535.f) + 8388608.f);
}
__device__ __forceinline__ float from_steps(uint32_t q) {
  const float s = (float)q;
  return q == 65535 ? 0.f : __builtin_amdgcn_exp2f(fmaxf(s, __builtin_fmaf(s, 4.f, -98304.f)) * (-1.f / STEPS));
}

// The tile's rows (in the wave's part: 32 i + 8 (r / 4) + 4 (lane / 32) + r % 4) are vocabulary
// entries, its columns (32 j + lane % 32) tokens.
template <bool TRAIN>
__global__ __launch_bounds__(NT, 1) void xent_logits_kernel(LinearXentArgs a, int first) {
  __shared__ __attribute__((aligned(1024))) bf16 smem[5 * OPE];
  const int n = chunk_rows(a, first), total = cdiv(a.V, BT) * cdiv(n, BT);
  if ((int)blockIdx.x >= total) return;
  int m0, n0;
  tile_origin(a.V, n, xcd_place(blockIdx.x, total), m0, n0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int v0 = m0 + (wave >> 1) * 128, t0 = n0 + (wave & 1) * 128;
  const int half = 4 * (lane >> 5);
  // the sums begin at the bias; entries behind the vocabulary are -inf
  floatx4 b[4][4];
  if (v0 + 128 <= a.V && a.bias != nullptr) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) b[i][g] = *reinterpret_cast<const floatx4_any*>(a.bias + v0 + 32 * i + 8 * g + half);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) b[i][g] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (v0 + 128 > a.V) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int v = v0 + 32 * i + 8 * (r >> 2) + half + (r & 3);
          b[i][r >> 2][r & 3] = v >= a.V ? -INF : a.bias != nullptr ? a.bias[v] : 0.f;
        }
    }
  }
  floatx16 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = b[i][r >> 2][r & 3];
  Operand<LAY_K> A = {a.w, a.ldw}, B;
  B.p = compact_x(a, B.ld);
  B.p += first * B.ld;
  tile_product<LAY_K, LAY_K>(acc, smem, A, nullptr, B, m0, a.V, n0, n, 0, a.d, wave);

  const int pieces = cdiv(a.V, PIECE);
  // the wave's 16 bits of its part, [32 tokens][128 entries] at a time
  uint32_t* st = reinterpret_cast<uint32_t*>(smem) + wave * 32 * QP;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int t = t0 + 32 * j + (lane & 31);
    const int off = t < n ? a.lab[first + t] - v0 : -1;
    if (__builtin_amdgcn_ballot_w64(off >= 0 && off < 128)) {
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) z = off - half == 32 * i + 8 * (r >> 2) + (r & 3) ? acc[i][j][r] : z;
      if (off >= 0 && off < 128 && (off & 4) == half) a.zlab[first + t] = z;
    }
    float m = -INF;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][j][r]);
    const auto mm = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = fmaxf(__uint_as_float(mm[0]), __uint_as_float(mm[1]));
    if (m == -INF) m = 0.f;  // no entry is left: every exp is 0
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // 0 for the largest, so that a sure row's loss is 0
          const float y = (m - acc[i][j][4 * g + e]) * (LOG2E * STEPS);
          s += __builtin_amdgcn_exp2f(y * (-1.f / STEPS));
          if (TRAIN) q[e] = to_steps(y);
        }
        if (TRAIN) {
          // the low halves of two words
          const u32x2 w = {__builtin_amdgcn_perm(q[1], q[0], 0x05040100), __builtin_amdgcn_perm(q[3], q[2], 0x05040100)};
          *reinterpret_cast<u32x2*>(st + (lane & 31) * QP + (32 * i + 8 * g + half) / 2) = w;
        }
      }
    const auto ss = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
    s = __uint_as_float(ss[0]) + __uint_as_float(ss[1]);
    if (lane < 32 && t < n && v0 < a.V) a.part[(long)t * pieces + v0 / PIECE] = make_float2(m, s);
    if constexpr (TRAIN) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int row = 4 * k + (lane >> 4);
        const u32x4 w = *reinterpret_cast<const u32x4*>(st + row * QP + 4 * (lane & 15));
        *reinterpret_cast<u32x4*>(a.e + (long)(t0 + 32 * j + row) * a.lde + v0 + 8 * (lane & 15)) = w;
      }
    }
  }
}

// 16 tokens x 16 slices of the pieces: lse and loss, and, for the gradients, every piece's factor c exp(m - lse).
template <bool TRAIN>
__global__ __launch_bounds__(256) void xent_join_kernel(LinearXentArgs a, int first) {
  __shared__ float2 sh[16][17];
  const int n = chunk_rows(a, first), tl = threadIdx.x >> 4, sl = threadIdx.x & 15;
  const int t0 = blockIdx.x * 16, t = t0 + tl;
  if (t0 >= n) return;
  const int pieces = cdiv(a.V, PIECE);
  float2* part = a.part + (long)min(t, n - 1) * pieces;
  float m = -INF, s = 0.f;
#pragma unroll 4
  for (int p = sl; p < pieces; p += 16) {
    const float2 q = part[p];
    if (q.y == 0.f) continue;  // no entry is left there
    const float top = fmaxf(m, q.x);
    s = s * __builtin_amdgcn_exp2f((m - top) * LOG2E) + q.y * __builtin_amdgcn_exp2f((q.x - top) * LOG2E);
    m = top;
  }
  sh[sl][tl] = make_float2(m, s);
  __syncthreads();
  m = -INF;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, sh[i][tl].x);
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float2 q = sh[i][tl];
    if (q.y != 0.f) s += q.y * __builtin_amdgcn_exp2f((q.x - m) * LOG2E);
  }
  if (t >= n) return;
  const bool none = s == 0.f;  // every entry is -inf
  const float log_s = none ? 0.f : logf(s), z = a.zlab[first + t] - m;
  const int row = a.idx[first + t];
  if (sl == 0) {
    a.lse[row] = none ? -INF : m + log_s;
    a.row_loss[row] = none ? 0.f : log_s - z;
  }
  if constexpr (TRAIN) {
    const float c = none ? 0.f : a.row_weight != nullptr ? a.row_weight[row] : a.inv_n[0];
    const float up = none ? 0.f : c / s;
    for (int p = sl; p < pieces; p += 16) {
      float2& q = part[p];
      q.x = none || q.y == 0.f ? 0.f : up * __builtin_amdgcn_exp2f((q.x - m) * LOG2E);
    }
    // the label's entry of dz
    if (sl == 0) a.zlab[first + t] = none ? 0.f : up * __builtin_amdgcn_exp2f(z * LOG2E) - c;
  }
}

// dz from the 16-bit numbers in place, for TB tokens and 2048 entries of the vocabulary: a thread has eight
// entries, of one piece, and goes from token to token.
template <bool DB>
__global__ __launch_bounds__(256) void xent_scale_kernel(LinearXentArgs a, int first) {
  const int n = chunk_rows(a, first), pieces = cdiv(a.V, PIECE), blocks = cdiv(a.V, 2048);
  const int tb = blockIdx.x / blocks, v = (blockIdx.x - tb * blocks) * 2048 + 8 * threadIdx.x;
  const int r0 = tb * TB, r1 = min(n, r0 + TB);
  if (r0 >= n || v >= a.V) return;
  const float2* part = a.part + v / PIECE;
  float db[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) db[e] = 0.f;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    u32x4* q = reinterpret_cast<u32x4*>(a.e + (long)r * a.lde + v);
    const u32x4 w = *q;
    const float f = part[(long)r * pieces].x;
    const int off = a.lab[first + r] - v;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = from_steps(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu) * f;
    if (off >= 0 && off < 8) {
      const float dl = a.zlab[first + r];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = off == e ? dl : x[e];
    }
    bf16x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (DB) db[e] += x[e];
      y[e] = f2bf(x[e]);
    }
    *reinterpret_cast<bf16x8*>(q) = y;
    if (n <= BT) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = f2bf(x[e] - bf2f(y[e]));
      *reinterpret_cast<bf16x8*>(a.e2 + (long)r * a.lde + v) = y;
    }
  }
  if (DB) store8<false>(a.dbpart + (long)tb * a.V + v, a.V - v, db);
}

// db of a chunk from its blocks of tokens, in order, added to the chunks before it.
__global__ __launch_bounds__(256) void xent_db_kernel(LinearXentArgs a, int first, int last) {
  const int v = blockIdx.x * 256 + threadIdx.x, blocks = cdiv(chunk_rows(a, first), TB);
  if (v >= a.V) return;
  float* f32 = reinterpret_cast<float*>(a.db);
  float* sum = a.dw_f32 ? f32 : a.dbsum;
  float s = (a.dw_f32 ? a.accumulate : 0) || first > 0 ? sum[v] : 0.f;
#pragma unroll 8
  for (int b = 0; b < blocks; ++b) s += a.dbpart[(long)b * a.V + v];
  if (a.dw_f32 || !last) sum[v] = s;
  else reinterpret_cast<bf16*>(a.db)[v] = f2bf(s);
}

// ---------------------------------------------------------------- the other products

// Where a row's eight columns go: fp32 or bf16, plus an fp32 addend.
struct RowsOut {
  void* out;
  long ld;
  bool f32;
  const float* add;  // may be out
  long ldadd;
  const int* map;    // row m is row map[m] of out
  __device__ __forceinline__ void put(int m, int col, float (&x)[8]) const {
    if (add != nullptr) {
      float b[8];
      widen8(load8<false>(add + (long)m * ldadd + col, 8), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += b[e];
    }
    const long o = (long)(map != nullptr ? map[m] : m) * ld + col;
    if (f32) store8<false>(reinterpret_cast<float*>(out) + o, 8, x);
    else store8<false>(reinterpret_cast<bf16*>(out) + o, 8, x);
  }
};

// C[m, c] = sum_k (A + A2)(m, k) B(c, k) of a tile (A2 may be absent), K split in S slices of kc: to `o`, or, with slices, to partial
// products [S][rows of whole tiles][N] in `partial`.
template <int AL>
__device__ __forceinline__ void product(bf16* smem, const Operand<AL>& A, const bf16* A2, const Operand<LAY_MN>& B, int M, int N,
                                         int K, int S, float* partial, const RowsOut& o) {
  const int tiles = cdiv(M, BT) * cdiv(N, BT), kc = cdiv(cdiv(K, BK), S) * BK;
  if ((int)blockIdx.x >= tiles * S) return;
  const int bid = xcd_place(blockIdx.x, tiles * S), slice = bid / tiles;
  int m0, n0;
  tile_origin(M, N, bid - slice * tiles, m0, n0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kb = slice * kc;
  floatx16 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  tile_product<AL, LAY_MN>(acc, smem, A, A2, B, m0, M, n0, N, kb, max(0, min(kc, K - kb)), wave);
  float* st = reinterpret_cast<float*>(smem) + wave * 32 * EP;
  const int cl = 8 * (lane & 15), col = n0 + (wave & 1) * 128 + cl;
  RowsOut q = o;
  if (S > 1) q = RowsOut{partial + (long)slice * cdiv(M, BT) * BT * N, N, true, nullptr, 0, nullptr};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        st[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * EP + 32 * j + (lane & 31)] = acc[i][j][r];
#pragma unroll 2
    for (int s = 0; s < 8; ++s) {
      const int rl = 4 * s + (lane >> 4), m = m0 + (wave >> 1) * 128 + 32 * i + rl;
      if (m >= M || col >= N) continue;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = st[rl * EP + cl + e];
      q.put(m, col, x);
    }
  }
}

__device__ __forceinline__ RowsOut dx_out(const LinearXentArgs& a, int first) {
  return RowsOut{a.dx, a.lddx, false, nullptr, 0, a.idx + first};
}
__device__ __forceinline__ int dx_split(const LinearXentArgs& a, int n) {
  return pick_split(cdiv(n, BT) * cdiv(a.d, BT), cdiv(a.V, BK));
}
// dw of one of several chunks goes to an fp32 sum; the last one's outcome to dw.
__device__ __forceinline__ RowsOut dw_out(const LinearXentArgs& a, int first, bool last) {
  const bool sum = a.dwsum != nullptr;
  RowsOut o = {a.dw, a.lddw, a.dw_f32 != 0, nullptr, 0, nullptr};
  if (sum) {
    if (first > 0) o.add = a.dwsum, o.ldadd = a.d;
    if (!last) o.out = a.dwsum, o.ld = a.d, o.f32 = true;
  } else if (first > 0 || a.accumulate) {
    o.add = reinterpret_cast<const float*>(a.dw);
    o.ldadd = a.lddw;
  }
  return o;
}
__device__ __forceinline__ int dw_split(const LinearXentArgs& a, int n) {
  return pick_split(cdiv(a.V, BT) * cdiv(a.d, BT), cdiv(n, BK));
}

__global__ __launch_bounds__(NT, 1) void xent_dx_kernel(LinearXentArgs a, int first) {
  __shared__ __attribute__((aligned(1024))) bf16 smem[5 * OPE];
  const int n = chunk_rows(a, first);
  const Operand<LAY_K> A = {a.e, a.lde};
  const Operand<LAY_MN> B = {a.w, a.ldw};
  product<LAY_K>(smem, A, n <= BT ? a.e2 : nullptr, B, n, a.d, a.V, dx_split(a, n), a.partial, dx_out(a, first));
}

__global__ __launch_bounds__(NT, 1) void xent_dw_kernel(LinearXentArgs a, int first, int last) {
  __shared__ __attribute__((aligned(1024))) bf16 smem[5 * OPE];
  const int n = chunk_rows(a, first);
  const Operand<LAY_MN> A = {a.e, a.lde};
  Operand<LAY_MN> B;
  B.p = compact_x(a, B.ld);
  B.p += first * B.ld;
  product<LAY_MN>(smem, A, n <= BT ? a.e2 : nullptr, B, a.V, a.d, n, dw_split(a, n), a.partial, dw_out(a, first, last));
}

// The slices of a product's tiles added in order; none where it was not split.
template <bool DW>
__global__ __launch_bounds__(256) void xent_slices_kernel(LinearXentArgs a, int first, int last) {
  const int n = chunk_rows(a, first), M = DW ? a.V : n, S = DW ? dw_split(a, n) : dx_split(a, n);
  if (S == 1) return;
  const RowsOut o = DW ? dw_out(a, first, last) : dx_out(a, first);
  const int n8 = a.d / 8;
  const long stride = (long)cdiv(M, BT) * BT * a.d, total = (long)M * n8;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long)gridDim.x * 256) {
    const int m = (int)(i / n8), col = (int)(i - (long)m * n8) * 8;
    const float* p = a.partial + (long)m * a.d + col;
    float x[8], b[8];
    widen8(load8<false>(p, 8), x);
    for (int s = 1; s < S; ++s) {
      widen8(load8<false>(p + s * stride, 8), b);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += b[e];
    }
    o.put(m, col, x);
  }
}

constexpr int64_t kMaxE = 1LL << 28;   // numbers of a chunk
constexpr int kMaxChunk = 16384;       // tokens of a chunk

// The workspace: 256-byte aligned parts, whose places go into `a` when it has a workspace.
struct Layout {
  int64_t bytes = 0;
  char* base;
  bool dx_split, dw_split;  // whether any number of rows has the product split
  template <class T>
  void part(T*& p, int64_t n) {
    p = n > 0 ? reinterpret_cast<T*>(base + bytes) : nullptr;
    bytes += (n * (int64_t)sizeof(T) + 255) / 256 * 256;
  }
};

void plan(LinearXentArgs& a, Layout& l) {
  const bool train = a.dx || a.dw || a.db;
  const int vp = cdiv(a.V, BT) * BT;
  int64_t cap = kMaxChunk;
  if (train) cap = std::min<int64_t>(cap, std::max<int64_t>(BT, kMaxE / vp / BT * BT));
  const int chunks = std::max(1, (int)((a.N + cap - 1) / cap));
  a.chunk = std::max(1, cdiv(cdiv(a.N, chunks), BT)) * BT;
  a.lde = vp;
  l.part(a.meta, 64);
  l.part(a.idx, a.N);
  l.part(a.pos, a.N);
  l.part(a.lab, a.N);
  l.part(a.zlab, a.N);
  l.part(a.part, (int64_t)cdiv(a.V, PIECE) * a.chunk);
  l.part(a.xc, (int64_t)a.N * a.d);
  l.part(a.e, train ? (int64_t)a.chunk * a.lde : 0);
  l.part(a.e2, train ? (int64_t)BT * a.lde : 0);
  l.part(a.dbpart, a.db ? (int64_t)cdiv(a.chunk, TB) * a.V : 0);
  l.part(a.dbsum, a.db && !a.dw_f32 && a.N > a.chunk ? a.V : 0);
  l.part(a.dwsum, a.dw && !a.dw_f32 && a.N > a.chunk ? (int64_t)a.V * a.d : 0);
  const int tn = cdiv(a.d, BT), tv = cdiv(a.V, BT);
  int64_t dx = 0, dw = 0;
  for (int n = BT; a.dx && n <= a.chunk; n += BT) {
    const int S = pick_split(n / BT * tn, cdiv(a.V, BK));
    if (S > 1) dx = std::max(dx, (int64_t)S * n * a.d);
  }
  for (int n = BK; a.dw && n <= a.chunk; n += BK) {
    const int S = pick_split(tv * tn, n / BK);
    if (S > 1) dw = std::max(dw, (int64_t)S * vp * a.d);
  }
  l.part(a.partial, std::max(dx, dw));
  l.dx_split = dx > 0;
  l.dw_split = dw > 0;
}

}  // namespace

int64_t linear_xent_ws(LinearXentArgs a) {
  Layout l;
  l.base = nullptr;
  plan(a, l);
  return l.bytes;
}

hipError_t launch_linear_xent(LinearXentArgs a, void* ws, hipStream_t s) {
  Layout l;
  l.base = (char*)ws;
  plan(a, l);
  const bool train = a.dx || a.dw || a.db;
  const int tn = cdiv(a.d, BT), tv = cdiv(a.V, BT), tt = cdiv(a.chunk, BT);
  hipLaunchKernelGGL(xent_rows_kernel, dim3(1), dim3(1024), 0, s, a);
  if (a.N > 0) hipLaunchKernelGGL(xent_copy_kernel, dim3(cdiv(a.N, 4)), dim3(256), 0, s, a);
  // without rows, too: dw and db of none
  for (int first = 0; first < std::max(a.N, 1); first += a.chunk) {
    const int last = first + a.chunk >= a.N;
    const auto logits = train ? xent_logits_kernel<true> : xent_logits_kernel<false>;
    hipLaunchKernelGGL(logits, dim3(tv * tt), dim3(NT), 0, s, a, first);
    hipLaunchKernelGGL(train ? xent_join_kernel<true> : xent_join_kernel<false>, dim3(cdiv(a.chunk, 16)), dim3(256), 0, s, a, first);
    if (!train) continue;
    hipLaunchKernelGGL(a.db ? xent_scale_kernel<true> : xent_scale_kernel<false>, dim3(cdiv(a.V, 2048) * cdiv(a.chunk, TB)), dim3(256), 0, s, a,
                       first);
    if (a.db) hipLaunchKernelGGL(xent_db_kernel, dim3(cdiv(a.V, 256)), dim3(256), 0, s, a, first, last);
    if (a.dx) {
      hipLaunchKernelGGL(xent_dx_kernel, dim3(std::max(tt * tn, 512)), dim3(NT), 0, s, a, first);
      if (l.dx_split) hipLaunchKernelGGL(xent_slices_kernel<false>, dim3(2048), dim3(256), 0, s, a, first, last);
    }
    if (a.dw) {
      hipLaunchKernelGGL(xent_dw_kernel, dim3(std::max(tv * tn, 512)), dim3(NT), 0, s, a, first, last);
      if (l.dw_split) hipLaunchKernelGGL(xent_slices_kernel<true>, dim3(2048), dim3(256), 0, s, a, first, last);
    }
  }
  return hipGetLastError();
}
