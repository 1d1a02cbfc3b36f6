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
// held as bf16 would double.  The label's entry, where 1 is subtracted, comes from the fp32 logit instead.  The
// numbers of a chunk of tokens are what is kept, at most 1 GiB, whatever N; several chunks add up dw in fp32
// (8192 x 50257 x 768 as two chunks instead of one takes 5% longer, as four 19%).
//
// dz is an operand in bf16.  A chunk with no more rows than a tile has keeps what that rounding loses as a
// second operand: few roundings do not average out, and the products of so few rows are bound by the
// way of w and dw through memory (64 x 50400 x 4096: 420 us, the logits 122, dx and dw 291; w twice and dw once at a
// copy's rate take 248).
//
// Bound by the matrix products (6 N V d operations), whose loop is the one of gemm256.hip.  8192 x 50257 x 768: 2.32 ms
// or 0.82 PFLOP/s, of which the logits take 0.77, dx 0.56, dw 0.56 and the pass that forms dz 0.36 (1.65 GB, 4.6
// TB/s); 4096 x 50400 x 4096: 4.50 ms, 1.13 PFLOP/s, 1.44, 1.31, 1.55 and 0.16 (means of one profile; cards differ by 5%).
// 8 x 50257 x 1024 without gradients: 28 us with w from HBM, the product 22.6 or 4.6 TB/s.  64 x 512 x 64: 26 us, of which
// dx and dw 12.7 and the logits 6.7, whose few workgroups each go through all of K; two launches the rest.
#include <algorithm>

#include "gemm256_tile.h"
#include "rows.h"

namespace {

constexpr int CUS = 256;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float STEPS = 1024.f;   // of the fixed-point numbers; 65535 of them stand for 0
constexpr float INF = __builtin_inff();

__host__ __device__ inline int cdiv(int a, int b) { return (a + b - 1) / b; }

// A product of `tiles` tiles of R rows and columns and `ktiles` 64-deep steps on 256 CUs: `full` tiles in whole
// rounds, one for each CU, and the rest, whose K is split in S slices where that shortens the last round.  Cost in ns:
// a round takes 1650 for each step and 11000 for its start and end, of tiles of 128 700 and 4000, but in whole rounds,
// with two on a CU, 580 and 1000; a partial tile's way to memory and back 100 (26), the launch that adds the slices
// 4000.  At most 128 MB of partial tiles a product.  Whole numbers: the host plans the workspace and the launch by what the
// rows' kernel then chooses on the device (by the number of rows that take part), so both have to choose alike.
constexpr int SLICES = 64;
struct Split {
  int full, rest, S;
  __host__ __device__ int groups() const { return full + rest * S; }
  __host__ __device__ int64_t partial(int R) const { return S > 1 ? (int64_t)rest * S * R * R : 0; }
};
__host__ __device__ inline bool slices_fit(int R, int tiles, int ktiles, int s) {
  return s == 1 || (tiles % CUS * s <= (R == BT ? 512 : 2048) && ktiles >= 4 * s);
}
__host__ __device__ inline int64_t round_ns(int R, int steps) {
  return R == BT ? (int64_t)steps * 1650 + 11000 : (int64_t)steps * 700 + 4000;
}
// Cost of the rest in s slices; the least number wins, of equal ones the fewest slices (the low bits).
__host__ __device__ inline int64_t slices_key(int R, int tiles, int ktiles, int s) {
  const int rest = tiles % CUS, way = R == BT ? 100 : 26;
  if (!slices_fit(R, tiles, ktiles, s)) return INT64_MAX;
  const int64_t ns = cdiv(rest * s, CUS) * round_ns(R, cdiv(ktiles, s)) + (s > 1 ? way * rest * s + 4000 : 0);
  return ns * 128 + s;
}
// The best number of slices up to `most`, by one wave.
__device__ __forceinline__ int wave_slices(int R, int tiles, int ktiles, int most) {
  const int s = 1 + (threadIdx.x & 63);
  int64_t key = s <= most ? slices_key(R, tiles, ktiles, s) : INT64_MAX;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) key = min(key, (int64_t)__shfl_xor((long long)key, o, SAT_WAVE));
  return (int)(key & 127);
}
inline Split split_of(int R, int tiles, int ktiles, int64_t* ns = nullptr, int most = SLICES) {
  int64_t key = INT64_MAX;
  for (int s = 1; s <= most && slices_fit(R, tiles, ktiles, s); ++s) key = std::min(key, slices_key(R, tiles, ktiles, s));
  if (ns) *ns = key / 128 + tiles / CUS * (R == BT ? round_ns(R, ktiles) : (int64_t)ktiles * 580 + 1000);
  return Split{tiles / CUS * CUS, tiles % CUS, (int)(key & 127)};
}
__host__ __device__ inline int tiles_of(int R, int M, int N) { return cdiv(M, R) * cdiv(N, R); }

// Tiles and K steps of dx = dz w and of dw = dz^T x for n rows.
__host__ __device__ inline int dx_tiles(int R, const LinearXentArgs& a, int n) { return tiles_of(R, n, a.d); }
__host__ __device__ inline int dx_steps(const LinearXentArgs& a) { return cdiv(a.V, BK); }
__host__ __device__ inline int dw_tiles(int R, const LinearXentArgs& a) { return tiles_of(R, a.V, a.d); }
__host__ __device__ inline int dw_steps(int n) { return cdiv(n, BK); }

// The compact rows, and those of the chunk that starts at `first`.
__device__ __forceinline__ int compact_rows(const LinearXentArgs& a) { return a.direct ? a.N : a.meta[0]; }
__device__ __forceinline__ int chunk_rows(const LinearXentArgs& a, int first) {
  return min(max(compact_rows(a) - first, 0), a.chunk);
}

// Whether the chunk has anything to do (the first one also without rows: gradients of none), and whether none
// comes after it.
__device__ __forceinline__ bool chunk_idle(const LinearXentArgs& a, int first) { return first > 0 && a.meta[0] <= first; }
__device__ __forceinline__ bool chunk_last(const LinearXentArgs& a, int first) { return a.meta[0] <= first + a.chunk; }

// What the sums of all rows' dz are multiplied by: dz holds a row's own weight, but without weights the common 1 / n
// stays out of it.  Labels' entries near -1 round best just below a power of two, those near -1 / n wherever that
// happens to lie (7232 rows, 66 entries, d 96: dx is off by 0.21% instead of 0.26%, of which its own rounding is 0.17%).
__device__ __forceinline__ float common_factor(const LinearXentArgs& a) { return a.row_weight != nullptr ? 1.f : a.inv_n[0]; }

// Row c of the compact rows of x: x itself where every row takes part.
__device__ __forceinline__ const bf16* compact_x(const LinearXentArgs& a, long& ld) {
  const bool all = compact_rows(a) == a.N;
  ld = all ? a.ldx : a.d;
  return all ? a.x : a.xc;
}

// Workgroup `bid` of `total`: the ids that an XCD is dealt are a contiguous range.
__device__ __forceinline__ int xcd_place(int bid, int total) {
  const int x = bid & 7, q = total >> 3, r = total & 7;
  return x * q + min(x, r) + (bid >> 3);
}

// How the products of the chunk that is not full are split, by one wave each: meta[1] dx, meta[2] dw (whose K is the
// chunk's rows: no more slices than a full one's).
__device__ __forceinline__ void choose_slices(const LinearXentArgs& a, int rows, int which) {
  const int n = rows % a.chunk;
  const int S = which == 1 ? wave_slices(a.rx, dx_tiles(a.rx, a, n), dx_steps(a), SLICES)
                           : wave_slices(a.rw, dw_tiles(a.rw, a), dw_steps(n), a.s_dw);
  if ((threadIdx.x & 63) == 0) a.meta[which] = S;
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
  if (wave == 1 || wave == 2) choose_slices(a, base, wave);
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

// Both at once for up to FEW rows: a workgroup, which has four rows, counts the rows before them (and all of them) for
// itself.  (1019 x 739 x 2576, 30% without a label: 6 us; with 64 rows for a workgroup, 33.  The whole of 8192 x 66 x
// 96, half without: 32 us, with the two kernels above 36; of 16384 rows 50 and 50, of 24000 74 and 67.)
constexpr int FEW = 12000;
__global__ __launch_bounds__(256) void xent_rows_few_kernel(LinearXentArgs a) {
  __shared__ int sums[2][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = blockIdx.x * 4, r = r0 + wave;
  const auto live = [&](int i) {
    const int label = i < a.N ? a.labels[i] : -1;
    return label >= 0 && label < a.V;
  };
  int before = 0, all = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < a.N; i += 256) {
    const int one = live(i);
    all += one;
    before += i < r0 ? one : 0;
  }
  before = (int)wave_total((float)before);  // whole numbers below 2^24: exact
  all = (int)wave_total((float)all);
  if (lane == 0) {
    sums[0][wave] = before;
    sums[1][wave] = all;
  }
  __syncthreads();
  all = sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3];
  if (r0 == 0) {
    if (threadIdx.x == 0) {
      a.meta[0] = all;
      a.inv_n[0] = 1.f / max(all, 1);
    }
    if (wave == 1 || wave == 2) choose_slices(a, all, wave);
  }
  if (r >= a.N) return;
  const int label = a.labels[r];
  const bool on = label >= 0 && label < a.V;
  int p = sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3];
  for (int i = r0; i < r; ++i) p += live(i);
  if (lane == 0) {
    if (on) {
      a.idx[p] = r;
      a.lab[p] = label;
    } else {
      a.row_loss[r] = a.lse[r] = 0.f;
    }
  }
  if (all == a.N || (!on && a.dx == nullptr)) return;
  const bf16* from = a.x + r * a.ldx;
  bf16* to = on ? a.xc + (long)p * a.d : a.dx + r * a.lddx;
#pragma unroll 4
  for (int c = lane * 8; c < a.d; c += 512) {
    u32x4 v = {0, 0, 0, 0};
    if (on) v = *reinterpret_cast<const u32x4*>(from + c);
    *reinterpret_cast<u32x4*>(to + c) = v;
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

// A tile of R x R, of which a wave has W = R / 2 rows and columns in S x S accumulators; elements of LDS with ST stages.
template <int R>
struct Tile {
  static constexpr int W = R / 2, S = W / 32;
};
constexpr int lds_of(int R, int ST) { return R == BT ? 5 * OPE : small_lds(ST); }
template <int R>
using Acc = floatx16[Tile<R>::S][Tile<R>::S];

// acc += A B over k in [kb, kb + K), and, where A2 is there, A2 B as well (A2's pitch is A's): each K-tile of B is
// asked for twice in a row, and comes from memory once.
template <int R, int ST, int AL, int BL>
__device__ __forceinline__ void tile_product(Acc<R>& acc, bf16* smem, const Operand<AL>& A, const bf16* A2, const Operand<BL>& B,
                                             int m0, int M, int n0, int N, int kb, int K, int wave) {
  Loader<AL, R> la;
  Loader<BL, R> lb;
  la.init(A.ld, M - m0, wave);
  lb.init(B.ld, N - n0, wave);
  Frags<AL, R> FA;
  Frags<BL, R> FB;
  FA.init((wave >> 1) * Tile<R>::W);
  FB.init((wave & 1) * Tile<R>::W);
  const int parts = A2 != nullptr ? 2 : 1, nk = parts * cdiv(K, BK);
  const auto rsA = [&](int t, int k0) { return Operand<AL>{t & (parts - 1) ? A2 : A.p, A.ld}.at(m0, kb, k0); };
  const auto rsB = [&](int, int k0) { return B.at(n0, kb, k0); };
  const auto kof = [&](int t) { return t < nk ? (t >> (parts - 1)) * BK : K; };
  if constexpr (R == BT) gemm256_loop<AL, BL>(acc, smem, la, lb, FA, FB, rsA, rsB, nk, kof, K, wave);
  else gemm128_loop<ST, AL, BL>(acc, smem, la, lb, FA, FB, rsA, rsB, nk, kof, K, wave);
}

// u = (z - m) log2 e <= 0 as 16 bits in the low half of a word: steps of 2^-10 from 0 down to -32, of 2^-8 from there to
// -160, 65535 for what is below.
__device__ __forceinline__ uint32_t to_steps(float u) {
  // 2^23 more: rounded to whole steps, which are the low bits
  constexpr float M = 8388608.f;
  return __float_as_uint(fminf(fminf(__builtin_fmaf(u, -STEPS, M), __builtin_fmaf(u, -STEPS / 4, M + 24576.f)), M + 65535.f));
}
__device__ __forceinline__ float from_steps(uint32_t q) {
  const float s = (float)q;
  return q == 65535 ? 0.f : __builtin_amdgcn_exp2f(fmaxf(s, __builtin_fmaf(s, 4.f, -98304.f)) * (-1.f / STEPS));
}

// The tile's rows (in the wave's part: 32 i + 8 (r / 4) + 4 (lane / 32) + r % 4) are vocabulary
// entries, its columns (32 j + lane % 32) tokens.
template <int R, int ST, bool TRAIN>
__global__ __launch_bounds__(NT, ST == 2 ? 2 : 1) void xent_logits_kernel(LinearXentArgs a, int first) {
  __shared__ __attribute__((aligned(1024))) bf16 smem[lds_of(R, ST)];
  constexpr int S = Tile<R>::S, W = Tile<R>::W;
  const int n = chunk_rows(a, first), total = tiles_of(R, a.V, n);
  if ((int)blockIdx.x >= total) return;
  int m0, n0;
  tile_origin<R>(a.V, n, xcd_place(blockIdx.x, total), m0, n0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int v0 = m0 + (wave >> 1) * W, t0 = n0 + (wave & 1) * W;
  const int half = 4 * (lane >> 5);
  // the sums begin at the bias; entries behind the vocabulary are -inf
  Acc<R> acc;
  const auto begin = [&](auto four) {
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx4 b = four(v0 + 32 * i + 8 * g + half);
#pragma unroll
        for (int j = 0; j < S; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] = b[e];
      }
  };
  if (v0 + W > a.V) {
    begin([&](int v) {
      floatx4 b;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = a.bias != nullptr ? a.bias[min(v + e, a.V - 1)] : 0.f;
        b[e] = v + e < a.V ? x : -INF;
      }
      return b;
    });
  } else if (a.bias != nullptr) {
    begin([&](int v) { return *reinterpret_cast<const floatx4_any*>(a.bias + v); });
  } else {
    begin([](int) { return floatx4{0.f, 0.f, 0.f, 0.f}; });
  }
  Operand<LAY_K> A = {a.w, a.ldw}, B;
  B.p = compact_x(a, B.ld);
  B.p += first * B.ld;
  tile_product<R, ST, LAY_K, LAY_K>(acc, smem, A, nullptr, B, m0, a.V, n0, n, 0, a.d, wave);

  const int pieces = cdiv(a.V, W);
  // the wave's 16 bits of its part, [32 tokens][W entries] at a time
  constexpr int QP = W / 2 + 4;
  uint32_t* st = reinterpret_cast<uint32_t*>(smem) + wave * 32 * QP;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const int t = t0 + 32 * j + (lane & 31);
    const int off = t < n ? (int)((uint32_t)a.lab[first + t] - (uint32_t)v0) : -1;  // (any label where rows are not numbered)
    if (__builtin_amdgcn_ballot_w64(off >= 0 && off < W)) {
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) z = off - half == 32 * i + 8 * (r >> 2) + (r & 3) ? acc[i][j][r] : z;
      if (off >= 0 && off < W && (off & 4) == half) a.zlab[first + t] = z;
    }
    float m = -INF;
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][j][r]);
    const auto mm = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = fmaxf(__uint_as_float(mm[0]), __uint_as_float(mm[1]));
    if (m == -INF) m = 0.f;  // no entry is left: every exp is 0
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // 0 for the largest, so that a sure row's loss is 0
          const float u = (acc[i][j][4 * g + e] - m) * LOG2E;
          s += __builtin_amdgcn_exp2f(u);
          if (TRAIN) q[e] = to_steps(u);
        }
        if (TRAIN) {
          // the low halves of two words
          const u32x2 w = {__builtin_amdgcn_perm(q[1], q[0], 0x05040100), __builtin_amdgcn_perm(q[3], q[2], 0x05040100)};
          *reinterpret_cast<u32x2*>(st + (lane & 31) * QP + (32 * i + 8 * g + half) / 2) = w;
        }
      }
    const auto ss = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
    s = __uint_as_float(ss[0]) + __uint_as_float(ss[1]);
    if (lane < 32 && t < n && v0 < a.V) a.part[(long)t * pieces + v0 / W] = make_float2(m, s);
    if constexpr (TRAIN) {
#pragma unroll
      for (int k = 0; k < W / 16; ++k) {
        const int row = 512 / W * k + lane / (W / 8), c = lane % (W / 8);
        const u32x4 w = *reinterpret_cast<const u32x4*>(st + row * QP + 4 * c);
        *reinterpret_cast<u32x4*>(a.e + (long)(t0 + 32 * j + row) * a.lde + v0 + 8 * c) = w;
      }
    }
  }
}

// A token's row on one wave: its pieces' statistics, up to 64 J of them in registers, joined to lse and loss.
struct Joined {
  float m, up, dlabel;  // what is common to all pieces, c / (sum of exp(z - m)), and the label's entry of dz
};
// f(p, q) for the lane's pieces.
template <int J, class F>
__device__ __forceinline__ void over_pieces(const float2 (&q)[J], const float2* part, int pieces, F f) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (lane + 64 * j < pieces) f(lane + 64 * j, q[j]);
  for (int p = lane + 64 * J; p < pieces; p += 64) f(p, part[p]);
}
template <int J>
__device__ __forceinline__ Joined join_row(const LinearXentArgs& a, int first, int t, int pieces, const float2* part, float2 (&q)[J]) {
  const int lane = threadIdx.x & 63;
  // (sum 0: no entry is left there)
#pragma unroll
  for (int j = 0; j < J; ++j) q[j] = lane + 64 * j < pieces ? part[lane + 64 * j] : make_float2(0.f, 0.f);
  const float zlab = a.zlab[first + t];
  const int row = a.direct ? t : a.idx[first + t];
  float top = -INF, sum = 0.f;
  over_pieces(q, part, pieces, [&](int, float2 x) { top = x.y != 0.f ? fmaxf(top, x.x) : top; });
  const float m = wave_max(top);
  over_pieces(q, part, pieces, [&](int, float2 x) { sum += x.y != 0.f ? x.y * __builtin_amdgcn_exp2f((x.x - m) * LOG2E) : 0.f; });
  const float s = wave_total(sum);
  const bool none = s == 0.f;  // every entry is -inf
  const float log_s = none ? 0.f : logf(s), z = zlab - m;
  if (lane == 0) {
    a.lse[row] = none ? -INF : m + log_s;
    a.row_loss[row] = none ? 0.f : log_s - z;
  }
  if (none) return Joined{m, 0.f, 0.f};
  const float c = a.row_weight != nullptr ? a.row_weight[row] : 1.f, up = c / s;
  return Joined{m, up, up * __builtin_amdgcn_exp2f(z * LOG2E) - c};
}
// What a piece's exp(z - its own maximum) is multiplied by to give c softmax.
__device__ __forceinline__ float piece_factor(const Joined& r, float2 q) {
  return r.up == 0.f || q.y == 0.f ? 0.f : r.up * __builtin_amdgcn_exp2f((q.x - r.m) * LOG2E);
}

// A wave a token: lse and loss, and, for the gradients, the pieces' factors and the label's entry.  Where rows are not
// numbered first, those that take no part end here.
template <bool TRAIN>
__global__ __launch_bounds__(256) void xent_join_kernel(LinearXentArgs a, int first) {
  const int n = chunk_rows(a, first), lane = threadIdx.x & 63;
  const int t = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (!TRAIN && a.direct) {
    const auto live = [&](int i) { return a.labels[i] >= 0 && a.labels[i] < a.V; };
    if (t == 0) {
      int all = 0;
      for (int i = lane; i < a.N; i += 64) all += live(i);
      all = (int)wave_total((float)all);
      if (lane == 0) a.inv_n[0] = 1.f / max(all, 1);
    }
    if (t < n && !live(t)) {
      if (lane == 0) a.row_loss[t] = a.lse[t] = 0.f;
      return;
    }
  }
  if (t >= n) return;
  const int pieces = cdiv(a.V, a.piece);
  float2* part = a.part + (long)t * pieces;
  float2 q[16];
  const Joined r = join_row(a, first, t, pieces, part, q);
  if constexpr (TRAIN) {
    over_pieces(q, part, pieces, [&](int p, float2 x) { part[p].x = piece_factor(r, x); });
    if (lane == 0) a.zlab[first + t] = r.dlabel;
  }
}

// dz of a token's eight entries from their 16-bit numbers, in place; in two parts where the chunk has few rows.
__device__ __forceinline__ void scale8(const LinearXentArgs& a, int r, int n, int v, u32x4 w, float f, int off, float dlabel,
                                       float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = from_steps(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu) * f;
    x[e] = off == e ? dlabel : x[e];
  }
  bf16x8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = f2bf(x[e]);
  *reinterpret_cast<bf16x8*>(a.e + (long)r * a.lde + v) = y;
  if (n <= BT) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = f2bf(x[e] - bf2f(y[e]));
    *reinterpret_cast<bf16x8*>(a.e2 + (long)r * a.lde + v) = y;
  }
}

// Both for a vocabulary of up to 64 pieces: a wave joins its token and scales its whole row.
__global__ __launch_bounds__(256) void xent_join_scale_kernel(LinearXentArgs a, int first) {
  const int n = chunk_rows(a, first), lane = threadIdx.x & 63;
  const int t = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= n) return;
  const int pieces = cdiv(a.V, a.piece), label = a.lab[first + t];
  float2 q[1];
  const Joined r = join_row(a, first, t, pieces, a.part + (long)t * pieces, q);
  const float f = piece_factor(r, q[0]);
  const bf16* e = a.e + (long)t * a.lde;
  for (int v0 = 0; v0 < a.V; v0 += 512) {
    const int v = v0 + 8 * lane;
    const float mine = __shfl(f, min(v, a.V - 1) / a.piece, SAT_WAVE);
    if (v >= a.V) continue;
    float x[8];
    scale8(a, t, n, v, *reinterpret_cast<const u32x4*>(e + v), mine, label - v, r.dlabel, x);
  }
}

// dz from the 16-bit numbers in place, for a.tb tokens and 2048 entries of the vocabulary: a thread has eight
// entries, of one piece, and goes from token to token.
template <bool DB>
__global__ __launch_bounds__(256) void xent_scale_kernel(LinearXentArgs a, int first) {
  const int n = chunk_rows(a, first), pieces = cdiv(a.V, a.piece), blocks = cdiv(a.V, 2048);
  const int tb = blockIdx.x / blocks, v = (blockIdx.x - tb * blocks) * 2048 + 8 * threadIdx.x;
  const int r0 = tb * a.tb, r1 = min(n, r0 + a.tb);
  if (r0 >= n || v >= a.V) return;
  const float2* part = a.part + v / a.piece;
  float db[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) db[e] = 0.f;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(a.e + (long)r * a.lde + v);
    float x[8];
    scale8(a, r, n, v, w, part[(long)r * pieces].x, a.lab[first + r] - v, a.zlab[first + r], x);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (DB) db[e] += x[e];
  }
  if (DB) store8<false>(a.dbpart + (long)tb * a.V + v, a.V - v, db);
}

// db of a chunk from its blocks of tokens, in order, added to the chunks before it: a workgroup has 64 entries, its waves
// a range of the blocks each.  (12378 x 18 x 920: 46 us with a thread for all blocks of an entry.)
constexpr int DB_WAVES = 16;
__global__ __launch_bounds__(64 * DB_WAVES) void xent_db_kernel(LinearXentArgs a, int first) {
  if (chunk_idle(a, first)) return;
  __shared__ float sums[DB_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, v = blockIdx.x * 64 + lane;
  const int blocks = cdiv(chunk_rows(a, first), a.tb), per = cdiv(blocks, DB_WAVES);
  float s = 0.f;
  if (v < a.V) {
#pragma unroll 8
    for (int b = wave * per; b < min(blocks, (wave + 1) * per); ++b) s += a.dbpart[(long)b * a.V + v];
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave > 0 || v >= a.V) return;
  for (int w = 1; w < DB_WAVES; ++w) s += sums[w][lane];
  float* f32 = reinterpret_cast<float*>(a.db);
  float* sum = a.dw_f32 ? f32 : a.dbsum;
  const float old = (a.dw_f32 ? a.accumulate : 0) || first > 0 ? sum[v] : 0.f;
  s = old + s * common_factor(a);
  if (a.dw_f32 || !chunk_last(a, first)) sum[v] = s;
  else reinterpret_cast<bf16*>(a.db)[v] = f2bf(s);
}

// ---------------------------------------------------------------- the other products

// Where a row's eight columns go: fp32 or bf16, times a factor, plus an fp32 addend.
struct RowsOut {
  void* out;
  long ld;
  bool f32;
  const float* add;  // may be out
  long ldadd;
  const int* map;    // row m is row map[m] of out
  float c;           // what the columns are multiplied by, before the addition
  __device__ __forceinline__ void put(int m, int col, float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= c;
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

// C[m, c] = sum_k (A + A2)(m, k) B(c, k) of a tile (A2 may be absent): to `o`, or, where the tile's K is split, to
// its slice's partial product [R][R] in `partial`.
template <int R, int ST, int AL>
__device__ __forceinline__ void product(bf16* smem, const Operand<AL>& A, const bf16* A2, const Operand<LAY_MN>& B, int M, int N,
                                        int K, const Split& sp, int bid, float* partial, const RowsOut& o) {
  if (bid >= sp.groups()) return;
  int tile, kb = 0, kc = K;
  float* part = nullptr;
  if (bid < sp.full) {
    tile = xcd_place(bid, sp.full);
  } else {
    const int i = xcd_place(bid - sp.full, sp.rest * sp.S), slice = i / sp.rest;
    tile = sp.full + i - slice * sp.rest;
    if (sp.S > 1) {
      kc = cdiv(cdiv(K, BK), sp.S) * BK;
      kb = slice * kc;
      kc = max(0, min(kc, K - kb));
      part = partial + (long)i * R * R;
    }
  }
  int m0, n0;
  tile_origin<R>(M, N, tile, m0, n0);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int S = Tile<R>::S, W = Tile<R>::W, EP = W + 8;
  Acc<R> acc;
#pragma unroll
  for (int i = 0; i < S; ++i)
#pragma unroll
    for (int j = 0; j < S; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  tile_product<R, ST, AL, LAY_MN>(acc, smem, A, A2, B, m0, M, n0, N, kb, kc, wave);
  float* st = reinterpret_cast<float*>(smem) + wave * 32 * EP;
  const int cl = 8 * (lane % (W / 8)), cw = (wave & 1) * W + cl;
#pragma unroll
  for (int i = 0; i < S; ++i) {
#pragma unroll
    for (int j = 0; j < S; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        st[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * EP + 32 * j + (lane & 31)] = acc[i][j][r];
#pragma unroll 2
    for (int s = 0; s < W / 16; ++s) {
      const int rl = 512 / W * s + lane / (W / 8), rw = (wave >> 1) * W + 32 * i + rl;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = st[rl * EP + cl + e];
      if (part != nullptr) store8<false>(part + rw * R + cw, 8, x);
      else if (m0 + rw < M && n0 + cw < N) o.put(m0 + rw, n0 + cw, x);
    }
  }
}

__device__ __forceinline__ RowsOut dx_out(const LinearXentArgs& a, int first) {
  return RowsOut{a.dx, a.lddx, false, nullptr, 0, a.idx + first, common_factor(a)};
}
__device__ __forceinline__ Split dx_split(int R, const LinearXentArgs& a, int n) {
  const int tiles = dx_tiles(R, a, n);
  return Split{tiles / CUS * CUS, tiles % CUS, n == a.chunk ? a.s_dx : a.meta[1]};
}
// dw of one of several chunks goes to an fp32 sum; the last one's outcome to dw.
__device__ __forceinline__ RowsOut dw_out(const LinearXentArgs& a, int first) {
  const bool sum = a.dwsum != nullptr;
  RowsOut o = {a.dw, a.lddw, a.dw_f32 != 0, nullptr, 0, nullptr, common_factor(a)};
  if (sum) {
    if (first > 0) o.add = a.dwsum, o.ldadd = a.d;
    if (!chunk_last(a, first)) o.out = a.dwsum, o.ld = a.d, o.f32 = true;
  } else if (first > 0 || a.accumulate) {
    o.add = reinterpret_cast<const float*>(a.dw);
    o.ldadd = a.lddw;
  }
  return o;
}
__device__ __forceinline__ Split dw_split(int R, const LinearXentArgs& a, int n) {
  const int tiles = dw_tiles(R, a);
  return Split{tiles / CUS * CUS, tiles % CUS, n == a.chunk ? a.s_dw : a.meta[2]};
}

template <int R, int ST>
__device__ __forceinline__ void dx_tile(const LinearXentArgs& a, int first, bf16* smem, int bid) {
  const int n = chunk_rows(a, first);
  const Operand<LAY_K> A = {a.e, a.lde};
  const Operand<LAY_MN> B = {a.w, a.ldw};
  product<R, ST, LAY_K>(smem, A, n <= BT ? a.e2 : nullptr, B, n, a.d, a.V, dx_split(R, a, n), bid, a.partial, dx_out(a, first));
}
template <int R, int ST>
__device__ __forceinline__ void dw_tile(const LinearXentArgs& a, int first, bf16* smem, int bid) {
  if (chunk_idle(a, first)) return;
  const int n = chunk_rows(a, first);
  const Operand<LAY_MN> A = {a.e, a.lde};
  Operand<LAY_MN> B;
  B.p = compact_x(a, B.ld);
  B.p += first * B.ld;
  product<R, ST, LAY_MN>(smem, A, n <= BT ? a.e2 : nullptr, B, a.V, a.d, n, dw_split(R, a, n), bid, a.partial_dw, dw_out(a, first));
}

template <int R, int ST>
__global__ __launch_bounds__(NT, ST == 2 ? 2 : 1) void xent_dx_kernel(LinearXentArgs a, int first) {
  __shared__ __attribute__((aligned(1024))) bf16 smem[lds_of(R, ST)];
  dx_tile<R, ST>(a, first, smem, blockIdx.x);
}
template <int R, int ST>
__global__ __launch_bounds__(NT, ST == 2 ? 2 : 1) void xent_dw_kernel(LinearXentArgs a, int first) {
  __shared__ __attribute__((aligned(1024))) bf16 smem[lds_of(R, ST)];
  dw_tile<R, ST>(a, first, smem, blockIdx.x);
}
// Both products at once, where each is small: the first `groups` workgroups dx, the others dw.
template <int ST>
__global__ __launch_bounds__(NT, ST == 2 ? 2 : 1) void xent_both_kernel(LinearXentArgs a, int first, int groups) {
  __shared__ __attribute__((aligned(1024))) bf16 smem[lds_of(RS, ST)];
  if ((int)blockIdx.x < groups) dx_tile<RS, ST>(a, first, smem, blockIdx.x);
  else dw_tile<RS, ST>(a, first, smem, blockIdx.x - groups);
}

// The slices of a product's split tiles added in order, 2048 elements of a tile at a time by each of `groups` workgroups.
template <bool DW>
__device__ __forceinline__ void add_slices(const LinearXentArgs& a, int first, int R, int bid, int groups) {
  const int n = chunk_rows(a, first), M = DW ? a.V : n, per = R * R / 2048;
  const Split sp = DW ? dw_split(R, a, n) : dx_split(R, a, n);
  if (sp.S == 1 || chunk_idle(a, first)) return;
  const RowsOut o = DW ? dw_out(a, first) : dx_out(a, first);
  for (int j = bid; j < per * sp.rest; j += groups) {
    const int i = j / per, e = (j % per) * 2048 + 8 * threadIdx.x;
    int m0, n0;
    if (R == BT) tile_origin<BT>(M, a.d, sp.full + i, m0, n0);
    else tile_origin<RS>(M, a.d, sp.full + i, m0, n0);
    const int m = m0 + e / R, col = n0 + e % R;
    if (m >= M || col >= a.d) continue;
    const float* p = (DW ? a.partial_dw : a.partial) + (long)i * R * R + e;
    float x[8], b[8];
    widen8(load8<false>(p, 8), x);
#pragma unroll 4
    for (int s = 1; s < sp.S; ++s) {
      widen8(load8<false>(p + (long)s * sp.rest * R * R, 8), b);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] += b[k];
    }
    o.put(m, col, x);
  }
}
// The first gx workgroups dx, the others dw.
__global__ __launch_bounds__(256) void xent_slices_kernel(LinearXentArgs a, int first, int rx, int gx, int rw) {
  if ((int)blockIdx.x < gx) add_slices<false>(a, first, rx, blockIdx.x, gx);
  else add_slices<true>(a, first, rw, blockIdx.x - gx, gridDim.x - gx);
}

constexpr int64_t kMaxE = 1LL << 29;   // numbers of a chunk
constexpr int kMaxChunk = 16384;       // tokens of a chunk
constexpr int64_t kMaxStats = 1LL << 30;  // bytes of a chunk's statistics, where they are all that is kept

struct Launch {
  int R = BT, groups = 1, split = 0;  // tile; workgroups of a product; tiles whose K is split
  int64_t partial = 0;
  void join(const Split& p) {
    groups = std::max(groups, p.groups());
    if (p.S > 1) split = std::max(split, p.rest);
    partial = std::max(partial, p.partial(R));
  }
  int slices() const { return split ? std::min(R * R / 2048 * split, 8 * CUS) : 0; }
};

// The workspace: 256-byte aligned parts, whose places go into `a` when it has a workspace.
struct Layout {
  int64_t bytes = 0;
  char* base;
  Launch logits, dx, dw;
  bool both;
  template <class T>
  void part(T*& p, int64_t n) {
    p = n > 0 ? reinterpret_cast<T*>(base + bytes) : nullptr;
    bytes += (n * (int64_t)sizeof(T) + 255) / 256 * 256;
  }
};

void plan(LinearXentArgs& a, Layout& l) {
  const bool train = a.dx || a.dw || a.db;
  const int vp = cdiv(a.V, BT) * BT;
  // Statistics are of pieces of 64 entries at least; where gradients are wanted, the numbers are the closer limit.  (A tenth
  // of it would give 16384 x 151936 x 1024, scored, three chunks of one: 4.47 -> 4.66 ms, and 4096 x 2^20 x 256 six: 3.27 -> 4.37.)
  int64_t cap = std::min<int64_t>(kMaxChunk, std::max<int64_t>(BT, kMaxStats / (8 * cdiv(a.V, RS / 2)) / BT * BT));
  if (train) cap = std::min<int64_t>(cap, std::max<int64_t>(BT, kMaxE / vp / BT * BT));
  const int chunks = std::max(1, (int)((a.N + cap - 1) / cap));
  a.chunk = std::max(1, cdiv(cdiv(a.N, chunks), BT)) * BT;
  a.lde = vp;
  // tokens of a workgroup of the scaling pass: fewer where there would be few workgroups
  a.tb = 64;
  while (a.tb > 4 && (int64_t)cdiv(a.V, 2048) * cdiv(std::min(a.N, a.chunk), a.tb) < 4 * CUS) a.tb /= 2;
  // tiles of 128 or 256 by the estimated time; a launch saved where both gradients take those of 128.  256 has the
  // larger rate (8192 x 50257 x 768: 2.26 ms, with tiles of 128 2.49), 128 the shorter ends and more tiles to share out
  // (64 x 50400 x 4096: 416 us against 522, 1024 x 1024 x 1024: 41 against 100)
  const int n = std::min(a.N, a.chunk);
  const auto cost = [](int R, int tiles, int steps, int most = SLICES) {
    int64_t ns;
    split_of(R, tiles, steps, &ns, most);
    return ns;
  };
  const auto logits = [&](int R) {  // with the exponentials, which tiles of 256 have within their 11000
    const int tiles = tiles_of(R, a.V, n);
    return cost(R, tiles, cdiv(a.d, BK), 1) + (R == RS ? tiles / CUS * 1000 : 0);
  };
  const auto dx = [&](int R) { return cost(R, dx_tiles(R, a, n), dx_steps(a)); };
  const auto dw = [&](int R) { return cost(R, dw_tiles(R, a), dw_steps(n)); };
  const int64_t x = dx(RS) - dx(BT), w = dw(RS) - dw(BT);
  const bool together = a.dx && a.dw && x + w - 8000 < std::min<int64_t>(x, 0) + std::min<int64_t>(w, 0);
  l.logits.R = logits(RS) < logits(BT) ? RS : BT;
  l.dx.R = a.rx = together || x < 0 ? RS : BT;
  l.dw.R = a.rw = together || w < 0 ? RS : BT;
  a.piece = l.logits.R / 2;
  l.part(a.meta, 64);
  l.part(a.idx, a.N);
  l.part(a.pos, a.N);
  l.part(a.lab, a.N);
  l.part(a.zlab, a.N);
  l.part(a.part, (int64_t)cdiv(a.V, a.piece) * a.chunk);
  l.part(a.xc, (int64_t)a.N * a.d);
  l.part(a.e, train ? (int64_t)a.chunk * a.lde : 0);
  l.part(a.e2, train ? (int64_t)BT * a.lde : 0);
  l.part(a.dbpart, a.db ? (int64_t)cdiv(a.chunk, a.tb) * a.V : 0);
  l.part(a.dbsum, a.db && !a.dw_f32 && a.N > a.chunk ? a.V : 0);
  l.part(a.dwsum, a.dw && !a.dw_f32 && a.N > a.chunk ? (int64_t)a.V * a.d : 0);
  // the most that any number of rows that take part asks for
  const auto split_dx = [&](int rows) { return split_of(a.rx, dx_tiles(a.rx, a, rows), dx_steps(a)); };
  const Split split_dw = split_of(a.rw, dw_tiles(a.rw, a), dw_steps(a.chunk));
  for (int i = 0; a.dx && i <= a.chunk; i += a.rx) l.dx.join(split_dx(i));
  if (a.dw) l.dw.join(split_dw);
  a.s_dx = split_dx(a.chunk).S;
  a.s_dw = split_dw.S;
  l.both = a.dx && a.dw && l.dx.R == RS && l.dw.R == RS;
  l.part(a.partial, l.both ? l.dx.partial : std::max(l.dx.partial, l.dw.partial));
  if (l.both) l.part(a.partial_dw, l.dw.partial);
  else a.partial_dw = a.partial;
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
  const int RL = l.logits.R, RX = l.dx.R, RW = l.dw.R;
  const int tiles = tiles_of(RL, a.V, a.chunk), live = tiles_of(RL, a.V, std::min(a.N, a.chunk));
  // tiles of 128: four stages where no CU has more than one (64 x 50400 x 4096: 142 us for the logits), else two and two
  // workgroups on a CU (131)
  const auto pick = [](int R, int groups, auto large, auto four, auto two) {
    return R == BT ? large : groups <= CUS ? four : two;
  };
  const auto logits = train ? pick(RL, live, xent_logits_kernel<BT, 4, true>, xent_logits_kernel<RS, 4, true>,
                                   xent_logits_kernel<RS, 2, true>)
                            : pick(RL, live, xent_logits_kernel<BT, 4, false>, xent_logits_kernel<RS, 4, false>,
                                   xent_logits_kernel<RS, 2, false>);
  const auto dx = pick(RX, l.dx.groups, xent_dx_kernel<BT, 4>, xent_dx_kernel<RS, 4>, xent_dx_kernel<RS, 2>);
  const auto dw = pick(RW, l.dw.groups, xent_dw_kernel<BT, 4>, xent_dw_kernel<RS, 4>, xent_dw_kernel<RS, 2>);
  const int groups = l.dx.groups + l.dw.groups;
  const auto both = groups <= CUS ? xent_both_kernel<4> : xent_both_kernel<2>;
  // rows of one tile that are only scored are not numbered first: each has a place in it (8 x 50257
  // x 1024, operands in turn: 30 -> 27 us)
  a.direct = !train && a.N <= RS;
  if (a.direct) {
    a.lab = const_cast<int*>(a.labels);
  } else if (a.N <= FEW) {
    hipLaunchKernelGGL(xent_rows_few_kernel, dim3(std::max(1, cdiv(a.N, 4))), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(xent_rows_kernel, dim3(1), dim3(1024), 0, s, a);
    hipLaunchKernelGGL(xent_copy_kernel, dim3(cdiv(a.N, 4)), dim3(256), 0, s, a);
  }
  // without rows, too: dw and db of none
  for (int first = 0; first < std::max(a.N, 1); first += a.chunk) {
    hipLaunchKernelGGL(logits, dim3(tiles), dim3(NT), 0, s, a, first);
    const dim3 tokens(cdiv(a.chunk, 4)), scaling(cdiv(a.V, 2048) * cdiv(a.chunk, a.tb));
    if (!train) {
      hipLaunchKernelGGL(xent_join_kernel<false>, tokens, dim3(256), 0, s, a, first);
      continue;
    }
    if (!a.db && cdiv(a.V, a.piece) <= 64) {
      hipLaunchKernelGGL(xent_join_scale_kernel, tokens, dim3(256), 0, s, a, first);
    } else {
      hipLaunchKernelGGL(xent_join_kernel<true>, tokens, dim3(256), 0, s, a, first);
      hipLaunchKernelGGL(a.db ? xent_scale_kernel<true> : xent_scale_kernel<false>, scaling, dim3(256), 0, s, a, first);
    }
    if (a.db) hipLaunchKernelGGL(xent_db_kernel, dim3(cdiv(a.V, 64)), dim3(64 * DB_WAVES), 0, s, a, first);
    const int gx = a.dx ? l.dx.slices() : 0, gw = a.dw ? l.dw.slices() : 0;
    const auto slices = [&](int x, int w) {
      if (x + w) hipLaunchKernelGGL(xent_slices_kernel, dim3(x + w), dim3(256), 0, s, a, first, RX, x, RW);
    };
    if (l.both) {
      hipLaunchKernelGGL(both, dim3(groups), dim3(NT), 0, s, a, first, l.dx.groups);
      slices(gx, gw);
      continue;
    }
    if (a.dx) {
      hipLaunchKernelGGL(dx, dim3(l.dx.groups), dim3(NT), 0, s, a, first);
      slices(gx, 0);
    }
    if (a.dw) {
      hipLaunchKernelGGL(dw, dim3(l.dw.groups), dim3(NT), 0, s, a, first);
      slices(0, gw);
    }
  }
  return hipGetLastError();
}
