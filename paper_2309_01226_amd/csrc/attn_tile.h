// Tiles of the attention kernels for heads of up to 128 dims: their layout in LDS, the
// copies and reads of it, and the products of one staged block (forward, dK / dV, dQ).
// attn_small.hip runs them over batches of equal rows, attn_packed.hip over packed sequences.
//
// Tile layout in LDS (R rows of a [rows][dh] bf16 block):
//  * each 64 dims (0..63; of 128-wide heads also 64..127): R rows of 128 B, eight 16-byte chunks, chunk c of row r
//    stored at c ^ swz(r).  Row-fragment reads (16 lanes = 16 consecutive
//    rows at one chunk) and transposing reads ds_read_b64_tr_b16 (32 lanes
//    = 4 consecutive rows x 4 chunks) then both touch 16 distinct 16-byte
//    bank groups per 256 bytes.
//  * dims 64..79 (80-wide heads): two chunks per row stored chunk-major,
//    [2][R] with row r of chunk t at slot r ^ 4t, after the 64-dim part.
// Products whose output rows are head dims (O^T, dV^T, dK^T, dQ^T) use
// 32-row MFMA tiles; for 80-wide heads the third tile's rows 80..95 read
// dims 64..79 again and are discarded at the store.  32- and 96-wide heads (packed sequences only) are
// staged as 64 and 128 dims, of which the products take theirs.
#pragma once

#include "common.h"
#include "kernels.h"

namespace {

constexpr int WR = 32;         // rows owned by a wave
constexpr int KB = 64;         // rows per staged block
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float RESCALE_SLACK = 8.f;
constexpr uint32_t OOB = 0x80000000u;

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

// The CDNA4 transposing LDS read through a restrict-qualified pointer: once
// inlined, the read carries alias-scope information, so the compiler does not
// make it wait for every LDS copy still in flight (the next block's, which
// land in another stage); the current stage's copies are waited for, and
// published by a barrier, before any wave reads it.
__device__ __forceinline__ bf16x4 ds_read_tr(const lds_bf16x4* __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(const_cast<lds_bf16x4*>(p));
}
__device__ __forceinline__ lds_void* lds(const bf16* p) { return (lds_void*)(const_cast<bf16*>(p)); }

template <int DH>
struct Cfg {
  static_assert(DH == 32 || DH == 64 || DH == 80 || DH == 96 || DH == 128, "32-, 64-, 80-, 96- or 128-wide heads");
  static constexpr bool TAIL = DH == 80;
  static constexpr int W = DH == 32 ? 64 : DH == 96 ? 128 : DH;  // dims of a staged row
  static constexpr int PARTS = W / 64;       // 64-dim parts of a staged tile
  static constexpr int KS = DH / 16;         // k-steps over the head dims
  static constexpr int RS = DH == 128 ? 4 : DH == 96 ? 3 : KS;  // k-steps whose row fragments are read together
  static constexpr int OT = (DH + 31) / 32;  // 32-dim output tiles
};

// chunk swizzle of the 64-dim part
__device__ __forceinline__ int swz(int r) { return (((r >> 1) & 1) << 2) | ((r >> 2) & 3); }

__device__ __forceinline__ floatx16 zero16() {
  floatx16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
// Row (within a 32 x 32 tile) held by accumulator register r of lane group g.
__device__ __forceinline__ int acc_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }
// Maximum over the two half-waves, exchanged on the vector unit (a shuffle goes
// through the LDS unit).
__device__ __forceinline__ float halves_max(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float halves_sum(float x) { return x + __shfl_xor(x, 32, 64); }

// Maximum of three.  fmaxf first quiets each operand (v_max x, x), since the
// compiler cannot know that an MFMA result is no signaling NaN; the maximum that hands
// NaN on does not, and becomes one v_maximum3.  (As inline asm the same
// instruction read its operands 2 wait states after the MFMA that writes them, which
// needs 12: the compiler keeps them apart only for instructions that it knows.)
// A NaN score leaves its query's maximum where it was; that query's sum, output and
// log-sum-exp are NaN whatever the maximum.
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const void* base, long byte_off) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)base + byte_off), (short)0, 0x7FFFFFFF,
                                           0x00020000);
}

// Copies of R rows (a block of K, V, Q or dO) into an LDS tile; rows >=
// nvalid read zero.  rs addresses row 0 of the block, rows ld elements apart.  PAD: so do
// dims >= dh (a multiple of 8), the heads being narrower than the kernel's.
template <int DH, int R, int NW, bool PAD = false>
__device__ __forceinline__ void copy_tile(__amdgpu_buffer_rsrc_t rs, long ld, int nvalid, bf16* dst,
                                          int wave, int dh = DH) {
  const int lane = threadIdx.x & 63;
  constexpr int NM = R / 8 * Cfg<DH>::PARTS;  // 1 KB instructions of the 64-dim parts
#pragma unroll
  for (int i = 0; i < (NM + NW - 1) / NW; ++i) {
    const int j = NW * i + wave;
    if (NM % NW == 0 || j < NM) {
      const int row = 8 * (j % (R / 8)) + (lane >> 3);
      const int c = 8 * (j / (R / 8)) + ((lane & 7) ^ swz(row));
      const uint32_t o = row < nvalid && (!PAD || 8 * c < dh) ? (uint32_t)(((long)row * ld + 8 * c) * 2) : OOB;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, lds(dst + j * 512), 16, o, 0, 0, 0);
    }
  }
  if constexpr (Cfg<DH>::TAIL) {
    if (wave < R / 32) {  // 2 R slots of 16 bytes
      const int slot = 64 * wave + lane;
      const int t = slot / R;
      const int row = (slot % R) ^ (4 * t);
      const uint32_t o =
          row < nvalid && (!PAD || 64 + 8 * t < dh) ? (uint32_t)(((long)row * ld + 64 + 8 * t) * 2) : OOB;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, lds(dst + R * 64 + 512 * wave), 16, o, 0, 0, 0);
    }
  }
}

// Lane-dependent LDS offsets of the two kinds of tile read.
template <int DH, int R>
struct TileOfs {
  int rf[4];   // row fragment, k-step c % 4 of a 64-dim part: row lane % 32, dims 16 c + 8 g .. + 7
  int rft;     // row fragment of k-step 4 (80-wide heads)
  int tr[2];   // transposed read, output tile ot % 2 of a 64-dim part, 16-row step 0, low half
  int trt;     // transposed read of output tile 2 (80-wide heads)
  __device__ __forceinline__ void init(int lane) {
    const int g = lane >> 5, l31 = lane & 31;
#pragma unroll
    for (int c = 0; c < 4; ++c) rf[c] = l31 * 64 + 8 * ((2 * c + g) ^ swz(l31));
    rft = R * 64 + 8 * (g * R + (l31 ^ (4 * g)));
    // lane group G = lane / 16 reads rows 4 (G >> 1) + {0..3} (lo; +8 hi) of
    // dims 32 ot + 16 (G & 1) + 0..15; lane 4 e + q: row e, dims 4 q .. 4 q + 3
    const int G = lane >> 4, ll = lane & 15;
    const int r = 4 * (G >> 1) + (ll >> 2);
#pragma unroll
    for (int ot = 0; ot < 2; ++ot) {
      const int c = 4 * ot + 2 * (G & 1) + ((ll >> 1) & 1);
      tr[ot] = r * 64 + 8 * (c ^ swz(r)) + 4 * (ll & 1);
    }
    const int t = (ll >> 1) & 1;
    trt = R * 64 + 8 * (t * R + (r ^ (4 * t))) + 4 * (ll & 1);
  }
  // Row fragment of k-step c for rows 32 u + lane % 32.
  __device__ __forceinline__ bf16x8 row(const bf16* tile, int u, int c) const {
    const int o = c < 4 * Cfg<DH>::PARTS ? rf[c & 3] + (c >> 2) * R * 64 + 32 * u * 64 : rft + 32 * u * 8;
    return *reinterpret_cast<const bf16x8*>(tile + o);
  }
  // Transposed operand (rows = head dims 32 ot + lane % 32, k = 16 tile rows
  // 16 kk .. + 15 in the accumulator permutation) of output tile ot.
  __device__ __forceinline__ bf16x8 trans(const bf16* tile, int kk, int ot) const {
    bf16x4 lo, hi;
    if (ot < 2 * Cfg<DH>::PARTS) {
      const int part = (ot >> 1) * R * 64 + 16 * kk * 64;
      const int o = tr[ot & 1];
      lo = ds_read_tr((const lds_bf16x4*)lds(tile + o + part));
      // rows + 8 flip bit 1 of swz, i.e. chunk bit 1
      hi = ds_read_tr((const lds_bf16x4*)lds(tile + (o ^ 16) + 8 * 64 + part));
    } else {
      const int o = trt + 16 * kk * 8;
      lo = ds_read_tr((const lds_bf16x4*)lds(tile + o));
      hi = ds_read_tr((const lds_bf16x4*)lds(tile + o + 8 * 8));
    }
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Row fragments (dims 16 c + 8 g .. + 7) of one row per lane, from global;
// rows >= nvalid (and, PAD, dims >= dh) read zero.
template <int DH, bool PAD = false>
__device__ __forceinline__ void load_rows(const bf16* base, long ld, int r0, int nvalid, int lane,
                                          bf16x8 (&f)[Cfg<DH>::KS], int dh = DH) {
  const __amdgpu_buffer_rsrc_t rs = rows_rsrc(base, (long)r0 * ld * 2);
  const int r = lane & 31, g = lane >> 5;
  const uint32_t o = r < nvalid ? (uint32_t)(((long)r * ld + 8 * g) * 2) : OOB;
#pragma unroll
  for (int c = 0; c < Cfg<DH>::KS; ++c)
    f[c] = __builtin_bit_cast(
        bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, !PAD || 16 * c + 8 * g < dh ? o : OOB, 32 * c, 0));
}

// Store a transposed accumulator set (rows = head dims, column = this lane's
// row) times f as bf16 into out[0 .. DH), PAD: out[0 .. dh).
template <int DH, bool PAD = false>
__device__ __forceinline__ void store_rowT(bf16* out, const floatx16 (&acc)[Cfg<DH>::OT], float f, int g, int dh = DH) {
#pragma unroll
  for (int ot = 0; ot < Cfg<DH>::OT; ++ot)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      if (32 * ot + acc_row(4 * r4, g) >= (PAD ? dh : DH)) continue;
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = f2bf(acc[ot][4 * r4 + e] * f);
      *reinterpret_cast<bf16x4*>(out + 32 * ot + acc_row(4 * r4, g)) = y;
    }
}

// ================================================================ forward
// The score tile is computed transposed, S^T = K Q^T: each lane owns one
// query (two lanes per query, 16 keys each per 32-key tile), so the running
// max and sum are per-lane scalars and the probabilities are directly the B
// operand of O^T += V^T P^T.

template <int DH>
struct FwdState {
  bf16x8 qf[Cfg<DH>::KS];
  floatx16 o[Cfg<DH>::OT];
  float m, l;  // running max (base 2, scaled, lazily raised); sum over this lane's keys
};

// One block of up to 64 keys.  MASK: some score of the block is masked (key >=
// lim, lim_rel = first excluded key of this lane's query relative to the block start
// and 4 g); two: keys 32..63 of the block hold a valid key for some query of
// the wave (always the case without MASK).  LOW: also masked are keys < low, low_rel likewise.
// PF: 16-key steps whose V fragments are read ahead of the exponentials (80-wide
// heads: one keeps three waves per SIMD, two make it two: 53 -> 60 us at 64 x 16 x 257).
template <int DH, bool MASK, bool LOW = false, int PF = DH <= 64 ? 4 : 1>
__device__ __forceinline__ void fwd_block(FwdState<DH>& st, const TileOfs<DH, KB>& to, const bf16* Ks,
                                          const bf16* Vs, float sc, bool two, int lim_rel, int low_rel = 0) {
  using C = Cfg<DH>;
  floatx16 s0 = zero16(), s1 = zero16();
#pragma unroll
  for (int c0 = 0; c0 < C::KS; c0 += C::RS) {
    bf16x8 k0[C::RS], k1[C::RS];
#pragma unroll
    for (int c = 0; c < C::RS; ++c) {
      k0[c] = to.row(Ks, 0, c0 + c);
      k1[c] = to.row(Ks, 1, c0 + c);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < C::RS; ++c) {
      s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0[c], st.qf[c0 + c], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1[c], st.qf[c0 + c], s1, 0, 0, 0);
    }
  }
  bf16x8 vf[PF ? PF : 1][C::OT];
#pragma unroll
  for (int kk = 0; kk < PF; ++kk)
#pragma unroll
    for (int ot = 0; ot < C::OT; ++ot) vf[kk][ot] = to.trans(Vs, kk, ot);
  __builtin_amdgcn_sched_barrier(0);
  float x[32];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    x[r] = s0[r];
    x[16 + r] = s1[r];
  }
  if (MASK) {
#pragma unroll
    for (int r = 0; r < 32; ++r) {
      const int kr = 32 * (r >> 4) + 8 * ((r & 15) >> 2) + (r & 3);
      x[r] = kr < lim_rel && (!LOW || kr >= low_rel) ? x[r] : -INFINITY;
    }
  }
  float mx4[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    mx4[i] = max3(x[i], x[4 + i], x[8 + i]);
    mx4[i] = max3(mx4[i], x[12 + i], x[16 + i]);
    mx4[i] = max3(mx4[i], x[20 + i], x[24 + i]);
  }
  mx4[0] = max3(mx4[0], x[28], x[29]);
  mx4[1] = max3(mx4[1], x[30], x[31]);
  const float mx = max3(mx4[0], mx4[1], max3(mx4[2], mx4[3], mx4[0]));
  const float mloc = halves_max(mx) * sc;
  const bool raise = mloc > st.m + RESCALE_SLACK;
  if (__builtin_amdgcn_ballot_w64(raise) != 0) {
    const float alpha = (raise && st.m != -INFINITY) ? __builtin_amdgcn_exp2f(st.m - mloc)
                                                     : (raise ? 0.f : 1.f);
    st.l *= alpha;
#pragma unroll
    for (int ot = 0; ot < C::OT; ++ot)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[ot][r] *= alpha;
    st.m = raise ? mloc : st.m;
  }
  const float nm = (st.m == -INFINITY) ? 0.f : -st.m;
  float lsum = 0.f;
  bf16x8 pb[4];
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    const float pr = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], sc, nm));
    lsum += pr;
    pb[r >> 3][r & 7] = f2bf(pr);
  }
  st.l += lsum;
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    if (MASK && kk >= 2 && !two) break;
#pragma unroll
    for (int ot = 0; ot < C::OT; ++ot)
      st.o[ot] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk < PF ? vf[kk < PF ? kk : 0][ot] : to.trans(Vs, kk, ot),
                                                         pb[kk], st.o[ot], 0, 0, 0);
  }
}

// ================================================================ backward, dK and dV
// Each wave owns 32 keys and holds their K and V rows in registers; 64-query
// blocks of Q and dO (with lse * log2 e and delta) stream through LDS.  Per
// 32-query sub-tile: S = Q K^T and dP = dO V^T with queries as rows (lane =
// key), P = exp2(S scale log2e - lse2), dS = P (dP - delta), then
// dV^T += dO^T P and dK^T += Q^T dS with dO^T / Q^T from transposing reads.
template <int DH>
struct DkvState {
  bf16x8 kf[Cfg<DH>::KS], vf[Cfg<DH>::KS];
  floatx16 dk[Cfg<DH>::OT], dv[Cfg<DH>::OT];
};

// Sub-tile u (32 queries) of a staged block.  MASK: query rows acc_row(r, g) are
// valid when acc_row - 4 g < lim_q and >= lim_k.
template <int DH, bool MASK>
__device__ __forceinline__ void dkdv_sub(DkvState<DH>& st, const TileOfs<DH, KB>& to, const bf16* Qs,
                                         const bf16* dOs, const float* l2s, const float* dls, int u,
                                         int g, float sc, int lim_q, int lim_k) {
  using C = Cfg<DH>;
  floatx16 x = zero16(), y = zero16();
#pragma unroll
  for (int c0 = 0; c0 < C::KS; c0 += C::RS) {
    bf16x8 k0[C::RS], k1[C::RS];
#pragma unroll
    for (int c = 0; c < C::RS; ++c) {
      k0[c] = to.row(Qs, u, c0 + c);
      k1[c] = to.row(dOs, u, c0 + c);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < C::RS; ++c) {
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0[c], st.kf[c0 + c], x, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1[c], st.vf[c0 + c], y, 0, 0, 0);
    }
  }
  bf16x8 pb[2], db[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 l4 = *reinterpret_cast<const floatx4*>(l2s + 32 * u + 8 * i + 4 * g);
    const floatx4 d4 = *reinterpret_cast<const floatx4*>(dls + 32 * u + 8 * i + 4 * g);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * i + e;
      float pr = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], sc, -l4[e]));
      if (MASK) {
        const int rr = 8 * i + e;  // acc_row - 4 g
        pr = (rr < lim_q && rr >= lim_k) ? pr : 0.f;
      }
      pb[r >> 3][r & 7] = f2bf(pr);
      db[r >> 3][r & 7] = f2bf(pr * (y[r] - d4[e]));
    }
  }
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int ot = 0; ot < C::OT; ++ot) {
      st.dv[ot] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(to.trans(dOs, 2 * u + hh, ot), pb[hh], st.dv[ot], 0, 0, 0);
      st.dk[ot] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(to.trans(Qs, 2 * u + hh, ot), db[hh], st.dk[ot], 0, 0, 0);
    }
}

// ================================================================ backward, dQ
// Each wave owns 32 queries and holds their Q and dO rows, lse2 and delta in
// registers; 64-key blocks of K and V stream through LDS.  Per 32-key
// sub-tile: S^T = K Q^T and dP^T = V dO^T (lane = query),
// dS^T = P^T (dP^T - delta), dQ^T += K^T dS^T with K^T from transposing reads.
// This kernel runs first and also computes delta = rowsum(dO * O) for the
// dK / dV kernel.
template <int DH>
struct DqState {
  bf16x8 qf[Cfg<DH>::KS], of[Cfg<DH>::KS];
  floatx16 dq[Cfg<DH>::OT];
  float nl2, dlt;  // -lse * log2 e and delta of this lane's query
  float pd;        // sum of P dP over this lane's keys (where it is taken)
};

// Sub-tile u (32 keys) of a staged block.  MASK: keys with acc_row - 4 g < lim_rel (LOW: and
// >= low_rel) are valid.  SUM: also adds P dP to st.pd; DQ: adds to dQ.
template <int DH, bool MASK, bool LOW = false, bool SUM = false, bool DQ = true>
__device__ __forceinline__ void dq_sub(DqState<DH>& st, const TileOfs<DH, KB>& to, const bf16* Ks,
                                       const bf16* Vs, int u, float sc, int lim_rel, int low_rel = 0) {
  using C = Cfg<DH>;
  floatx16 x = zero16(), y = zero16();
#pragma unroll
  for (int c0 = 0; c0 < C::KS; c0 += C::RS) {
    bf16x8 k0[C::RS], k1[C::RS];
#pragma unroll
    for (int c = 0; c < C::RS; ++c) {
      k0[c] = to.row(Ks, u, c0 + c);
      k1[c] = to.row(Vs, u, c0 + c);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < C::RS; ++c) {
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0[c], st.qf[c0 + c], x, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1[c], st.of[c0 + c], y, 0, 0, 0);
    }
  }
  bf16x8 kt[2][C::OT];
  if constexpr (DQ) {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int ot = 0; ot < C::OT; ++ot) kt[hh][ot] = to.trans(Ks, 2 * u + hh, ot);
  }
  __builtin_amdgcn_sched_barrier(0);
  bf16x8 db[2];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    float pr = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], sc, st.nl2));
    if (MASK) {
      const int kr = 8 * (r >> 2) + (r & 3);
      pr = kr < lim_rel && (!LOW || kr >= low_rel) ? pr : 0.f;
    }
    if (SUM) st.pd = __builtin_fmaf(pr, y[r], st.pd);
    if (DQ) db[r >> 3][r & 7] = f2bf(pr * (y[r] - st.dlt));
  }
  if constexpr (DQ) {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int ot = 0; ot < C::OT; ++ot)
        st.dq[ot] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kt[hh][ot], db[hh], st.dq[ot], 0, 0, 0);
  }
}

bool ok16(const void* p, long ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0; }
bool ok8(const void* p, long ld) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0 && ld % 4 == 0; }
// byte offsets of a staged block and of a wave's rows stay below 2^31
bool rows_fit(long ld) { return 128 * ld * 2 < (1L << 30); }

}  // namespace
