// Attention inside packed sequences, forward and backward, on gfx950 MFMA.
//
// Rows cu[s] .. cu[s + 1] - 1 of q, k, v are sequence s; query head h reads K / V head
// h / (H / Hkv).  Query i sees key j of its own sequence when j <= i (causal) and
// |i - j| < window.
//   x = scale q k^T;  lse = log sum exp x;  p = exp(x - lse);  o = p v
//   delta = rowsum(dO * O);  dV = sum over the heads of p^T dO;  dS = p (dO V^T - delta)
//   dQ = scale dS K;  dK = sum over the heads of scale dS^T Q
// p is recomputed from lse in the backward.  Products take bf16 operands (p and dS rounded to
// nearest, at most 2^-8 of the value) and sum in fp32, as do the softmax's statistics, delta and the
// sums over heads; the results are rounded once.  No atomics: every result has one order of sums.
// Where the blocks are too few for the chip a block's steps are split among workgroups, whose fp32 partial
// results a second kernel joins in their order.
//
// A workgroup is 2 or 4 waves of 32 rows of one sequence and head; blocks of 64 rows of the
// other operand stream through LDS (attn_tile.h).  Only blocks that some row's mask
// cuts are masked; blocks that no row sees are not read.  Rows of another sequence, and rows outside
// every sequence, read as zeros and are never written.  Heads narrower than 32, 64, 80, 96 or 128
// dims run in the next wider kernel with zeros behind them; 256-wide ones are in attn256.hip.  (In the kernels of 64 and
// 128 dims, 4 x 4096 rows of 16 heads take forward 268 us and backward 837 for 32 dims, 476 and 1655 for 96; in
// their own 221 and 630, 426 and 1461.)
//
// Bounds and times: 64- and 80-wide heads by a wave's chain of LDS reads, products and exponentials (an exponential and
// about ten other instructions a pair against 4 dh flop: vector unit busy half, matrix cores a quarter to a third of the
// cycles on these documents), 128-wide ones by the same chain, with the matrix cores busy in 0.43 to 0.54 of the
// cycles and the clock at 1.8 to 2.1 GHz of 2.4 meanwhile (the large matrix product: 1.4 PFLOP/s).  Forward, dQ, dK / dV of
//   32 documents of 16 to 2048 rows in 16384, 16 heads of 64, causal       77, 100, 131 us (forward 450 TFLOP/s)
//   64 images of 65 to 577 rows in 16448, 16 heads of 80, no mask          72, 102, 123 us
//   4 documents in 16001 rows, 16 heads of 128 on 4 K / V heads, causal    299, 404, 663 us (forward 1.0 PFLOP/s; the
//     backward executes 7 products for the 5 counted: 1.0 PFLOP/s executed)
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_packed.h"
#include "attn_tile.h"

namespace {

// 80-wide heads of four waves are held to the registers of three waves on a SIMD (one value spilled before the
// loop): 50 images, 16 heads, 61.4 -> 56.5 us; 4 x 4096 rows causal 246 -> 235.  64-wide ones have three anyway, and
// four would spill in the loop (30 -> 35 us on 16 short documents).
template <int DH, int NW, bool PAD>
__global__ __launch_bounds__(64 * NW, DH == 80 && NW == 4 ? 3 : 2) void attn_packed_fwd_kernel(AttnPackedArgs a) {
  using C = Cfg<DH>;
  constexpr int TILE = KB * C::W, WGR = NW * WR;
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * 2 * TILE];  // 2 stages x (K, V)
  const int G = a.H / a.Hkv;
  int tile, kvh, part, s0, S, qb;
  if (!packed_item(a, G * a.split, tile, kvh, part)) return;
  if (!find_rows(a, tile, WGR, s0, S, qb)) return;
  const int sp = part % a.split, h = kvh * G + part / a.split;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  const int q0 = qb * WGR, wq0 = q0 + wave * WR, q = wq0 + (lane & 31);
  const bf16* Qb = a.q + (long)s0 * a.ldq + (long)h * a.dh;
  const bf16* Kb = a.k + (long)s0 * a.ldk + (long)kvh * a.dh;
  const bf16* Vb = a.v + (long)s0 * a.ldv + (long)kvh * a.dh;

  FwdState<DH> st;
  load_rows<DH, PAD>(Qb, a.ldq, wq0, S - wq0, lane, st.qf, a.dh);
#pragma unroll
  for (int t = 0; t < C::OT; ++t) st.o[t] = zero16();
  st.m = -INFINITY;
  st.l = 0.f;
  TileOfs<DH, KB> to;
  to.init(lane);
  const float sc = a.scale * LOG2E;
  // blocks of the workgroup [jb, je), those that every query of the wave sees whole [j1, j2),
  // keys that some query of the wave sees [wlo, whi), those of this lane's [lo, hi)
  int jb = key_lo(a, q0) / KB, je = (key_hi(a, q0 + WGR - 1, S) + KB - 1) / KB;
  part_of(sp, a.split, jb, je);
  const bool idle = wq0 >= S;
  const int wlo = key_lo(a, wq0), whi = idle ? 0 : key_hi(a, wq0 + WR - 1, S);
  const int lo = key_lo(a, q), hi = key_hi(a, q, S);
  const int j1 = min(max((key_lo(a, wq0 + WR - 1) + KB - 1) / KB, jb), je);
  const int j2 = idle ? j1 : min(max(key_hi(a, wq0, S) / KB, j1), je);

  auto copy = [&](int j) {
    bf16* dst = smem + (j & 1) * 2 * TILE;
    copy_tile<DH, KB, NW, PAD>(rows_rsrc(Kb, (long)j * KB * a.ldk * 2), a.ldk, S - j * KB, dst, wave, a.dh);
    copy_tile<DH, KB, NW, PAD>(rows_rsrc(Vb, (long)j * KB * a.ldv * 2), a.ldv, S - j * KB, dst + TILE, wave, a.dh);
  };
  auto masked = [&](int j) {
    const int kv0 = j * KB;
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < je) copy(j + 1);
    if (kv0 < whi && kv0 + KB > wlo)
      fwd_block<DH, true, true>(st, to, Ks, Ks + TILE, sc, whi - kv0 > 32, hi - kv0 - 4 * g, lo - kv0 - 4 * g);
    wait_vm_lgkm0<0>();
    cta_barrier();
  };
  if (jb < je) copy(jb);  // a part may be empty
  wait_vm_lgkm0<0>();
  cta_barrier();
  int j = jb;
  for (; j < j1; ++j) masked(j);
  for (; j < j2; ++j) {
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < je) copy(j + 1);
    fwd_block<DH, false>(st, to, Ks, Ks + TILE, sc, true, 0);
    wait_vm_lgkm0<0>();
    cta_barrier();
  }
  for (; j < je; ++j) masked(j);
  st.l = halves_sum(st.l);
  if (a.split > 1) {
    float* p = wave_share(a.ws, ((long)tile * a.H + h) * a.split + sp, NW, 16 * C::OT + 4, wave);
    put_acc<C::OT>(p, st.o);
    *reinterpret_cast<floatx2*>(p + 16 * C::OT * 64) = floatx2{st.m, st.l};
    return;
  }
  if (q < S) {
    const float inv = (st.l > 0.f) ? 1.f / st.l : 0.f;
    store_rowT<DH, PAD>(a.o + (long)(s0 + q) * a.ldo + (long)h * a.dh, st.o, inv, g, a.dh);
    if (g == 0) a.lse[(long)h * a.T + s0 + q] = (st.m + log2f(st.l)) * LN2;
  }
}

// dQ, and delta for the dK / dV kernel, which runs after it.
// delta = rowsum(dO * O) comes from the rounded O, which is off by 2^-8 of it where a query sees few keys and
// O is as large as V.  The same sum over the keys, sum P dP, has no such error: it is formed beside dQ (a
// multiply-add per pair) for the dK / dV kernel and, where all keys of the workgroup fit the two stages, in a pass
// of its own before dQ.  Gradients of 24 rows: 0.27 % -> 0.24 % off, of which 0.17 % is the results' rounding.
// A part of a split block has a part of the sum, which the join adds; blocks that fit the stages stay whole, in the
// first part.
template <int DH, int NW, bool PAD>
__global__ __launch_bounds__(64 * NW, 2) void attn_packed_dq_kernel(AttnPackedBwdArgs ba) {
  using C = Cfg<DH>;
  constexpr int TILE = KB * C::W, WGR = NW * WR;
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * 2 * TILE];  // 2 stages x (K, V)
  const AttnPackedArgs& a = ba.f;
  const int G = a.H / a.Hkv;
  int tile, kvh, part, s0, S, qb;
  if (!packed_item(a, G * a.split, tile, kvh, part)) return;
  if (!find_rows(a, tile, WGR, s0, S, qb)) return;
  const int sp = part % a.split, h = kvh * G + part / a.split;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  const int q0 = qb * WGR, wq0 = q0 + wave * WR, q = wq0 + (lane & 31);
  const long hs = (long)h * a.T + s0;
  const bf16* Kb = a.k + (long)s0 * a.ldk + (long)kvh * a.dh;
  const bf16* Vb = a.v + (long)s0 * a.ldv + (long)kvh * a.dh;
  const float sc = a.scale * LOG2E;

  DqState<DH> st;
  load_rows<DH, PAD>(a.q + (long)s0 * a.ldq + (long)h * a.dh, a.ldq, wq0, S - wq0, lane, st.qf, a.dh);
  load_rows<DH, PAD>(ba.dout + (long)s0 * ba.lddo + (long)h * a.dh, ba.lddo, wq0, S - wq0, lane, st.of, a.dh);
  st.nl2 = q < S ? -a.lse[hs + q] * LOG2E : 0.f;
  {
    bf16x8 ov[C::KS];
    load_rows<DH, PAD>(a.o + (long)s0 * a.ldo + (long)h * a.dh, a.ldo, wq0, S - wq0, lane, ov, a.dh);
    float acc = 0.f;
#pragma unroll
    for (int c = 0; c < C::KS; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc = __builtin_fmaf(bf2f(st.of[c][e]), bf2f(ov[c][e]), acc);
    st.dlt = halves_sum(acc);
  }
  st.pd = 0.f;
#pragma unroll
  for (int t = 0; t < C::OT; ++t) st.dq[t] = zero16();
  TileOfs<DH, KB> to;
  to.init(lane);
  int jb = key_lo(a, q0) / KB, je = (key_hi(a, q0 + WGR - 1, S) + KB - 1) / KB;  // as in the forward
  const bool brief = je - jb <= 2;
  if (!brief) part_of(sp, a.split, jb, je);
  else if (sp > 0) je = jb;
  const bool idle = wq0 >= S;
  const int wlo = key_lo(a, wq0), whi = idle ? 0 : key_hi(a, wq0 + WR - 1, S);
  const int lo = key_lo(a, q), hi = key_hi(a, q, S);
  const int j1 = min(max((key_lo(a, wq0 + WR - 1) + KB - 1) / KB, jb), je);
  const int j2 = idle ? j1 : min(max(key_hi(a, wq0, S) / KB, j1), je);

  auto copy = [&](int j) {
    bf16* dst = smem + (j & 1) * 2 * TILE;
    copy_tile<DH, KB, NW, PAD>(rows_rsrc(Kb, (long)j * KB * a.ldk * 2), a.ldk, S - j * KB, dst, wave, a.dh);
    copy_tile<DH, KB, NW, PAD>(rows_rsrc(Vb, (long)j * KB * a.ldv * 2), a.ldv, S - j * KB, dst + TILE, wave, a.dh);
  };
  // the pairs of block j that the mask leaves
  auto masked = [&](int j, auto sum, auto dq) {
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int kv = j * KB + 32 * u;
      if (kv < whi && kv + 32 > wlo)
        dq_sub<DH, true, true, decltype(sum)::value, decltype(dq)::value>(st, to, Ks, Ks + TILE, u, sc, hi - kv - 4 * g,
                                                                        lo - kv - 4 * g);
    }
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (jb < je) copy(jb);  // a part may be empty
  if (brief) {
    if (je - jb == 2) copy(jb + 1);
    wait_vm_lgkm0<0>();
    cta_barrier();
    for (int j = jb; j < je; ++j) masked(j, Yes(), No());
    st.dlt = st.pd = halves_sum(st.pd);
    for (int j = jb; j < je; ++j) masked(j, No(), Yes());
  } else {
    auto step = [&](int j) {
      if (j + 1 < je) copy(j + 1);
      masked(j, Yes(), Yes());
      wait_vm_lgkm0<0>();
      cta_barrier();
    };
    wait_vm_lgkm0<0>();
    cta_barrier();
    int j = jb;
    for (; j < j1; ++j) step(j);
    for (; j < j2; ++j) {
      const bf16* Ks = smem + (j & 1) * 2 * TILE;
      if (j + 1 < je) copy(j + 1);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        dq_sub<DH, false, false, true>(st, to, Ks, Ks + TILE, u, sc, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      wait_vm_lgkm0<0>();
      cta_barrier();
    }
    for (; j < je; ++j) step(j);
    st.pd = halves_sum(st.pd);
  }
  if (a.split > 1) {
    float* p = wave_share(a.ws, ((long)tile * a.H + h) * a.split + sp, NW, 16 * C::OT + 4, wave);
    put_acc<C::OT>(p, st.dq);
    p[16 * C::OT * 64] = st.pd;
    return;
  }
  if (q < S) {
    if (g == 0) ba.delta[hs + q] = st.pd;
    store_rowT<DH, PAD>(ba.dq + (long)(s0 + q) * ba.lddq + (long)h * a.dh, st.dq, a.scale, g, a.dh);
  }
}

// ================================================================ dK and dV
// dK and dV of one K / V head, up to 80-wide: the blocks of Q and dO of all its query heads in turn.
template <int DH, int NW, bool PAD>
__global__ __launch_bounds__(64 * NW, 2) void attn_packed_dkdv_kernel(AttnPackedBwdArgs ba) {
  using C = Cfg<DH>;
  constexpr int BQ = KB, WGR = NW * WR;
  constexpr int QT = BQ * C::W;
  constexpr int STG = 2 * QT + 2 * 2 * BQ;  // Q, dO, lse2[64], delta[64]
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * STG];
  const AttnPackedArgs& a = ba.f;
  const int G = a.H / a.Hkv;
  int tile, kvh, part, s0, S, blk;
  if (!packed_item(a, a.split, tile, kvh, part)) return;
  if (!find_rows(a, tile, WGR, s0, S, blk)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  // causal: the first keys see the most queries, so the places count from the end
  const int k0 = (a.causal ? (S + WGR - 1) / WGR - 1 - blk : blk) * WGR;
  const int kmin = k0 + wave * WR;
  const int key = kmin + (lane & 31);
  const float sc = a.scale * LOG2E;

  DkvState<DH> st;
  load_rows<DH, PAD>(a.k + (long)s0 * a.ldk + (long)kvh * a.dh, a.ldk, kmin, S - kmin, lane, st.kf, a.dh);
  load_rows<DH, PAD>(a.v + (long)s0 * a.ldv + (long)kvh * a.dh, a.ldv, kmin, S - kmin, lane, st.vf, a.dh);
#pragma unroll
  for (int t = 0; t < C::OT; ++t) {
    st.dk[t] = zero16();
    st.dv[t] = zero16();
  }
  TileOfs<DH, BQ> to;
  to.init(lane);

  const int q_start = query_lo(a, k0);
  const int nqb = (query_hi(a, k0 + WGR - 1, S) - q_start + BQ - 1) / BQ;
  int first = 0, total = nqb * G;  // block j of head kvh G + i is step i nqb + j
  part_of(part, a.split, first, total);
  float lsd = 0.f;            // wave 0: lse of the next block's query `lane`; wave 1: its delta

  auto stage = [&](int it) { return smem + (it & 1) * STG; };
  auto fetch = [&](int it) {
    const int i = it / nqb, qs = q_start + (it - i * nqb) * BQ;
    const int h = kvh * G + i;
    bf16* sj = stage(it);
    copy_tile<DH, BQ, NW, PAD>(rows_rsrc(a.q + (long)(s0 + qs) * a.ldq + (long)h * a.dh, 0), a.ldq, S - qs, sj, wave, a.dh);
    copy_tile<DH, BQ, NW, PAD>(rows_rsrc(ba.dout + (long)(s0 + qs) * ba.lddo + (long)h * a.dh, 0), ba.lddo, S - qs, sj + QT,
                               wave, a.dh);
    if (wave < 2) {
      const int qi = qs + lane;
      const long at = (long)h * a.T + s0 + qi;
      lsd = qi < S ? (wave ? ba.delta[at] : a.lse[at]) : 0.f;
    }
  };
  auto publish = [&](int it) {
    if (wave < 2) reinterpret_cast<float*>(stage(it) + 2 * QT)[wave * BQ + lane] = wave ? lsd : lsd * LOG2E;
  };
  auto next = [&](int it) {
    if (it + 1 < total) {
      wait_vm_lgkm0<0>();
      publish(it + 1);
      wait_vm_lgkm0<0>();
      cta_barrier();
    }
  };
  const bool idle = kmin >= S;
  // queries that some key of the wave sees [wlo, whi), those of this lane's key [lo, hi)
  const int wlo = query_lo(a, kmin), whi = idle ? 0 : query_hi(a, kmin + WR - 1, S);
  const int lo = query_lo(a, key), hi = query_hi(a, key, S);
  // the masked variant of a block: sub-tiles without a valid pair are skipped
  auto masked = [&](int it, int j) {
    const bf16* Qs = stage(it);
    const float* l2s = reinterpret_cast<const float*>(Qs + 2 * QT);
    if (it + 1 < total) fetch(it + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int qs = q_start + j * BQ + 32 * u;
      if (qs < whi && qs + 32 > wlo)
        dkdv_sub<DH, true>(st, to, Qs, Qs + QT, l2s, l2s + BQ, u, g, sc, hi - qs - 4 * g, lo - qs - 4 * g);
    }
    next(it);
  };

  if (first < total) {
    fetch(first);
    wait_vm_lgkm0<0>();
    publish(first);
  }
  wait_vm_lgkm0<0>();
  cta_barrier();

  // blocks [j1, j2) hold only valid pairs for this wave (loops of their own: a join of two
  // variants would copy the accumulators)
  const int j1 = min(max((query_lo(a, kmin + WR - 1) - q_start + BQ - 1) / BQ, 0), nqb);
  const int j2 = idle ? j1 : min(max((query_hi(a, kmin, S) - q_start) / BQ, j1), nqb);
  for (int it = first; it < total;) {  // head by head
    const int i0 = it / nqb * nqb, end = min(total - i0, nqb);
    int j = it - i0;
    for (; j < min(j1, end); ++j) masked(i0 + j, j);
    for (; j < min(j2, end); ++j) {
      const bf16* Qs = stage(i0 + j);
      const float* l2s = reinterpret_cast<const float*>(Qs + 2 * QT);
      if (i0 + j + 1 < total) fetch(i0 + j + 1);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        dkdv_sub<DH, false>(st, to, Qs, Qs + QT, l2s, l2s + BQ, u, g, sc, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      next(i0 + j);
    }
    for (; j < end; ++j) masked(i0 + j, j);
    it = i0 + end;
  }
  if (a.split > 1) {
    float* p = wave_share(a.ws, ((long)tile * a.Hkv + kvh) * a.split + part, NW, 2 * 16 * C::OT, wave);
    put_acc<C::OT>(p, st.dk);
    put_acc<C::OT>(p + 16 * C::OT * 64, st.dv);
    return;
  }
  if (key < S) {
    store_rowT<DH, PAD>(ba.dk + (long)(s0 + key) * ba.lddk + (long)kvh * a.dh, st.dk, a.scale, g, a.dh);
    store_rowT<DH, PAD>(ba.dv + (long)(s0 + key) * ba.lddv + (long)kvh * a.dh, st.dv, 1.f, g, a.dh);
  }
}

// 96- and 128-wide heads.  A wave owns 32 keys and takes 32 queries (a slot) at a time: S = Q K^T and dP = dO V^T with
// queries as rows (lane = key), P = exp2(S scale log2e - lse2), dS = P (dP - delta), then dV^T += dO^T P and
// dK^T += Q^T dS.  Its 256 registers of operands and accumulators leave room for one wave on a SIMD, which
// has to keep the matrix cores busy alone: the products S and dP of the next slot are issued between the
// exponentials of the current one, and their subtractions between the products dV and dK, in an order
// that scheduling barriers pin.  4 x 4096 rows, 16 heads, no mask: 1055 us against 1140 with the step that
// the narrower heads take, whose two waves on a SIMD fill each other's gaps (64: 580 against 570).
struct Slot {
  float t[16], u[16];  // S scale log2e - lse2 and dP - delta
};

// NEXT: the slot of rows Qn, dOn, half un of a block, with its lse2 ln and delta dn, into `nx`.  CUR: `cur`, of
// rows Qc, dOc, half uc, into dV and dK.
template <int DH, bool NEXT, bool CUR>
__device__ __forceinline__ void dkdv_step(DkvState<DH>& st, const TileOfs<DH, KB>& to, const Slot& cur, Slot& nx, const bf16* Qn,
                                          const float* ln, int un, const bf16* Qc, int uc, int g, float sc) {
  constexpr int KS = Cfg<DH>::KS, OT = Cfg<DH>::OT, QT = KB * Cfg<DH>::W;
  constexpr int PFR = 3, PFT = 3;  // k-steps, pairs of transposed fragments in flight
  bf16x8 qr[PFR + 1], dr[PFR + 1], qt[PFT + 1], dt[PFT + 1], pb[2], db[2];
  floatx16 x, y;
  auto rows = [&](int c) {
    qr[c % (PFR + 1)] = to.row(Qn, un, c);
    dr[c % (PFR + 1)] = to.row(Qn + QT, un, c);
  };
  auto cols = [&](int i) {
    dt[i % (PFT + 1)] = to.trans(Qc + QT, 2 * uc + i / OT, i % OT);
    qt[i % (PFT + 1)] = to.trans(Qc, 2 * uc + i / OT, i % OT);
  };
  if constexpr (NEXT) {
#pragma unroll
    for (int c = 0; c < PFR; ++c) rows(c);
    x = zero16();
    y = zero16();
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int c = 0; c < KS; ++c) {
    if constexpr (NEXT) {
      if (c + PFR < KS) rows(c + PFR);
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qr[c % (PFR + 1)], st.kf[c], x, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dr[c % (PFR + 1)], st.vf[c], y, 0, 0, 0);
    }
    if constexpr (CUR) {
      if (c >= KS - PFT) cols(c - (KS - PFT));
#pragma unroll
      for (int r = 16 * c / KS; r < 16 * (c + 1) / KS; ++r) {
        const float pr = __builtin_amdgcn_exp2f(cur.t[r]);
        pb[r >> 3][r & 7] = f2bf(pr);
        db[r >> 3][r & 7] = f2bf(pr * cur.u[r]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  floatx4 l4[4], d4[4];
  if constexpr (NEXT) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      l4[i] = *reinterpret_cast<const floatx4*>(ln + 32 * un + 8 * i + 4 * g);
      d4[i] = *reinterpret_cast<const floatx4*>(ln + KB + 32 * un + 8 * i + 4 * g);
    }
  }
  constexpr int NP = 2 * OT;  // pairs of products; one goes ahead of the first look at x and y
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    if constexpr (CUR) {
      const int hh = i / OT, ot = i % OT;
      if (i + PFT < NP) cols(i + PFT);
      st.dv[ot] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dt[i % (PFT + 1)], pb[hh], st.dv[ot], 0, 0, 0);
      st.dk[ot] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qt[i % (PFT + 1)], db[hh], st.dk[ot], 0, 0, 0);
    }
    if constexpr (NEXT) {
      if (i >= 1) {
#pragma unroll
        for (int r = 16 * (i - 1) / (NP - 1); r < 16 * i / (NP - 1); ++r) {
          nx.t[r] = __builtin_fmaf(x[r], sc, -l4[r >> 2][r & 3]);
          nx.u[r] = y[r] - d4[r >> 2][r & 3];
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <int DH, bool PAD>
__global__ __launch_bounds__(256, 1) void attn_packed_dkdv_wide_kernel(AttnPackedBwdArgs ba) {
  constexpr int NW = 4;
  using C = Cfg<DH>;
  constexpr int BQ = KB, WGR = NW * WR, NS = 3;  // stages: a block, the next, whose first slot is begun with it, and one on its way
  constexpr int QT = BQ * C::W;
  constexpr int STG = 2 * QT + 2 * 2 * BQ;  // Q, dO, lse2[64], delta[64]
  __shared__ __attribute__((aligned(1024))) bf16 smem[NS * STG];
  const AttnPackedArgs& a = ba.f;
  const int G = a.H / a.Hkv;
  int tile, kvh, part, s0, S, blk;
  if (!packed_item(a, a.split, tile, kvh, part)) return;
  if (!find_rows(a, tile, WGR, s0, S, blk)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  // causal: the first keys see the most queries, so the places count from the end
  const int k0 = (a.causal ? (S + WGR - 1) / WGR - 1 - blk : blk) * WGR;
  const int kmin = k0 + wave * WR;
  const int key = kmin + (lane & 31);
  const float sc = a.scale * LOG2E;

  DkvState<DH> st;
  load_rows<DH, PAD>(a.k + (long)s0 * a.ldk + (long)kvh * a.dh, a.ldk, kmin, S - kmin, lane, st.kf, a.dh);
  load_rows<DH, PAD>(a.v + (long)s0 * a.ldv + (long)kvh * a.dh, a.ldv, kmin, S - kmin, lane, st.vf, a.dh);
#pragma unroll
  for (int t = 0; t < C::OT; ++t) {
    st.dk[t] = zero16();
    st.dv[t] = zero16();
  }
  TileOfs<DH, BQ> to;
  to.init(lane);

  const int q_start = query_lo(a, k0);
  const int nqb = (query_hi(a, k0 + WGR - 1, S) - q_start + BQ - 1) / BQ;
  int first = 0, total = nqb * G;  // block j of head kvh G + i is step i nqb + j
  part_of(part, a.split, first, total);
  float lsd = 0.f;            // wave 0: lse of the next block's query `lane`; wave 1: its delta

  auto stage = [&](int it) { return smem + it % NS * STG; };
  auto fetch = [&](int it) {
    if (it >= total) return;
    const int i = it / nqb, qs = q_start + (it - i * nqb) * BQ;
    const int h = kvh * G + i;
    bf16* sj = stage(it);
    copy_tile<DH, BQ, NW, PAD>(rows_rsrc(a.q + (long)(s0 + qs) * a.ldq + (long)h * a.dh, 0), a.ldq, S - qs, sj, wave, a.dh);
    copy_tile<DH, BQ, NW, PAD>(rows_rsrc(ba.dout + (long)(s0 + qs) * ba.lddo + (long)h * a.dh, 0), ba.lddo, S - qs, sj + QT,
                               wave, a.dh);
    if (wave < 2) {
      const int qi = qs + lane;
      const long at = (long)h * a.T + s0 + qi;
      lsd = qi < S ? (wave ? ba.delta[at] : a.lse[at]) : 0.f;
    }
  };
  auto publish = [&](int it) {
    if (wave < 2) reinterpret_cast<float*>(stage(it) + 2 * QT)[wave * BQ + lane] = wave ? lsd : lsd * LOG2E;
  };
  // before block `it`: the next one lands too, and the one after it is fetched over the block before
  // `it`, which every wave has left
  auto middle = [&](int it) {
    wait_vm_lgkm0<0>();
    if (it + 1 < total) publish(it + 1);
    wait_vm_lgkm0<0>();
    cta_barrier();
    fetch(it + 2);
  };
  const bool idle = kmin >= S;
  // queries that some key of the wave sees [wlo, whi), those of this lane's key [lo, hi)
  const int wlo = query_lo(a, kmin), whi = idle ? wlo : query_hi(a, kmin + WR - 1, S);
  const int lo = query_lo(a, key), hi = query_hi(a, key, S);
  // blocks of a head that hold a valid pair for this wave
  const int ja = max(wlo - q_start, 0) / BQ, jb = idle ? 0 : (whi - q_start + BQ - 1) / BQ;
  // queries that all keys of the wave see
  const int flo = query_lo(a, kmin + WR - 1), fhi = query_hi(a, kmin, S);

  fetch(first);
  wait_vm_lgkm0<0>();
  if (first < total) publish(first);
  wait_vm_lgkm0<0>();
  cta_barrier();
  fetch(first + 1);

  auto lse2 = [&](const bf16* st_) { return reinterpret_cast<const float*>(st_ + 2 * QT); };
  // blocks of a head whose pairs are all valid for this wave
  const int fa = (max(flo - q_start, 0) + BQ - 1) / BQ, fb = (fhi - q_start) / BQ;
  Slot A, B;
  int it = first, i0 = 0;
  // one block: its two slots, and the products of the next block's first one, which go unused behind
  // this wave's last block
  auto block = [&](auto whole) {
    middle(it);
    const bf16* Qc = stage(it);
    const bf16* Qn = stage(it + 1);
    auto mask = [&](Slot& p, int u) {  // exp2 makes closed pairs 0
      const int qs = q_start + (it - i0) * BQ + 32 * u + 4 * g;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int q = qs + 8 * (r >> 2) + (r & 3);
        p.t[r] = q >= lo && q < hi ? p.t[r] : -INFINITY;
      }
    };
    if (!decltype(whole)::value) mask(A, 0);
    dkdv_step<DH, true, true>(st, to, A, B, Qc, lse2(Qc), 1, Qc, 0, g, sc);
    if (!decltype(whole)::value) mask(B, 1);
    dkdv_step<DH, true, true>(st, to, B, A, Qn, lse2(Qn), 0, Qc, 1, g, sc);
    ++it;
  };
  while (it < total) {  // head by head: its blocks before this wave's, this wave's, those behind
    i0 = it / nqb * nqb;
    const int end = min(total, i0 + nqb);
    const int from = min(max(it, i0 + ja), end), until = min(max(from, i0 + jb), end);
    for (; it < from; ++it) middle(it);
    if (it < until) dkdv_step<DH, true, false>(st, to, B, A, stage(it), lse2(stage(it)), 0, stage(it), 0, g, sc);
    const int w0 = min(max(it, i0 + fa), until), w1 = min(max(w0, i0 + fb), until);
    while (it < w0) block(std::false_type{});
    while (it < w1) block(std::true_type{});
    while (it < until) block(std::false_type{});
    for (; it < end; ++it) middle(it);
  }
  if (a.split > 1) {
    float* p = wave_share(a.ws, ((long)tile * a.Hkv + kvh) * a.split + part, NW, 2 * 16 * C::OT, wave);
    put_acc<C::OT>(p, st.dk);
    put_acc<C::OT>(p + 16 * C::OT * 64, st.dv);
    return;
  }
  if (key < S) {
    store_rowT<DH, PAD>(ba.dk + (long)(s0 + key) * ba.lddk + (long)kvh * a.dh, st.dk, a.scale, g, a.dh);
    store_rowT<DH, PAD>(ba.dv + (long)(s0 + key) * ba.lddv + (long)kvh * a.dh, st.dv, 1.f, g, a.dh);
  }
}

// ================================================================ parts
// A workgroup joins 32 dims of a block: a lane's values of all parts are independent loads, so that the time is one
// way to memory and not one for each part (one wave for all dims took 106 us for dK and dV of 2048 rows of 80 in 16
// parts, this 6).  ot: 32-dim tiles of the kernel's head in the scratch, of which the first (dh + 31) / 32 are taken.

// O and lse of a split forward: each part's o and l under the common maximum.
template <int NW>
__global__ __launch_bounds__(64 * NW) void attn_packed_join_kernel(AttnPackedArgs a, int ot) {
  const int G = a.H / a.Hkv, nt = (a.dh + 31) / 32;
  int tile, kvh, part, s0, S, qb;
  if (!packed_item(a, G * nt, tile, kvh, part)) return;
  if (!find_rows(a, tile, NW * WR, s0, S, qb)) return;
  const int h = kvh * G + part / nt, t = part % nt;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q = qb * NW * WR + wave * WR + (lane & 31);
  const int regs = 16 * ot + 4;
  const long step = (long)NW * regs * 64;  // from part to part
  const float* p = wave_share(a.ws, ((long)tile * a.H + h) * a.split, NW, regs, wave);
  const float* ml = p + 16 * ot * 64;
  p += 16 * t * 64;
  float m = -INFINITY, l = 0.f;
#pragma unroll 4
  for (int sp = 0; sp < a.split; ++sp) m = fmaxf(m, ml[sp * step]);
  floatx4 o[4] = {};
#pragma unroll 4
  for (int sp = 0; sp < a.split; ++sp) {
    const floatx2 x = *reinterpret_cast<const floatx2*>(ml + sp * step);
    // a part without keys for this query: nothing.  A NaN l stays.
    const float f = x[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[0] - m);
    l = __builtin_fmaf(x[1], f, l);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const floatx4 y = *reinterpret_cast<const floatx4*>(p + sp * step + i * 256);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = __builtin_fmaf(y[e], f, o[i][e]);
    }
  }
  if (q < S) {
    store_tile(a.o + (long)(s0 + q) * a.ldo + (long)h * a.dh, o, t, (l > 0.f) ? 1.f / l : 0.f, lane >> 5, a.dh);
    if (t == 0 && lane < 32) a.lse[(long)h * a.T + s0 + q] = (m + log2f(l)) * LN2;
  }
}

// dQ, or (KV) dK and dV, of split blocks: the parts' sum in their order.  With dQ of up to 128 dims also delta (the
// 256-wide kernel has written it: its delta is that of the rounded O).
template <int NW, bool KV>
__global__ __launch_bounds__(64 * NW) void attn_packed_add_kernel(AttnPackedBwdArgs ba, int ot) {
  const AttnPackedArgs& a = ba.f;
  const int G = a.H / a.Hkv, nt = (a.dh + 31) / 32;
  int tile, kvh, part, s0, S, blk;
  if (!packed_item(a, (KV ? 2 : G) * nt, tile, kvh, part)) return;
  if (!find_rows(a, tile, NW * WR, s0, S, blk)) return;
  if (KV && a.causal) blk = (S + NW * WR - 1) / (NW * WR) - 1 - blk;
  const int t = part % nt, which = part / nt, h = KV ? kvh : kvh * G + which;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blk * NW * WR + wave * WR + (lane & 31);
  const bool sums = !KV && ot <= 4;
  const int regs = (KV ? 2 : 1) * 16 * ot + (sums ? 4 : 0);
  const long step = (long)NW * regs * 64;  // from part to part
  const float* p = wave_share(a.ws, ((long)tile * (KV ? a.Hkv : a.H) + h) * a.split, NW, regs, wave);
  if (sums && t == 0) {
    const float* pd = p + 16 * ot * 64;
    float sum = 0.f;
#pragma unroll 4
    for (int sp = 0; sp < a.split; ++sp) sum += pd[sp * step];
    if (row < S && lane < 32) ba.delta[(long)h * a.T + s0 + row] = sum;
  }
  p += 16 * ((KV ? which * ot : 0) + t) * 64;
  floatx4 acc[4] = {};
#pragma unroll 4
  for (int sp = 0; sp < a.split; ++sp)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const floatx4 x = *reinterpret_cast<const floatx4*>(p + sp * step + i * 256);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][e] += x[e];
    }
  bf16* out = !KV ? ba.dq + (long)(s0 + row) * ba.lddq
              : which ? ba.dv + (long)(s0 + row) * ba.lddv : ba.dk + (long)(s0 + row) * ba.lddk;
  if (row < S) store_tile(out + (long)h * a.dh, acc, t, KV && which ? 1.f : a.scale, lane >> 5, a.dh);
}

// Launch shape of one kernel: waves per workgroup, parts of a block's work, scratch.
struct Plan {
  int nw, split;
  long ws;
};
enum Pass { FWD, DQ, DKDV };

// Width of the kernel that heads of dh dims run in.
int width(int dh) { return dh <= 32 ? 32 : dh <= 64 ? 64 : dh <= 80 ? 80 : dh <= 96 ? 96 : dh <= 128 ? 128 : 256; }

// Waves (of 32 rows): four share the staged blocks; two where that leaves CUs idle or where the
// sequences are mostly too short for four (the idle waves wait).
// Parts of a block's steps (64 keys; of dK / dV, 64 queries of each head):
//  * As many as let all blocks fill the CUs.  Blocks of equal work (no causal mask, or a window) in one round of
//    workgroups at most, since a second one would be as long; a causal mask's unequal ones to the nearest round, and
//    where a CU holds one workgroup to the next.
//  * A part keeps at least 4 steps of a long block, of dK / dV (more products a step) and of 256-wide dQ 2, and the
//    parts save at least what the join's launch takes, 8 steps of a 64-wide forward.
//  * The host does not know the lengths: sequences without a causal mask (images) are taken to be alike, those with one
//    (documents) to differ, the long ones T / n_seq^(2/3) rows.  8 documents in 8000 rows, 4 heads of 64, forward
//    and backward 47 and 138 us by the mean, 38 and 104 so; 8 of 1500 rows each 25 and 72, 30 and 75.
//  * A causal mask without a window makes the longest block of dK / dV the last to end, twice the mean for one
//    sequence, more for several lengths: up to four rounds, of 32 steps at least.
// Forward and backward without parts and with, us: 2048 rows, 4 heads of 128, 45 and 114, 24 and 63; 8192 rows, one
// head of 256, 249 and 880, 82 and 264; documents of 700 and 300 rows, 8 heads of 64 on 2, backward 77 and 31; 4 documents
// in 15992 rows, 16 heads of 64 on 4, backward 965 and 710.
Plan plan(const AttnPackedArgs& a, Pass pass) {
  const int G = a.H / a.Hkv, per = pass == DKDV ? 1 : G;
  const long rows = a.T / std::max(1, a.n_seq);
  Plan p;
  const int dh = width(a.dh);
  p.nw = (long)(a.T / 128 + 1) * a.Hkv * per < 192 || rows < (pass == FWD ? 96 : 160) ? 2 : 4;
  if (dh == 256 || (dh >= 96 && pass == DKDV)) p.nw = 4;  // 256: 128 rows, in the backward by eight waves
  const int R = p.nw * WR;
  const bool tail = a.causal && a.window >= a.T;
  // a sequence shorter than a block is one all the same: else parts and their scratch, which is sized for
  // T / R + n_seq blocks, would go by far fewer blocks than there are (4096 sequences in 16384 rows, 8 heads
  // of 128 on one: 1.1 GB and 1431 us forward and backward, so none and 1097)
  const long items = std::max(a.T / R + 1L, (long)a.n_seq) * a.Hkv * per;
  const int on_cu = dh == 256 || (dh >= 96 && pass == DKDV) ? 1 : dh == 32 ? (pass == DKDV ? 3 : 4)
                    : pass != DKDV && (dh == 64 || (dh == 80 && pass == FWD)) ? 3 : 2;
  const long slots = 256L * (4 / p.nw) * on_cu;  // workgroups that the CUs hold
  const long longer = a.causal ? (long)(a.T / cbrt((double)std::max(1, a.n_seq) * std::max(1, a.n_seq))) : rows;
  const long steps = std::min(longer, 2L * a.window) / KB * (pass == DKDV ? G : 1) / (a.causal ? 2 : 1);
  const long least = pass == DKDV || (dh == 256 && pass == DQ) ? 2 : 4;
  const long spare = !tail ? 0 : on_cu == 1 ? items - 1 : items / 2;  // to the round below, above, the nearest
  p.split = (int)std::min(16L, std::max(1L, std::min((slots + spare) / items, steps / least)));
  const long products = pass == FWD ? 2 : pass == DQ ? 3 : 4;  // of a step
  if (steps * (p.split - 1) * products * std::max(dh, 64) < 1024 * p.split) p.split = 1;  // 32: the exponentials' time
  if (pass == DKDV && tail) p.split = (int)std::min(16L, std::max((long)p.split, std::min(4 * slots / items, steps / 32)));
  const int ot = (dh + 31) / 32;
  // of a lane in the scratch: accumulators, and m and l, or (up to 128 dims) the sum of P dP
  const int regs = pass == DKDV ? 32 * ot : 16 * ot + (pass == FWD || dh <= 128 ? 4 : 0);
  p.ws = p.split == 1 ? 0 : (a.T / R + a.n_seq) * (long)a.Hkv * per * p.split * p.nw * regs * 64;
  return p;
}
// The plan that the scratch allows.
Plan plan_in(const AttnPackedArgs& a, Pass pass) {
  Plan p = plan(a, pass);
  if (p.ws > a.ws_elems) p.split = 1;
  return p;
}

// Launches the two-wave or the four-wave instance of a kernel.
#define PACKED_LAUNCH(NW_, GRID, ...)                                                                        \
  do {                                                                                                       \
    if ((NW_) == 2) hipLaunchKernelGGL((__VA_ARGS__(2)), GRID, dim3(128), 0, s, a);                          \
    else hipLaunchKernelGGL((__VA_ARGS__(4)), GRID, dim3(256), 0, s, a);                                     \
    const hipError_t e_ = hipGetLastError();                                                                 \
    if (e_ != hipSuccess) return e_;                                                                         \
  } while (0)

template <int DH, bool PAD>
hipError_t fwd(AttnPackedArgs a, hipStream_t s) {
#define FWD_K(NW) attn_packed_fwd_kernel<DH, NW, PAD>
  const int per = a.H / a.Hkv;
  const Plan p = plan_in(a, FWD);
  a.split = p.split;
  PACKED_LAUNCH(p.nw, dim3(packed_grid(a, p.nw * WR, per * p.split, false)), FWD_K);
  return p.split > 1 ? launch_attn_packed_join(a, p.nw, s) : hipSuccess;
}

template <int DH, bool PAD>
hipError_t bwd(AttnPackedBwdArgs a, hipStream_t s) {
#define DQ_K(NW) attn_packed_dq_kernel<DH, NW, PAD>
#define DKDV_K(NW) attn_packed_dkdv_kernel<DH, NW, PAD>
  const int per = a.f.H / a.f.Hkv;
  Plan p = plan_in(a.f, DQ);
  a.f.split = p.split;
  PACKED_LAUNCH(p.nw, dim3(packed_grid(a.f, p.nw * WR, per * p.split, false)), DQ_K);
  if (p.split > 1) {
    const hipError_t e = launch_attn_packed_add(a, p.nw, false, s);
    if (e != hipSuccess) return e;
  }
  p = plan_in(a.f, DKDV);
  a.f.split = p.split;
  const dim3 grid(packed_grid(a.f, p.nw * WR, p.split, true));
  if constexpr (DH >= 96) {
    hipLaunchKernelGGL((attn_packed_dkdv_wide_kernel<DH, PAD>), grid, dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  } else {
    PACKED_LAUNCH(p.nw, grid, DKDV_K);
  }
  return p.split > 1 ? launch_attn_packed_add(a, p.nw, true, s) : hipSuccess;
}

}  // namespace

hipError_t launch_attn_packed_join(const AttnPackedArgs& args, int nw, hipStream_t s) {
  AttnPackedArgs a = args;
  const int ot = (width(a.dh) + 31) / 32;
  const dim3 grid(packed_grid(a, nw * WR, a.H / a.Hkv * ((a.dh + 31) / 32), false));
  if (nw == 2) hipLaunchKernelGGL(attn_packed_join_kernel<2>, grid, dim3(128), 0, s, a, ot);
  else hipLaunchKernelGGL(attn_packed_join_kernel<4>, grid, dim3(256), 0, s, a, ot);
  return hipGetLastError();
}

hipError_t launch_attn_packed_add(const AttnPackedBwdArgs& args, int nw, bool kv, hipStream_t s) {
  AttnPackedBwdArgs a = args;
  const int ot = (width(a.f.dh) + 31) / 32;
  const dim3 grid(packed_grid(a.f, nw * WR, (kv ? 2 : a.f.H / a.f.Hkv) * ((a.f.dh + 31) / 32), kv));
  if (kv && nw == 2) hipLaunchKernelGGL((attn_packed_add_kernel<2, true>), grid, dim3(128), 0, s, a, ot);
  else if (kv) hipLaunchKernelGGL((attn_packed_add_kernel<4, true>), grid, dim3(256), 0, s, a, ot);
  else if (nw == 2) hipLaunchKernelGGL((attn_packed_add_kernel<2, false>), grid, dim3(128), 0, s, a, ot);
  else hipLaunchKernelGGL((attn_packed_add_kernel<4, false>), grid, dim3(256), 0, s, a, ot);
  return hipGetLastError();
}

long attn_packed_ws(const AttnPackedArgs& a, bool backward) {
  if (a.T == 0 || a.n_seq == 0) return 0;
  return backward ? std::max(plan(a, DQ).ws, plan(a, DKDV).ws) : plan(a, FWD).ws;
}

hipError_t launch_attn_packed_fwd(const AttnPackedArgs& a, hipStream_t s) {
  if (a.T == 0 || a.n_seq == 0) return hipSuccess;
  if (a.dh > 128) return launch_attn256_packed_fwd(a, plan_in(a, FWD).split, s);
  if (a.dh <= 32) return fwd<32, true>(a, s);
  if (a.dh == 64) return fwd<64, false>(a, s);
  if (a.dh < 64) return fwd<64, true>(a, s);
  if (a.dh == 80) return fwd<80, false>(a, s);
  if (a.dh < 80) return fwd<80, true>(a, s);
  if (a.dh <= 96) return fwd<96, true>(a, s);
  if (a.dh == 128) return fwd<128, false>(a, s);
  return fwd<128, true>(a, s);
}

hipError_t launch_attn_packed_bwd(const AttnPackedBwdArgs& a, hipStream_t s) {
  if (a.f.T == 0 || a.f.n_seq == 0) return hipSuccess;
  if (a.f.dh > 128) return launch_attn256_packed_bwd(a, plan_in(a.f, DQ).split, plan_in(a.f, DKDV).split, s);
  if (a.f.dh <= 32) return bwd<32, true>(a, s);
  if (a.f.dh == 64) return bwd<64, false>(a, s);
  if (a.f.dh < 64) return bwd<64, true>(a, s);
  if (a.f.dh == 80) return bwd<80, false>(a, s);
  if (a.f.dh < 80) return bwd<80, true>(a, s);
  if (a.f.dh <= 96) return bwd<96, true>(a, s);
  if (a.f.dh == 128) return bwd<128, false>(a, s);
  return bwd<128, true>(a, s);
}
