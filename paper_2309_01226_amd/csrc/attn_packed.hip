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
//
// A workgroup is 2 or 4 waves of 32 rows of one sequence and head; blocks of 64 rows of the
// other operand stream through LDS (attn_tile.h).  Only blocks that some row's mask
// cuts are masked; blocks that no row sees are not read.  Rows of another sequence, and rows outside
// every sequence, read as zeros and are never written.  Heads narrower than 64, 80 or 128
// dims run in the next wider kernel with zeros behind them; 256-wide ones are in attn256.hip.
#include <algorithm>

#include "attn_packed.h"
#include "attn_tile.h"

namespace {

template <int DH, int NW, bool PAD>
__global__ __launch_bounds__(64 * NW, 2) void attn_packed_fwd_kernel(AttnPackedArgs a) {
  using C = Cfg<DH>;
  constexpr int TILE = KB * DH, WGR = NW * WR;
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * 2 * TILE];  // 2 stages x (K, V)
  const int G = a.H / a.Hkv;
  int tile, kvh, part, s0, S, qb;
  if (!packed_item(a, G, tile, kvh, part)) return;
  if (!find_rows(a, tile, WGR, a.causal, s0, S, qb)) return;
  const int h = kvh * G + part;
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
  const int jb = key_lo(a, q0) / KB, je = (key_hi(a, q0 + WGR - 1, S) + KB - 1) / KB;
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
  copy(jb);
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
  if (q < S) {
    const float inv = (st.l > 0.f) ? 1.f / st.l : 0.f;
    store_rowT<DH, PAD>(a.o + (long)(s0 + q) * a.ldo + (long)h * a.dh, st.o, inv, g, a.dh);
    if (g == 0) a.lse[(long)h * a.T + s0 + q] = (st.m + log2f(st.l)) * LN2;
  }
}

// dQ, and delta for the dK / dV kernel, which runs after it.
template <int DH, int NW, bool PAD>
__global__ __launch_bounds__(64 * NW, 2) void attn_packed_dq_kernel(AttnPackedBwdArgs ba) {
  using C = Cfg<DH>;
  constexpr int TILE = KB * DH, WGR = NW * WR;
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * 2 * TILE];  // 2 stages x (K, V)
  const AttnPackedArgs& a = ba.f;
  const int G = a.H / a.Hkv;
  int tile, kvh, part, s0, S, qb;
  if (!packed_item(a, G, tile, kvh, part)) return;
  if (!find_rows(a, tile, WGR, a.causal, s0, S, qb)) return;
  const int h = kvh * G + part;
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
    if (g == 0 && q < S) ba.delta[hs + q] = st.dlt;
  }
#pragma unroll
  for (int t = 0; t < C::OT; ++t) st.dq[t] = zero16();
  TileOfs<DH, KB> to;
  to.init(lane);
  const int jb = key_lo(a, q0) / KB, je = (key_hi(a, q0 + WGR - 1, S) + KB - 1) / KB;  // as in the forward
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
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < je) copy(j + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int kv = j * KB + 32 * u;
      if (kv < whi && kv + 32 > wlo)
        dq_sub<DH, true, true>(st, to, Ks, Ks + TILE, u, sc, hi - kv - 4 * g, lo - kv - 4 * g);
    }
    wait_vm_lgkm0<0>();
    cta_barrier();
  };
  copy(jb);
  wait_vm_lgkm0<0>();
  cta_barrier();
  int j = jb;
  for (; j < j1; ++j) masked(j);
  for (; j < j2; ++j) {
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < je) copy(j + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      dq_sub<DH, false>(st, to, Ks, Ks + TILE, u, sc, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_vm_lgkm0<0>();
    cta_barrier();
  }
  for (; j < je; ++j) masked(j);
  if (q < S) store_rowT<DH, PAD>(ba.dq + (long)(s0 + q) * ba.lddq + (long)h * a.dh, st.dq, a.scale, g, a.dh);
}

// dK and dV of one K / V head: the blocks of Q and dO of all its query heads in turn.
template <int DH, int NW, bool PAD>
__global__ __launch_bounds__(64 * NW, DH == 128 ? 1 : 2) void attn_packed_dkdv_kernel(AttnPackedBwdArgs ba) {
  using C = Cfg<DH>;
  constexpr int BQ = KB, WGR = NW * WR;
  constexpr int QT = BQ * DH;
  constexpr int STG = 2 * QT + 2 * 2 * BQ;  // Q, dO, lse2[64], delta[64]
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * STG];
  const AttnPackedArgs& a = ba.f;
  const int G = a.H / a.Hkv;
  int tile, kvh, part, s0, S, blk;
  if (!packed_item(a, 1, tile, kvh, part)) return;
  if (!find_rows(a, tile, WGR, a.causal, s0, S, blk)) return;
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
  const int total = nqb * G;  // block j of head kvh G + i is step i nqb + j
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

  fetch(0);
  wait_vm_lgkm0<0>();
  publish(0);
  wait_vm_lgkm0<0>();
  cta_barrier();

  // blocks [j1, j2) hold only valid pairs for this wave (loops of their own: a join of two
  // variants would copy the accumulators)
  const int j1 = min(max((query_lo(a, kmin + WR - 1) - q_start + BQ - 1) / BQ, 0), nqb);
  const int j2 = idle ? j1 : min(max((query_hi(a, kmin, S) - q_start) / BQ, j1), nqb);
  for (int i = 0; i < G; ++i) {
    const int i0 = i * nqb;
    int j = 0;
    for (; j < j1; ++j) masked(i0 + j, j);
    for (; j < j2; ++j) {
      const bf16* Qs = stage(i0 + j);
      const float* l2s = reinterpret_cast<const float*>(Qs + 2 * QT);
      if (i0 + j + 1 < total) fetch(i0 + j + 1);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        dkdv_sub<DH, false>(st, to, Qs, Qs + QT, l2s, l2s + BQ, u, g, sc, 0, 0);
        if (DH != 128) __builtin_amdgcn_sched_barrier(0);
      }
      next(i0 + j);
    }
    for (; j < nqb; ++j) masked(i0 + j, j);
  }
  if (key < S) {
    store_rowT<DH, PAD>(ba.dk + (long)(s0 + key) * ba.lddk + (long)kvh * a.dh, st.dk, a.scale, g, a.dh);
    store_rowT<DH, PAD>(ba.dv + (long)(s0 + key) * ba.lddv + (long)kvh * a.dh, st.dv, 1.f, g, a.dh);
  }
}

// Waves (of 32 rows) per workgroup: four share the staged blocks; two where that leaves CUs
// idle or where the sequences are mostly too short for four (the idle waves wait).
int packed_waves(const AttnPackedArgs& a, int per) {
  const long rows = a.T / std::max(1, a.n_seq);
  if ((long)(a.T / 128 + 1) * a.Hkv * per < 192 || rows < 96) return 2;
  return 4;
}

template <int DH, bool PAD>
hipError_t fwd(AttnPackedArgs a, hipStream_t s) {
  const int per = a.H / a.Hkv, nw = packed_waves(a, per);
  const dim3 grid(packed_grid(a, nw * WR, per));
  if (nw == 2) hipLaunchKernelGGL((attn_packed_fwd_kernel<DH, 2, PAD>), grid, dim3(128), 0, s, a);
  else hipLaunchKernelGGL((attn_packed_fwd_kernel<DH, 4, PAD>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int DH, bool PAD>
hipError_t bwd(AttnPackedBwdArgs a, hipStream_t s) {
  const int per = a.f.H / a.f.Hkv, nq = packed_waves(a.f, per), nk = packed_waves(a.f, 1);
  const dim3 qgrid(packed_grid(a.f, nq * WR, per));
  if (nq == 2) hipLaunchKernelGGL((attn_packed_dq_kernel<DH, 2, PAD>), qgrid, dim3(128), 0, s, a);
  else hipLaunchKernelGGL((attn_packed_dq_kernel<DH, 4, PAD>), qgrid, dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 kgrid(packed_grid(a.f, nk * WR, 1));
  if (nk == 2) hipLaunchKernelGGL((attn_packed_dkdv_kernel<DH, 2, PAD>), kgrid, dim3(128), 0, s, a);
  else hipLaunchKernelGGL((attn_packed_dkdv_kernel<DH, 4, PAD>), kgrid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_packed_fwd(const AttnPackedArgs& a, hipStream_t s) {
  if (a.T == 0 || a.n_seq == 0) return hipSuccess;
  if (a.dh > 128) return launch_attn256_packed_fwd(a, s);
  if (a.dh == 64) return fwd<64, false>(a, s);
  if (a.dh < 64) return fwd<64, true>(a, s);
  if (a.dh == 80) return fwd<80, false>(a, s);
  if (a.dh < 80) return fwd<80, true>(a, s);
  if (a.dh == 128) return fwd<128, false>(a, s);
  return fwd<128, true>(a, s);
}

hipError_t launch_attn_packed_bwd(const AttnPackedBwdArgs& a, hipStream_t s) {
  if (a.f.T == 0 || a.f.n_seq == 0) return hipSuccess;
  if (a.f.dh > 128) return launch_attn256_packed_bwd(a, s);
  if (a.f.dh == 64) return bwd<64, false>(a, s);
  if (a.f.dh < 64) return bwd<64, true>(a, s);
  if (a.f.dh == 80) return bwd<80, false>(a, s);
  if (a.f.dh < 80) return bwd<80, true>(a, s);
  if (a.f.dh == 128) return bwd<128, false>(a, s);
  return bwd<128, true>(a, s);
}
