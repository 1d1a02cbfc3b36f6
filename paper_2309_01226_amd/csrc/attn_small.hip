// Attention forward and backward for 64-, 80- and 128-wide heads (GPT-2-style
// decoders, ViT-H/14), causal or bidirectional, on gfx950 MFMA
// (v_mfma_f32_32x32x16_bf16, bf16 operands, fp32 accumulation).
//
// Forward: O = softmax(scale * Q K^T + mask) V per head and the per-query
// natural-log log-sum-exp.  Backward: dV = P^T dO, dP = dO V^T,
// dS = P * (dP - delta), dK = scale dS^T Q, dQ = scale dS K, with P
// recomputed from the saved log-sum-exp and delta = rowsum(dO * O).
//
// Small heads make the softmax, not the matrix cores, the scarce resource:
// per score there are only 4 dh (forward) or 8 dh (backward) MFMA flops
// against one exp and a handful of vector instructions.  So these kernels
// keep the vector work per score minimal (scores are scaled inside the FMA
// that feeds exp2, the running max is raised lazily, masks are evaluated
// only on blocks that cross the diagonal or the sequence end) and keep
// several waves per SIMD so that one wave's exp overlaps another's MFMAs.
//
// They are bound by latency before either unit is full: a wave's block is a chain of LDS
// reads, MFMAs, the max, the exponentials and MFMAs again (vector unit busy a
// third, matrix cores a sixth of the cycles at 8 x 12 heads of 1024 x 64).  So the
// row fragments of a step are read together ahead of its MFMAs, whose two
// chains alternate, the transposed ones ahead of the exponentials where
// registers allow, and masked and whole blocks run in loops of their own.
// Forward / backward, before and after: 1 x 8 heads of 1359 x 64 causal 25 / 68 and
// 17.6 / 52 us; 2 x 12 of 2048 x 80 causal 45 / 128 and 37 / 104; 8 x 12 of 1024 x 64
// causal 31 / 84 and 28 / 76.
//
// 128-wide heads have twice the MFMA work per score of 64-wide ones, in twice the
// registers: the row fragments are read four k-steps at a time, and the dK/dV kernel,
// with 256 registers of operands and accumulators, runs one wave per SIMD whose two
// sub-tiles of a block the compiler overlaps instead.  Against the kernels
// that stage V and dO^T through register transposes (attention.hip), forward /
// backward: 2 x 16 heads of 2048 causal 218 / 723 and 53 / 155 us; 32 x 12 of 512
// causal 186 / 653 and 56 / 200; 7 x 16 of 1500 502 / 1617 and 151 / 517; 1 x 8 of 100
// causal 10.6 / 34 and 8.9 / 18.
//
// Workgroup = 2 to 4 waves x 32 rows (queries for the forward and dQ kernels,
// keys for the dK/dV kernel) of one (batch, head); the other operand streams
// through LDS in blocks of 64 rows, two stages, copied HBM -> LDS with
// buffer_load ... lds (no VGPR staging).
//
// The layout of a staged tile and the products of a block are in attn_tile.h.
#include <algorithm>

#include "attn_tile.h"

namespace {

// Which head and which block of its rows a workgroup takes.  Workgroups are dealt
// round-robin over the 8 XCDs, each with its own 4 MB L2.  With at least 64
// heads, each XCD takes a contiguous eighth of them, in groups whose staged
// operands (K and V, or Q and dO: 4 S dh bytes per head) fit its L2 together, and
// within a group all first (with a causal mask: heaviest) blocks, then all second
// ones.  So a head's blocks read the staged operand from HBM once, and
// neighbouring 80-wide heads, whose rows share 128-byte lines, share the L2.
// 64 x 16 heads of 257 x 80, blocks outermost over all heads: the forward read K and V
// three times (forward 79 us, backward 229), now 53 and 175.  Fewer heads are dealt out one by one.
__device__ __forceinline__ bool wg_item(int BH, int nb, int group, int& blk, int& bh) {
  const int id = blockIdx.x;
  if (BH < 64) {
    blk = id / BH;
    bh = id % BH;
    return true;
  }
  const int hx = (BH + 7) >> 3, slot = id >> 3;
  const int g = slot / (group * nb), r = slot - g * group * nb;
  const int gh = min(group, hx - g * group);
  blk = r / gh;
  bh = (id & 7) * hx + g * group + r % gh;
  return bh < BH;
}

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_small_fwd_kernel(AttnArgs a, int group) {
  using C = Cfg<DH>;
  constexpr int TILE = KB * DH, WGR = NW * WR;
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * 2 * TILE];  // 2 stages x (K, V)
  const int S = a.S;
  const int nqb = (S + WGR - 1) / WGR;
  // causal: heaviest block of every head first
  const int BH = a.B * a.H;
  int xb, bh;
  if (!wg_item(BH, nqb, group, xb, bh)) return;
  const int qb = a.causal ? (nqb - 1 - xb) : xb;
  const int b = bh / a.H, h = bh % a.H;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  const int q0 = qb * WGR, wq0 = q0 + wave * WR, q = wq0 + (lane & 31);
  const bf16* Qb = a.q + (long)b * S * a.ldq + (long)h * DH;
  const bf16* Kb = a.k + (long)b * S * a.ldk + (long)h * DH;
  const bf16* Vb = a.v + (long)b * S * a.ldv + (long)h * DH;

  FwdState<DH> st;
  load_rows<DH>(Qb, a.ldq, wq0, S - wq0, lane, st.qf);
#pragma unroll
  for (int t = 0; t < C::OT; ++t) st.o[t] = zero16();
  st.m = -INFINITY;
  st.l = 0.f;
  TileOfs<DH, KB> to;
  to.init(lane);
  const float sc = a.scale * LOG2E;
  const int kv_end = a.causal ? min(S, q0 + WGR) : S;
  const int nblk = (kv_end + KB - 1) / KB;
  // keys this wave's queries may see: [0, wk_end); this lane's: [0, lim)
  const int wk_end = wq0 >= S ? 0 : a.causal ? min(S, wq0 + WR) : S;
  const int lim = a.causal ? min(S, q + 1) : S;
  // blocks that every query of the wave sees whole; the rest run the masked variant (two
  // loops, not a branch in one: where the variants join, the accumulators
  // would be copied on every block)
  const int nfull = (wq0 >= S ? 0 : a.causal ? min(S, wq0 + 1) : S) / KB;

  auto copy = [&](int j) {
    bf16* dst = smem + (j & 1) * 2 * TILE;
    copy_tile<DH, KB, NW>(rows_rsrc(Kb, (long)j * KB * a.ldk * 2), a.ldk, S - j * KB, dst, wave);
    copy_tile<DH, KB, NW>(rows_rsrc(Vb, (long)j * KB * a.ldv * 2), a.ldv, S - j * KB, dst + TILE, wave);
  };
  copy(0);
  wait_vm_lgkm0<0>();
  cta_barrier();
  int j = 0;
  for (; j < nfull; ++j) {
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < nblk) copy(j + 1);
    fwd_block<DH, false>(st, to, Ks, Ks + TILE, sc, true, 0);
    wait_vm_lgkm0<0>();
    cta_barrier();
  }
  for (; j < nblk; ++j) {
    const int kv0 = j * KB;
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < nblk) copy(j + 1);
    if (kv0 < wk_end) fwd_block<DH, true>(st, to, Ks, Ks + TILE, sc, wk_end - kv0 > 32, lim - kv0 - 4 * g);
    wait_vm_lgkm0<0>();
    cta_barrier();
  }
  st.l = halves_sum(st.l);
  if (q < S) {
    const float inv = (st.l > 0.f) ? 1.f / st.l : 0.f;
    store_rowT<DH>(a.o + ((long)b * S + q) * a.ldo + (long)h * DH, st.o, inv, g);
    if (g == 0) a.lse[((long)b * a.H + h) * S + q] = (st.m + log2f(st.l)) * LN2;
  }
}

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, DH == 128 ? 1 : 2) void attn_small_dkdv_kernel(AttnBwdArgs a, int group) {
  using C = Cfg<DH>;
  constexpr int BQ = KB, WGR = NW * WR;
  constexpr int QT = BQ * DH;
  constexpr int STG = 2 * QT + 2 * 2 * BQ;  // Q, dO, lse2[64], delta[64]
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * STG];
  const int S = a.f.S;
  // with a causal mask the first keys see the most queries
  const int BH = a.f.B * a.f.H;
  int kblk, bh;
  if (!wg_item(BH, (S + WGR - 1) / WGR, group, kblk, bh)) return;
  const int b = bh / a.f.H, h = bh % a.f.H;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  const int k0 = kblk * WGR;
  const int kmin = k0 + wave * WR;
  const int key = kmin + (lane & 31);
  const long hs = ((long)b * a.f.H + h) * S;
  const bf16* Qb = a.f.q + (long)b * S * a.f.ldq + (long)h * DH;
  const bf16* Kb = a.f.k + (long)b * S * a.f.ldk + (long)h * DH;
  const bf16* Vb = a.f.v + (long)b * S * a.f.ldv + (long)h * DH;
  const bf16* dOb = a.dout + (long)b * S * a.lddo + (long)h * DH;
  const float sc = a.f.scale * LOG2E;

  DkvState<DH> st;
  load_rows<DH>(Kb, a.f.ldk, kmin, S - kmin, lane, st.kf);
  load_rows<DH>(Vb, a.f.ldv, kmin, S - kmin, lane, st.vf);
#pragma unroll
  for (int t = 0; t < C::OT; ++t) {
    st.dk[t] = zero16();
    st.dv[t] = zero16();
  }
  TileOfs<DH, BQ> to;
  to.init(lane);

  const int q_start = a.f.causal ? k0 : 0;
  const int nqb = (S - q_start + BQ - 1) / BQ;
  float lsd = 0.f;  // wave 0: lse of the next block's query `lane`; wave 1: its delta

  auto stage = [&](int j) { return smem + (j & 1) * STG; };
  auto fetch = [&](int j) {
    const int qs = q_start + j * BQ;
    bf16* sj = stage(j);
    copy_tile<DH, BQ, NW>(rows_rsrc(Qb, (long)qs * a.f.ldq * 2), a.f.ldq, S - qs, sj, wave);
    copy_tile<DH, BQ, NW>(rows_rsrc(dOb, (long)qs * a.lddo * 2), a.lddo, S - qs, sj + QT, wave);
    if (wave < 2) {
      const int qi = qs + lane;
      lsd = qi < S ? (wave ? a.delta[hs + qi] : a.f.lse[hs + qi]) : 0.f;
    }
  };
  auto publish = [&](int j) {
    if (wave < 2) reinterpret_cast<float*>(stage(j) + 2 * QT)[wave * BQ + lane] = wave ? lsd : lsd * LOG2E;
  };
  auto next = [&](int j) {
    if (j + 1 < nqb) {
      wait_vm_lgkm0<0>();
      publish(j + 1);
      wait_vm_lgkm0<0>();
      cta_barrier();
    }
  };
  // the masked variant of a block: sub-tiles without a valid pair are skipped
  auto masked = [&](int j) {
    const bf16* Qs = stage(j);
    const float* l2s = reinterpret_cast<const float*>(Qs + 2 * QT);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int qs = q_start + j * BQ + 32 * u;
      if (kmin >= S || qs >= S || (a.f.causal && qs + 31 < kmin)) continue;
      dkdv_sub<DH, true>(st, to, Qs, Qs + QT, l2s, l2s + BQ, u, g, sc, S - qs - 4 * g,
                         a.f.causal ? key - qs - 4 * g : -(1 << 30));
    }
  };

  fetch(0);
  wait_vm_lgkm0<0>();
  publish(0);
  wait_vm_lgkm0<0>();
  cta_barrier();

  // blocks [j1, j2) hold only valid pairs for this wave: past the diagonal, short of S
  // (loops of their own: a join of two variants would copy the accumulators)
  const int j1 = a.f.causal ? min(nqb, (kmin + 31 - q_start + BQ - 1) / BQ) : 0;
  const int j2 = kmin >= S ? j1 : max(j1, (S - q_start) / BQ);
  int j = 0;
  for (; j < j1; ++j) {
    if (j + 1 < nqb) fetch(j + 1);
    masked(j);
    next(j);
  }
  for (; j < j2; ++j) {
    const bf16* Qs = stage(j);
    const float* l2s = reinterpret_cast<const float*>(Qs + 2 * QT);
    if (j + 1 < nqb) fetch(j + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) { dkdv_sub<DH, false>(st, to, Qs, Qs + QT, l2s, l2s + BQ, u, g, sc, 0, 0); if (DH != 128) __builtin_amdgcn_sched_barrier(0); }
    next(j);
  }
  for (; j < nqb; ++j) {
    if (j + 1 < nqb) fetch(j + 1);
    masked(j);
    next(j);
  }
  if (key < S) {
    store_rowT<DH>(a.dk + ((long)b * S + key) * a.lddk + (long)h * DH, st.dk, a.f.scale, g);
    store_rowT<DH>(a.dv + ((long)b * S + key) * a.lddv + (long)h * DH, st.dv, 1.f, g);
  }
}

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_small_dq_kernel(AttnBwdArgs a, int group) {
  using C = Cfg<DH>;
  constexpr int TILE = KB * DH, WGR = NW * WR;
  __shared__ __attribute__((aligned(1024))) bf16 smem[2 * 2 * TILE];  // 2 stages x (K, V)
  const int S = a.f.S;
  const int nqb = (S + WGR - 1) / WGR;
  const int BH = a.f.B * a.f.H;
  int xb, bh;
  if (!wg_item(BH, nqb, group, xb, bh)) return;
  const int qb = a.f.causal ? (nqb - 1 - xb) : xb;
  const int b = bh / a.f.H, h = bh % a.f.H;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  const int q0 = qb * WGR, wq0 = q0 + wave * WR, q = wq0 + (lane & 31);
  const long hs = ((long)b * a.f.H + h) * S;
  const bf16* Qb = a.f.q + (long)b * S * a.f.ldq + (long)h * DH;
  const bf16* Kb = a.f.k + (long)b * S * a.f.ldk + (long)h * DH;
  const bf16* Vb = a.f.v + (long)b * S * a.f.ldv + (long)h * DH;
  const bf16* dOb = a.dout + (long)b * S * a.lddo + (long)h * DH;
  const float sc = a.f.scale * LOG2E;

  DqState<DH> st;
  load_rows<DH>(Qb, a.f.ldq, wq0, S - wq0, lane, st.qf);
  load_rows<DH>(dOb, a.lddo, wq0, S - wq0, lane, st.of);
  st.nl2 = q < S ? -a.f.lse[hs + q] * LOG2E : 0.f;
  // delta = rowsum(dO * O) of this lane's query, from the two halves of its row
  {
    bf16x8 ov[C::KS];
    load_rows<DH>(a.f.o + (long)b * S * a.f.ldo + (long)h * DH, a.f.ldo, wq0, S - wq0, lane, ov);
    float acc = 0.f;
#pragma unroll
    for (int c = 0; c < C::KS; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc = __builtin_fmaf(bf2f(st.of[c][e]), bf2f(ov[c][e]), acc);
    st.dlt = halves_sum(acc);
    if (g == 0 && q < S) a.delta[hs + q] = st.dlt;
  }
#pragma unroll
  for (int t = 0; t < C::OT; ++t) st.dq[t] = zero16();
  TileOfs<DH, KB> to;
  to.init(lane);

  const int kv_end = a.f.causal ? min(S, q0 + WGR) : S;
  const int nkb = (kv_end + KB - 1) / KB;
  const int wk_end = wq0 >= S ? 0 : a.f.causal ? min(S, wq0 + WR) : S;
  const int lim = a.f.causal ? min(S, q + 1) : S;
  const int nfull = (wq0 >= S ? 0 : a.f.causal ? min(S, wq0 + 1) : S) / KB;  // as in the forward

  auto copy = [&](int j) {
    bf16* dst = smem + (j & 1) * 2 * TILE;
    copy_tile<DH, KB, NW>(rows_rsrc(Kb, (long)j * KB * a.f.ldk * 2), a.f.ldk, S - j * KB, dst, wave);
    copy_tile<DH, KB, NW>(rows_rsrc(Vb, (long)j * KB * a.f.ldv * 2), a.f.ldv, S - j * KB, dst + TILE, wave);
  };
  copy(0);
  wait_vm_lgkm0<0>();
  cta_barrier();
  int j = 0;
  for (; j < nfull; ++j) {
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < nkb) copy(j + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) { dq_sub<DH, false>(st, to, Ks, Ks + TILE, u, sc, 0); __builtin_amdgcn_sched_barrier(0); }
    wait_vm_lgkm0<0>();
    cta_barrier();
  }
  for (; j < nkb; ++j) {
    const bf16* Ks = smem + (j & 1) * 2 * TILE;
    if (j + 1 < nkb) copy(j + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int kv = j * KB + 32 * u;
      if (kv < wk_end) dq_sub<DH, true>(st, to, Ks, Ks + TILE, u, sc, lim - kv - 4 * g);
    }
    wait_vm_lgkm0<0>();
    cta_barrier();
  }
  if (q < S) store_rowT<DH>(a.dq + ((long)b * S + q) * a.lddq + (long)h * DH, st.dq, a.f.scale, g);
}

// Staged operand bytes of the heads an XCD works on at a time, of its 4 MB L2.
// Causal blocks differ in work: a larger group balances them better (96 heads of
// 1024 x 64, 3 MB per XCD: forward 28 us as one group, 33 us as 10 + 2 heads).
inline long l2_group(bool causal) { return causal ? 9L << 19 : 3L << 19; }

// Waves (of 32 rows) per workgroup.  Four, which share the staged blocks of the
// other operand; fewer where that leaves wave slots or CUs idle: in the forward
// three when the rows then fill the last workgroup better (257 rows are 9 wave
// tiles: three workgroups either way, of 9 waves instead of 12; 64 x 16 heads 58 ->
// 56 us; the backward, at two waves per SIMD either way, took 185 -> 196), two
// when four give fewer than 192 workgroups.
int waves_per_wg(int S, long BH, bool fwd) {
  const int tiles = (S + WR - 1) / WR;
  if ((long)((tiles + 3) / 4) * BH < 192) return 2;
  return fwd && (tiles + 2) / 3 * 3 < (tiles + 3) / 4 * 4 ? 3 : 4;
}

}  // namespace

bool attn_small_fwd_eligible(const AttnArgs& a) {
  return (a.dh == 64 || a.dh == 80 || a.dh == 128) && a.scale > 0.f && ok16(a.q, a.ldq) && ok16(a.k, a.ldk) && ok16(a.v, a.ldv) &&
         ok8(a.o, a.ldo) && rows_fit(a.ldq) && rows_fit(a.ldk) && rows_fit(a.ldv);
}

bool attn_small_bwd_eligible(const AttnBwdArgs& a) {
  return attn_small_fwd_eligible(a.f) && ok16(a.dout, a.lddo) && rows_fit(a.lddo) && ok16(a.f.o, a.f.ldo) &&
         rows_fit(a.f.ldo) && a.delta != nullptr && ok8(a.dq, a.lddq) &&
         ok8(a.dk, a.lddk) && ok8(a.dv, a.lddv);
}

// One kernel of a head width: `three` also instantiates it for three waves (the forward).
#define SMALL_LAUNCH(KERNEL, DH, args, f, three)                                                   \
  do {                                                                                             \
    const int BH_ = (f).B * (f).H, hx_ = (BH_ + 7) / 8;                                            \
    const int nw_ = waves_per_wg((f).S, BH_, three);                                               \
    const long nb_ = sat_cdiv((f).S, nw_ * WR);                                                    \
    const int group_ =                                                                             \
        (int)std::max(1L, std::min((long)hx_, l2_group((f).causal) / (4L * (f).S * DH)));          \
    const dim3 grid_((unsigned)(nb_ * (BH_ < 64 ? BH_ : 8 * hx_)));                                \
    if (nw_ == 2) hipLaunchKernelGGL((KERNEL<DH, 2>), grid_, dim3(128), 0, s, args, group_);       \
    else if (three && nw_ == 3) hipLaunchKernelGGL((KERNEL<DH, three ? 3 : 4>), grid_, dim3(192), 0, s, args, group_); \
    else hipLaunchKernelGGL((KERNEL<DH, 4>), grid_, dim3(256), 0, s, args, group_);                \
  } while (0)

hipError_t launch_attn_small_fwd(const AttnArgs& a, hipStream_t s) {
  if (a.dh == 64) SMALL_LAUNCH(attn_small_fwd_kernel, 64, a, a, true);
  else if (a.dh == 80) SMALL_LAUNCH(attn_small_fwd_kernel, 80, a, a, true);
  else SMALL_LAUNCH(attn_small_fwd_kernel, 128, a, a, true);
  return hipGetLastError();
}

// dQ (which also writes delta), then dK / dV.
hipError_t launch_attn_small_bwd(const AttnBwdArgs& a, hipStream_t s) {
  if (a.f.dh == 64) SMALL_LAUNCH(attn_small_dq_kernel, 64, a, a.f, false);
  else if (a.f.dh == 80) SMALL_LAUNCH(attn_small_dq_kernel, 80, a, a.f, false);
  else SMALL_LAUNCH(attn_small_dq_kernel, 128, a, a.f, false);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.f.dh == 64) SMALL_LAUNCH(attn_small_dkdv_kernel, 64, a, a.f, false);
  else if (a.f.dh == 80) SMALL_LAUNCH(attn_small_dkdv_kernel, 80, a, a.f, false);
  else SMALL_LAUNCH(attn_small_dkdv_kernel, 128, a, a.f, false);
  return hipGetLastError();
}
