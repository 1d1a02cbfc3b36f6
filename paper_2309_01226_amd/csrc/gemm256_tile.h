// The 256 x 256 tile of the bf16 products: how its operands come from memory to LDS and from there to the
// matrix cores, and the loop over K, for gemm256.hip (the products of a step's layers) and linear_xent.hip (the
// head with its cross entropy).  Why it is laid out as it is, and what it measures, stands at the top of
// gemm256.hip, whose kernel has the same loop in its body: with the loop in a function the compiler places the waits of
// the first k-step otherwise, and a GPT-J-shaped step took 0.3% longer.
#pragma once

#include "common.h"
#include "kernels.h"

namespace {

constexpr int BT = 256;               // tile rows and columns
constexpr int NT = 256;               // 4 wavefronts, 2 x 2
constexpr uint32_t OOB = 0x80000000u; // buffer offset past num_records: reads zero

typedef __attribute__((address_space(3))) void lds_void;

// Chunk swizzle of the K-contiguous tile layout (eight 16-byte chunks per row)
__device__ __forceinline__ int swz_k(int row) { return (row >> 1) & 7; }

__device__ __forceinline__ lds_void* lds(const bf16* p) { return (lds_void*)(const_cast<bf16*>(p)); }

constexpr int BK = 64;                // K-tile depth
constexpr int OPE = BT * BK;          // bf16 elements of one operand tile

// Copies of one K-contiguous operand tile: 32 instructions of 1 KB, eight per
// wave.  Instruction j = 4 i + wave fills LDS bytes [1024 j, 1024 j + 1024) of
// the tile (rows 8 j .. 8 j + 7); lane L writes the 16 bytes at 1024 j + 16 L.
// A copy whose k lies at or past K (the K tail, and the tiles past the last
// one that the steady-state loop issues to keep its wait counts constant)
// reads zeros and touches no memory.

// M/N-contiguous operands lie [64 k][256 rows] (512 bytes per k-row) and are read
// with the transposing LDS read; chunk c (of 32) of k-row k is stored at c ^ 4 (k % 4), so
// that the 4 k-rows x 4 chunks that 32 lanes read at once are on distinct banks.

// R: rows of the tile (256, or 128 for the smaller tile below, with rows of 256 bytes where they are 512 here).
template <int LAY, int R = BT>
struct Loader {
  static constexpr int NI = (R * BK * 2 / 1024) / 4;  // copy instructions per wave
  uint32_t off[NI];  // byte offsets relative to (tile row 0, k0)
  int kof[NI];       // k of this lane's chunk relative to k0
  __device__ __forceinline__ void init(long ld, int nrows, int wave) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (LAY == LAY_K) {
        const int row = 8 * (4 * i + wave) + lane / 8;
        const int c = (lane % 8) ^ swz_k(row);
        off[i] = row < nrows ? (uint32_t)(((long)row * ld + 8 * c) * 2) : OOB;
        kof[i] = 8 * c;
      } else {
        constexpr int C = R / 8;  // chunks of a k-row
        const int k = 64 / C * (4 * i + wave) + lane / C;
        const int row = 8 * ((lane % C) ^ (4 * (k & 3)));
        off[i] = row < nrows ? (uint32_t)(((long)k * ld + row) * 2) : OOB;
        kof[i] = k;
      }
    }
  }
  // rs: the operand at (tile row 0, k = 0) when K-contiguous, else at (tile row 0,
  // k = k0): whole columns of k-rows may span more than a 32-bit offset.
  template <int I0 = 0, int I1 = NI>
  __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, int k0, int K, bf16* dst,
                                        int wave) const {
    const uint32_t so = LAY == LAY_K ? (uint32_t)(k0 * 2) : 0u;
#pragma unroll
    for (int i = I0; i < I1; ++i) {
      const uint32_t o = (k0 + kof[i] < K) ? off[i] : OOB;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, lds(dst + (4 * i + wave) * 512), 16, o, so, 0, 0);
    }
  }
};

// The transposing LDS read through a restrict-qualified pointer: its alias-scope
// information keeps the compiler from making it wait for the LDS copies in flight,
// which land in other slots.
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
__device__ __forceinline__ bf16x4 ds_read_tr(const lds_bf16x4* __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(const_cast<lds_bf16x4*>(p));
}

// Fragment addressing of one operand inside a slot, for the wave's half of the rows
// (or columns), from `w0` (0 or R / 2) on.  read(sub, ks) is the 32 x 16 MFMA operand
// of rows w0 + 32 sub .. + 31, k = 16 ks .. + 15.
template <int LAY, int R = BT>
struct Frags {
  static constexpr int KS = LAY == LAY_K ? BK / 16 : 1;
  int o[KS];  // element offsets (K-contiguous: of k-step ks)
  __device__ __forceinline__ void init(int w0) {
    const int lane = threadIdx.x & 63;
    if constexpr (LAY == LAY_K) {
      const int r = lane & 31;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) o[ks] = (w0 + r) * BK + 8 * ((2 * ks + (lane >> 5)) ^ swz_k(r));
    } else {
      // lane group G = lane / 16 hands in k-rows 8 (G / 2) + e of rows 16 (G % 2) + 4 q
      // (lane 4 e + q) and receives four k values of one row
      const int G = lane >> 4, ll = lane & 15;
      const int k = 8 * (G >> 1) + (ll >> 2);
      const int c = w0 / 8 + 2 * (G & 1) + ((ll >> 1) & 1);
      o[0] = k * R + 8 * (c ^ (4 * (k & 3))) + 4 * (ll & 1);
    }
  }
  __device__ __forceinline__ bf16x8 read(const bf16* tile, int sub, int ks) const {
    if constexpr (LAY == LAY_K) {
      return *reinterpret_cast<const bf16x8*>(tile + o[ks] + sub * 32 * BK);
    } else {
      // rows + 32: chunk + 4, a field of its own under the XOR; k + 4: the same k % 4
      const bf16* q = tile + (o[0] ^ (sub << 5)) + ks * 16 * R;
      const bf16x4 lo = ds_read_tr((const lds_bf16x4*)lds(q));
      const bf16x4 hi = ds_read_tr((const lds_bf16x4*)lds(q + 4 * R));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

// Output tile of this workgroup.  Workgroups are dealt round-robin over the 8
// XCDs; renumber so that each XCD walks a contiguous range of the tile order,
// then order tiles in groups of 8 tile-rows so that the B tiles of a group
// stay in L2.
// With split-K the grid is (slice, tile) pairs: the renumbered id gives the
// slice (id / tiles) and the tile (id % tiles), so each XCD walks tiles of one
// slice.
__device__ __forceinline__ int xcd_order_id() {
  const int nwg = gridDim.x;
  int bid = blockIdx.x;
  if ((nwg & 7) == 0) bid = (bid & 7) * (nwg >> 3) + (bid >> 3);
  return bid;
}

template <int R = BT>
__device__ __forceinline__ void tile_origin(int M, int N, int bid, int& m0, int& n0) {
  const int tiles_m = (M + R - 1) / R, tiles_n = (N + R - 1) / R;
  constexpr int G = 8;
  const int per_group = G * tiles_n;
  const int group = bid / per_group;
  const int first_m = group * G;
  const int gsize = min(tiles_m - first_m, G);
  const int in_g = bid - group * per_group;
  m0 = (first_m + in_g % gsize) * R;
  n0 = (in_g / gsize) * R;
}

// The five-slot ring.
//
// Slots 0 - 2 hold A tiles (A_t in slot t % 3), slots 3 - 4 B tiles (B_t in
// slot 3 + t % 2).  Iteration t runs k-steps 0 - 2 of tile t, then waits for
// its copies and passes barrier_t, then runs k-step 3 of tile t while reading
// the first fragments of tile t + 1.  After barrier_t no wave reads tile t
// again, so the slots of A_t and B_t are free; the copies of one iteration go
// to slots freed by the previous barrier or by this one:
//   k-step 0: B_{t+1}, second half      k-step 2: A_{t+2}, second half
//   k-step 1: A_{t+2}, first half       k-step 3: B_{t+2}, first half
// Each k-step thus carries exactly four copies per wave, one after every
// fourth MFMA, and eight fragment reads, one after every second MFMA, in the
// order the next k-step consumes them.  At barrier_t only A_{t+2}'s eight
// copies may still be in flight.  Bunching the copies (four or eight at a
// time) stalls the in-order instruction stream behind a full address queue;
// this even spacing measured 3 - 5% faster on the GPT-J shapes.

// Fragment q (0 - 7) of a k-step in the order the MFMAs use it: a0, b0 - b3, a1 - a3.
template <int AL, int BL>
__device__ __forceinline__ void read_q(bf16x8 (&fa)[4], bf16x8 (&fb)[4], const Frags<AL>& FA,
                                       const Frags<BL>& FB, const bf16* sa, const bf16* sb, int ks,
                                       int q) {
  if (q == 0) fa[0] = FA.read(sa, 0, ks);
  else if (q <= 4) fb[q - 1] = FB.read(sb, q - 1, ks);
  else fa[q - 4] = FA.read(sa, q - 4, ks);
}

// One k-step: 16 MFMAs on (ca, cb); after MFMA i, fragment read i / 2 of the
// next k-step (odd i) and copy i / 4 (i % 4 == 2).  The scheduling barrier
// after every MFMA pins this order.
template <int AL, int BL, typename CopyF>
__device__ __forceinline__ void kstep_ring(floatx16 (&acc)[4][4], const bf16x8 (&ca)[4],
                                           const bf16x8 (&cb)[4], bf16x8 (&na)[4], bf16x8 (&nb)[4],
                                           const Frags<AL>& FA, const Frags<BL>& FB, const bf16* sa,
                                           const bf16* sb, int ks, CopyF copy) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    acc[i >> 2][i & 3] =
        __builtin_amdgcn_mfma_f32_32x32x16_bf16(ca[i >> 2], cb[i & 3], acc[i >> 2][i & 3], 0, 0, 0);
    if (i & 1) read_q(na, nb, FA, FB, sa, sb, ks, i >> 1);
    if ((i & 3) == 2) copy(i >> 2);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The loop: acc += the tile's product over nk K-tiles.  la, lb, FA and FB are initialised; K-tile t begins at
// k = kof(t), whose operands' resources are rsA(t, k) and rsB(t, k) (Loader::issue); for t >= nk (a few past the end
// are asked for) kof gives K, the end of k.  Afterwards no copy is in flight and every wave is done with
// smem (5 * OPE elements).
template <int AL, int BL, class KO, class RA, class RB>
__device__ __forceinline__ void gemm256_loop(floatx16 (&acc)[4][4], bf16* smem, const Loader<AL>& la,
                                             const Loader<BL>& lb, const Frags<AL>& FA, const Frags<BL>& FB,
                                             RA rsA, RB rsB, int nk, KO kof, int K, int wave) {
  constexpr int NI = Loader<LAY_K>::NI;
  static_assert(5 * OPE * 2 <= 163840 && BK == 64 && NI == 8, "LDS budget / copies");
  auto sA = [&](int t) { return smem + (t % 3) * OPE; };
  auto sB = [&](int t) { return smem + (3 + (t & 1)) * OPE; };
  // tile 0 resident; A_1 and the first half of B_1 in flight
  la.issue(rsA(0, 0), 0, K, sA(0), wave);
  lb.issue(rsB(0, 0), 0, K, sB(0), wave);
  wait_vm_lgkm0<0>();
  cta_barrier();
  la.issue(rsA(1, kof(1)), kof(1), K, sA(1), wave);
  __amdgpu_buffer_rsrc_t rB1 = rsB(1, kof(1));  // of B_{t+1}
  lb.template issue<0, 4>(rB1, kof(1), K, sB(1), wave);
  bf16x8 f0a[4], f0b[4], f1a[4], f1b[4];
#pragma unroll
  for (int q = 0; q < 8; ++q) read_q(f0a, f0b, FA, FB, sA(0), sB(0), 0, q);
  for (int t = 0; t < nk; ++t) {
    const bf16* a = sA(t);
    const bf16* b = sB(t);
    bf16* b1 = sB(t + 1);
    bf16* a2 = sA(t + 2);
    bf16* b2 = sB(t + 2);
    const int k1 = kof(t + 1), k2 = kof(t + 2);
    const __amdgpu_buffer_rsrc_t rA2 = rsA(t + 2, k2), rB2 = rsB(t + 2, k2);
    __builtin_amdgcn_sched_barrier(0);
    kstep_ring(acc, f0a, f0b, f1a, f1b, FA, FB, a, b, 1, [&](int c) {
      switch (c) {
        case 0: lb.template issue<4, 5>(rB1, k1, K, b1, wave); break;
        case 1: lb.template issue<5, 6>(rB1, k1, K, b1, wave); break;
        case 2: lb.template issue<6, 7>(rB1, k1, K, b1, wave); break;
        default: lb.template issue<7, 8>(rB1, k1, K, b1, wave); break;
      }
    });
    kstep_ring(acc, f1a, f1b, f0a, f0b, FA, FB, a, b, 2, [&](int c) {
      switch (c) {
        case 0: la.template issue<0, 1>(rA2, k2, K, a2, wave); break;
        case 1: la.template issue<1, 2>(rA2, k2, K, a2, wave); break;
        case 2: la.template issue<2, 3>(rA2, k2, K, a2, wave); break;
        default: la.template issue<3, 4>(rA2, k2, K, a2, wave); break;
      }
    });
    kstep_ring(acc, f0a, f0b, f1a, f1b, FA, FB, a, b, 3, [&](int c) {
      switch (c) {
        case 0: la.template issue<4, 5>(rA2, k2, K, a2, wave); break;
        case 1: la.template issue<5, 6>(rA2, k2, K, a2, wave); break;
        case 2: la.template issue<6, 7>(rA2, k2, K, a2, wave); break;
        default: la.template issue<7, 8>(rA2, k2, K, a2, wave); break;
      }
    });
    wait_vm_lgkm0<NI>();  // A_{t+1}, B_{t+1} resident; reads of tile t done
    cta_barrier();                // ... in every wave: A_t's and B_t's slots are free
    kstep_ring(acc, f1a, f1b, f0a, f0b, FA, FB, sA(t + 1), b1, 0, [&](int c) {
      switch (c) {
        case 0: lb.template issue<0, 1>(rB2, k2, K, b2, wave); break;
        case 1: lb.template issue<1, 2>(rB2, k2, K, b2, wave); break;
        case 2: lb.template issue<2, 3>(rB2, k2, K, b2, wave); break;
        default: lb.template issue<3, 4>(rB2, k2, K, b2, wave); break;
      }
    });
    rB1 = rB2;
  }
  wait_vm_lgkm0<0>();  // the zero-filling copies past the last tile
  __syncthreads();
}

// The same product on a tile of 128 x 128 (a wave: 64 x 64), for products that are too small to give every CU a
// tile of 256: STAGES stages of both operands (32 KB each), the copies STAGES - 1 K-tiles ahead, one barrier for each.
// Four stages where no CU has more than one such tile, two (and two workgroups on a CU) where there are more.  A k-step's
// fragments are read before the products of the one before it, with four stages across tiles too (a linear head of 296
// x 101 x 1288: 32.4 -> 30.7 us); five stages are no faster (32.2).
constexpr int RS = 128;
constexpr int small_lds(int stages) { return stages * 2 * RS * BK; }  // elements
template <int STAGES, int AL, int BL, class KO, class RA, class RB>
__device__ __forceinline__ void gemm128_loop(floatx16 (&acc)[2][2], bf16* smem, const Loader<AL, RS>& la,
                                             const Loader<BL, RS>& lb, const Frags<AL, RS>& FA, const Frags<BL, RS>& FB,
                                             RA rsA, RB rsB, int nk, KO kof, int K, int wave) {
  constexpr int COPIES = Loader<AL, RS>::NI + Loader<BL, RS>::NI;
  auto sA = [&](int t) { return smem + (t % STAGES) * 2 * RS * BK; };
  auto copy = [&](int t) {
    const int k = kof(t);
    la.issue(rsA(t, k), k, K, sA(t), wave);
    lb.issue(rsB(t, k), k, K, sA(t) + RS * BK, wave);
  };
  constexpr int KS = BK / 16;
  // LDS reads of a k-step's fragments
  constexpr int READS = 2 * (AL == LAY_K ? 1 : 2) + 2 * (BL == LAY_K ? 1 : 2);
  constexpr bool AHEAD = STAGES > 2;  // the next tile's first fragments too, for which it has to be there a tile early
  bf16x8 fa[2][2], fb[2][2];
  const auto read = [&](int t, int ks) {
    const bf16* a = sA(t);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[ks & 1][i] = FA.read(a, i, ks);
      fb[ks & 1][i] = FB.read(a + RS * BK, i, ks);
    }
  };
#pragma unroll
  for (int t = 0; t < STAGES - 1; ++t) copy(t);
  if constexpr (AHEAD) {
    wait_vm_lgkm0<(STAGES - 2) * COPIES>();
    cta_barrier();
    read(0, 0);
  }
  for (int t = 0; t < nk; ++t) {
    // tile t (with AHEAD t + 1) resident; this wave's reads of tile t - 1 done
    wait_vm_lgkm0<(AHEAD ? STAGES - 3 : 0) * COPIES>();
    cta_barrier();  // ... every wave's: its stage is free
    if constexpr (!AHEAD) {
      copy(t + STAGES - 1);
      read(t, 0);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bool more = AHEAD || ks + 1 < KS;
      if (more) read(ks + 1 < KS ? t : t + 1, (ks + 1) % KS);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[ks & 1][i], fb[ks & 1][j], acc[i][j], 0, 0, 0);
      if (more) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 4, 0);
      if (AHEAD && ks == 0) {
        __builtin_amdgcn_sched_barrier(0);
        copy(t + STAGES - 1);
      }
    }
  }
  wait_vm_lgkm0<0>();  // the zero-filling copies past the last tile
  __syncthreads();
}

}  // namespace
