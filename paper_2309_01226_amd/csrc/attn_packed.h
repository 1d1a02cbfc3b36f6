// Where a workgroup of the packed-sequence attention kernels works: which sequence, which
// block of its rows, which heads; and which keys a query sees (device side).
#pragma once

#include "common.h"
#include "kernels.h"

namespace {

// Sum / maximum over the wave on the vector unit: lanes 1 and 2 away, 4 and 8 around the row of
// 16, then the rows and the halves.
template <class Op>
__device__ __forceinline__ int wave_all(int v, Op op) {
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 15, 15, true));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 15, 15, true));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 15, 15, true));
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 15, 15, true));
  const auto r = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
  v = op((int)r[0], (int)r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
  return __builtin_amdgcn_readfirstlane(op((int)h[0], (int)h[1]));
}

__device__ __forceinline__ int row_at(const AttnPackedArgs& a, int i) { return min(max(a.cu[i], 0), a.T); }

// Lane of the n-th set bit of a wave's mask (n below their number).
__device__ __forceinline__ int nth_bit(uint64_t mask, int n) {
  const int lane = threadIdx.x & 63;
  const bool me = (mask >> lane & 1) && (int)__popcll(mask & ((1ull << lane) - 1)) == n;
  return (int)__ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(me)) - 1;
}

// Block number `rank` (R rows each) of all sequences, in the order of their work, the longest first, so
// that the last blocks to end are short ones.  Nothing is sorted: nb is a sequence's number of blocks,
// held by the lanes.  By place: causal blocks have the work of their place b in the sequence, and sum
// max(0, nb - x) of them a place of x or more.  By sequence: sum [nb > x] nb blocks are in
// sequences of more than x, each sequence's own in a row.  A walk or a bisection over x finds the level
// that holds the rank, bit counts the sequence on it.  Causal blocks go by place where sequences are long
// (a mean of 256 rows with up to 64 dims, 1024 with over 128, else 2048; always dK / dV of 96 and 128 dims, one
// workgroup on a CU, and of shared heads, whose blocks are long) and all K and V stay in the last-level cache
// of 256 MB, since all sequences' are read over and over; else by sequence, where a sequence's are read once.
// By place and by sequence, us: 4 x 4096 rows, 16 heads of 64, forward 158 and 174; 24 documents in 8192 rows, 12
// heads of 64, 24.3 and 26.5; 16 x 1024, 16 heads of 80, 97 and 83; backward of 50 images of 128 dims 263 and
// 283, of 64 x 1024, 16 heads of 80 on 4, 848 and 1022; 64 x 1024, 16 heads of 128 (537 MB), forward 612 and
// 411, backward 1747 and 1466.  Beyond 256 sequences (four a lane) the blocks are short on average and are
// numbered from first(i) = cu[i] / R + i instead, which leaves each sequence at least as many numbers as it
// has blocks.  Row numbers are held to [0, T], so no row outside the buffers is touched whatever
// cu holds.  blk counts the places in the order of causal work (a query block's own place; a key block's
// from the end of its sequence).  False: no such block.
constexpr int kSortedSeqs = 256;
// C sequences a lane: first rows, rows and blocks, and the most blocks of one.
template <int C>
struct SeqLanes {
  int s[C], len[C], nb[C], most;
  __device__ __forceinline__ void load(const AttnPackedArgs& a, int R) {
    most = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int i = (threadIdx.x & 63) + 64 * c, j = min(i, a.n_seq - 1);
      s[c] = row_at(a, j);
      len[c] = max(row_at(a, j + 1), s[c]) - s[c];
      nb[c] = i < a.n_seq ? (len[c] + R - 1) / R : 0;
      most = max(most, nb[c]);
    }
    most = wave_all(most, [](int p, int q) { return max(p, q); });
  }
  __device__ __forceinline__ bool find(const AttnPackedArgs& a, int rank, int& s0, int& S, int& blk) const {
    // blocks on level x, and on the levels from x on
    auto level = [&](int x) {
      int n = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) n += (int)__popcll(__builtin_amdgcn_ballot_w64(a.by_place ? nb[c] > x : nb[c] == x + 1));
      return a.by_place ? n : n * (x + 1);
    };
    auto from = [&](int x) {
      int n = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) n += a.by_place ? max(0, nb[c] - x) : nb[c] > x ? nb[c] : 0;
      return wave_all(n, [](int p, int q) { return p + q; });
    };
    int lo, above = 0;  // the rank's level, blocks on the levels above it
    if (most <= 16) {   // level by level: a compare and a bit count each
      for (lo = most - 1; lo >= 0; --lo) {
        const int n = level(lo);
        if (above + n > rank) break;
        above += n;
      }
      if (lo < 0) return false;
    } else {
      if (rank >= from(0)) return false;
      lo = 0;
      for (int hi = most; hi - lo > 1;) {
        const int mid = (lo + hi) >> 1, n = from(mid);
        if (n > rank) {
          lo = mid;
        } else {
          hi = mid;
          above = n;
        }
      }
    }
    const int k = rank - above;  // among the blocks of the level
    const int of = a.by_place ? 1 : lo + 1;
    int seq = a.by_place ? k : k / of;
    blk = a.by_place ? lo : a.causal ? lo - (k - seq * of) : k - seq * of;
    s0 = S = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint64_t on = __builtin_amdgcn_ballot_w64(a.by_place ? nb[c] > lo : nb[c] == lo + 1);
      const int n = (int)__popcll(on);
      if (seq >= 0 && seq < n) {
        const int i = nth_bit(on, seq);
        s0 = __builtin_amdgcn_readlane(s[c], i);
        S = __builtin_amdgcn_readlane(len[c], i);
      }
      seq -= n;  // below 0 from there on
    }
    return true;
  }
};

__device__ __forceinline__ bool find_rows(const AttnPackedArgs& a, int rank, int R, int& s0, int& S, int& blk) {
  const int lane = threadIdx.x & 63;
  if (a.n_seq <= 64) {
    SeqLanes<1> q;
    q.load(a, R);
    return q.find(a, rank, s0, S, blk);
  }
  if (a.n_seq <= kSortedSeqs) {
    SeqLanes<4> q;
    q.load(a, R);
    return q.find(a, rank, s0, S, blk);
  }
  int lo = 0, hi = a.n_seq, s, e;
  for (;;) {
    const int step = (hi - lo + 63) >> 6;
    const int i = min(lo + lane * step, a.n_seq - 1);
    s = row_at(a, i);
    e = row_at(a, i + 1);
    const bool at = lo + lane * step < hi && s / R + i <= rank;
    const int n = (int)__popcll(__builtin_amdgcn_ballot_w64(at));
    if (n == 0) return false;
    if (step <= 1) {
      s0 = __builtin_amdgcn_readlane(s, n - 1);
      S = __builtin_amdgcn_readlane(e, n - 1) - s0;
      blk = rank - (s0 / R + lo + n - 1);
      return blk >= 0 && blk * R < S;
    }
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
}

// The workgroup's block number and head.  Workgroups are dealt round-robin over the 8 XCDs, each
// with its own L2.  Each K / V head's blocks belong to one XCD or, where the heads are no multiple of 8, every
// parts-th of them: its K and V come from HBM into one L2 (parts of them), and the XCDs have the same work.
// An XCD takes the blocks in their order, each for all its heads and the `per` query heads (or head parts) on
// them: a long block that starts late ends late, since three workgroups share a CU's time.
__device__ __forceinline__ bool packed_item(const AttnPackedArgs& a, int per, int& rank, int& kv, int& part) {
  const int id = blockIdx.x, slot = id >> 3;
  const int units = a.Hkv * a.parts >> 3;  // of an XCD
  const int block = slot / (units * per), w = slot - block * units * per;
  const int unit = w / per * 8 + (id & 7);
  part = w % per;
  kv = unit % a.Hkv;
  rank = block * a.parts + unit / a.Hkv;
  return rank < a.ntile;
}

// Keys [key_lo, key_hi) of query q, and queries [query_lo, query_hi) of key k, in a sequence of S rows.
__device__ __forceinline__ int key_lo(const AttnPackedArgs& a, int q) { return max(0, q - a.window + 1); }
__device__ __forceinline__ int key_hi(const AttnPackedArgs& a, int q, int S) {
  return min(S, a.causal ? q + 1 : q + a.window);
}
__device__ __forceinline__ int query_lo(const AttnPackedArgs& a, int k) { return a.causal ? k : max(0, k - a.window + 1); }
__device__ __forceinline__ int query_hi(const AttnPackedArgs& a, int k, int S) { return min(S, k + a.window); }

// Part sp of `split` of a block's steps [j0, j1).
__device__ __forceinline__ void part_of(int sp, int split, int& j0, int& j1) {
  const int n = j1 - j0, b = j0;
  j0 = b + (int)((long)sp * n / split);
  j1 = b + (int)((long)(sp + 1) * n / split);
}

// Partial results of a part: a wave's accumulators, 64 lanes side by side, at `at` (a part's place in the
// scratch) + its own share of `regs` registers.
__device__ __forceinline__ float* wave_share(float* ws, long at, int NW, int regs, int wave) {
  return ws + ((at * NW + wave) * regs) * 64 + (threadIdx.x & 63) * 4;
}
template <int OT>
__device__ __forceinline__ void put_acc(float* p, const floatx16 (&acc)[OT]) {
#pragma unroll
  for (int t = 0; t < OT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<floatx4*>(p + (4 * t + i) * 256) =
          floatx4{acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
}
// Tile t of a transposed accumulator set (32 head dims, column = this lane's row) times f to out[0 .. dh).
__device__ __forceinline__ void store_tile(bf16* out, const floatx4 (&acc)[4], int t, float f, int g, int dh) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = 32 * t + 8 * i + 4 * g;
    if (col >= dh) continue;
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = f2bf(acc[i][e] * f);
    *reinterpret_cast<bf16x4*>(out + col) = y;
  }
}

}  // namespace

// Launch shape for blocks of R rows and `per` workgroups on each block and K / V head (kv: of dK / dV): sets
// a.ntile, a.parts and a.by_place, returns the workgroups.
inline unsigned packed_grid(AttnPackedArgs& a, int R, int per, bool kv) {
  a.ntile = a.T / R + a.n_seq;
  const long bytes = 4L * a.T * a.Hkv * a.dh;  // of K and V
  const bool always = kv && (a.H > a.Hkv || (a.dh > 80 && a.dh <= 128));
  const long least = always ? 0 : a.dh <= 64 ? 256 : a.dh > 128 ? 1024 : 2048;
  a.by_place = a.causal && bytes <= (1L << 28) && a.T >= least * a.n_seq;
  a.parts = a.Hkv % 8 == 0 ? 1 : a.Hkv % 4 == 0 ? 2 : a.Hkv % 2 == 0 ? 4 : 8;
  return (unsigned)((long)a.Hkv * a.parts * sat_cdiv(a.ntile, a.parts) * per);
}
