// Where a workgroup of the packed-sequence attention kernels works: which sequence, which
// block of its rows, which heads; and which keys a query sees (device side).
#pragma once

#include "common.h"
#include "kernels.h"

namespace {

// Block `tile` of R rows.  Sequence i's blocks are numbered from first(i) = cu[i] / R + i, which
// leaves at least as many numbers as it has blocks (some stay unused), is known from cu alone and
// rises with i: no table of blocks is needed, and no length on the host.  A round of the search
// looks at 64 sequences at once, one per lane.  Row numbers are held to [0, T], so that
// no row outside the buffers is touched whatever cu holds.  False: the number is unused.
__device__ __forceinline__ bool find_rows(const AttnPackedArgs& a, int tile, int R, int& s0, int& S, int& blk) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = a.n_seq;
  for (;;) {
    const int step = (hi - lo + 63) >> 6;
    const int i = lo + lane * step;
    const bool at = i < hi && min(max(a.cu[i < hi ? i : lo], 0), a.T) / R + i <= tile;
    const int n = (int)__popcll(__builtin_amdgcn_ballot_w64(at));
    if (n == 0) return false;
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
    if (step <= 1) break;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  s0 = min(max(a.cu[lo], 0), a.T);
  S = min(max(a.cu[lo + 1], s0), a.T) - s0;
  blk = tile - (s0 / R + lo);
  return blk >= 0 && blk * R < S;
}

// The workgroup's block and head.  Workgroups are dealt round-robin over the 8 XCDs, each with
// its own L2.  Units of `run` consecutive blocks of all `per` heads (or head parts) that read
// one K / V head go to an XCD whole, so that the K and V rows of a stretch come from HBM into
// one L2, and the units of a stretch, alike in work, to different XCDs.
__device__ __forceinline__ bool packed_item(const AttnPackedArgs& a, int per, int& tile, int& kv, int& part) {
  const int id = blockIdx.x, slot = id >> 3;
  const int unit = slot / (a.run * per) * 8 + (id & 7), w = slot % (a.run * per);
  kv = unit % a.Hkv;
  tile = unit / a.Hkv * a.run + w / per;
  part = w % per;
  return tile < a.ntile;
}

// Keys [key_lo, key_hi) of query q, and queries [query_lo, query_hi) of key k, in a sequence of S rows.
__device__ __forceinline__ int key_lo(const AttnPackedArgs& a, int q) { return max(0, q - a.window + 1); }
__device__ __forceinline__ int key_hi(const AttnPackedArgs& a, int q, int S) {
  return min(S, a.causal ? q + 1 : q + a.window);
}
__device__ __forceinline__ int query_lo(const AttnPackedArgs& a, int k) { return a.causal ? k : max(0, k - a.window + 1); }
__device__ __forceinline__ int query_hi(const AttnPackedArgs& a, int k, int S) { return min(S, k + a.window); }

}  // namespace

// Launch shape for blocks of R rows and `per` workgroups on each block and K / V head: sets
// a.ntile and a.run, returns the workgroups.  A unit holds up to 16 blocks (2048 rows share their K and V
// reads in an L2), fewer while that leaves an XCD fewer than four units.
inline unsigned packed_grid(AttnPackedArgs& a, int R, int per) {
  a.ntile = a.T / R + a.n_seq;
  a.run = 16;
  while (a.run > 1 && (long)sat_cdiv(a.ntile, a.run) * a.Hkv < 32) a.run /= 2;
  const long units = (long)sat_cdiv(a.ntile, a.run) * a.Hkv;
  return (unsigned)((units + 7) / 8 * 8 * a.run * per);
}
