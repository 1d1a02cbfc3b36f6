// Counter-based random numbers: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC'11).  Four words of 32 bits for every counter of 128 bits
// and key of 64, so that any element's numbers can be formed again without those before it.
#pragma once

#include "common.h"

__device__ __forceinline__ void philox_round(uint32_t& c0, uint32_t& c1, uint32_t& c2,
                                             uint32_t& c3, uint32_t k0, uint32_t k1) {
  const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
  const uint32_t n0 = (uint32_t)(q >> 32) ^ c1 ^ k0, n2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
  c0 = n0; c1 = (uint32_t)q; c2 = n2; c3 = (uint32_t)p;
}
__device__ __forceinline__ void philox4x32_10(uint32_t ctr[4], uint32_t k0, uint32_t k1) {
  const uint32_t W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    philox_round(ctr[0], ctr[1], ctr[2], ctr[3], k0, k1);
    k0 += W0;
    k1 += W1;
  }
}

// Dropout of a row-major matrix: eight columns share a counter (column / 8, row, step), each takes
// 16 of its 128 bits and is dropped when they are below `limit` = round(65536 p).  What
// is kept is multiplied by up = 65536 / (65536 - limit), so that the mean stays exact
// for the p that 16 bits can say.
struct DropConsts {
  uint32_t k0, k1, limit;
  float up;                // 0 when everything is dropped
  const uint64_t* step;    // device; NULL: step 0
};

struct DropRow {
  uint32_t w[4];
};

__device__ __forceinline__ uint64_t drop_step(const DropConsts& c) { return c.step ? *c.step : 0; }

__device__ __forceinline__ DropRow drop_bits(const DropConsts& c, uint64_t step, uint32_t row, uint32_t c8) {
  DropRow r = {{c8, row, (uint32_t)step, (uint32_t)(step >> 32)}};
  philox4x32_10(r.w, c.k0, c.k1);
  return r;
}

// Whether element e of the eight is kept.
__device__ __forceinline__ bool drop_keeps(const DropConsts& c, const DropRow& r, int e) {
  const uint32_t w = r.w[e >> 1];
  return ((e & 1) ? w >> 16 : w & 0xFFFFu) >= c.limit;
}
