// Dropout of a matrix's elements from a counter-based generator: nothing is stored, every kernel that
// needs the mask makes it again.  The generator is Philox (Salmon, Moraes, Dror, Shaw: "Parallel random
// numbers: as easy as 1, 2, 3", 2011) on four 32-bit words with seven rounds, the fewest that the paper
// reports as passing its whole test battery (ten cost 40 % more multiplications).  One call serves eight
// consecutive columns of a row, 16 bits each, which is what a 16-byte load of bf16 holds.
#pragma once
#include "common.h"

namespace mixlora {

struct DropKey {            // what is uniform over a launch
  uint32_t k0, k1, c2, c3, thr16;
};
__device__ __forceinline__ DropKey drop_key(const DropArgs &d) {
  const uint64_t o = d.offset + (d.step ? *d.step : 0);
  return DropKey{d.k0, d.k1, (uint32_t)o, (uint32_t)(o >> 32), d.thr << 16};
}

// bit e: column 8 col8 + e of the row stays
__device__ __forceinline__ uint32_t drop_keep8(const DropKey &k, uint32_t row, uint32_t col8) {
  uint32_t c0 = col8, c1 = row, c2 = k.c2, c3 = k.c3, k0 = k.k0, k1 = k.k1;
#pragma unroll
  for (int i = 0; i < 7; i++) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  const uint32_t w[4] = {c0, c1, c2, c3};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    m |= ((w[i] << 16) >= k.thr16 ? 1u : 0u) << (2 * i);
    m |= (w[i] >= k.thr16 ? 2u : 0u) << (2 * i);
  }
  return m;
}

// zeros for the columns that are dropped (a selection: what is dropped may be infinite or NaN)
__device__ __forceinline__ bf16x8_t drop_mask8(const DropKey &k, uint32_t row, uint32_t col8, bf16x8_t v) {
  const uint32_t m = drop_keep8(k, row, col8);
#pragma unroll
  for (int e = 0; e < 8; e++) v[e] = (m >> e & 1) ? v[e] : (bf16_t)0.f;
  return v;
}

}  // namespace mixlora
