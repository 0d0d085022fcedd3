// Operand rows that change lanes in LDS, shared by the few-rows product with 4-bit codes and the rank-r projection.
#pragma once
#include "common.h"

namespace mixlora {

// Rows of a bf16 matrix as MFMA operands: 16 rows x 128 inputs, 4 KB.  In the operand's own layout neighbouring
// lanes hold different rows, and a load of it is 64 requests of 16 bytes (the rank-r rows of one token's product
// cost 5.1 us that way at 16 x 4096, 1.5 this way).  So they are loaded 256 bytes of a row at a time and change
// lanes in a piece of LDS that belongs to the wavefront alone, its 16-byte chunks in an order that leaves no two
// lanes of a group in one bank.
constexpr int STAGE_COLS = 128, STAGE_BYTES = 16 * STAGE_COLS * 2;
struct RowOffsets {
  uint32_t off[4];   // bytes: rows * K < 2^31
  // rows first .. first + 15 of `rows` (clamped: what is past the last one is not used)
  __device__ __forceinline__ RowOffsets(int first, int rows, int K, int lane) {
#pragma unroll
    for (int p = 0; p < 4; p++) {
      const int row = first + p * 4 + (lane >> 4);
      off[p] = (uint32_t)(row < rows ? row : rows - 1) * (uint32_t)K * 2u + (lane & 15) * 16;
    }
  }
};
// (kb is uniform over the wavefront; past K, in the last tile, the tile's first chunk is read instead)
__device__ __forceinline__ void rows_load(const bf16_t *base, const RowOffsets &o, int kb, int K, int lane, bf16x8_t (&v)[4]) {
  const unsigned char *p = reinterpret_cast<const unsigned char *>(base) + (int64_t)kb * (STAGE_COLS * 2);
  if ((kb + 1) * STAGE_COLS <= K) {
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = *reinterpret_cast<const bf16x8_t *>(p + o.off[i]);
  } else {
    const uint32_t back = kb * STAGE_COLS + (lane & 15) * 8 < K ? 0u : (lane & 15) * 16;
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = *reinterpret_cast<const bf16x8_t *>(p + (o.off[i] - back));
  }
}
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bf16x8_t zero_unless(bool in, bf16x8_t v) {
  u32x4_t w = __builtin_bit_cast(u32x4_t, v);
#pragma unroll
  for (int e = 0; e < 4; e++) w[e] = in ? w[e] : 0u;
  return __builtin_bit_cast(bf16x8_t, w);
}
__device__ __forceinline__ void rows_to_lds(unsigned char *lds, bf16x8_t (&v)[4], int kb, int K, int lane) {
  if ((kb + 1) * STAGE_COLS > K) {
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = zero_unless(kb * STAGE_COLS + (lane & 15) * 8 < K, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int row = i * 4 + (lane >> 4);
    *reinterpret_cast<bf16x8_t *>(lds + row * 256 + ((lane ^ row) & 15) * 16) = v[i];
  }
}
__device__ __forceinline__ void rows_from_lds(const unsigned char *lds, int lane, bf16x8_t (&f)[4]) {
  const int l15 = lane & 15, hi = lane >> 4;
#pragma unroll
  for (int st = 0; st < 4; st++)
    f[st] = *reinterpret_cast<const bf16x8_t *>(lds + l15 * 256 + (((st * 4 + hi) ^ l15) & 15) * 16);
}
// the first 16 of `rows` rows at base, wherever (offsets inside them stay below 2^32 for K < 2^27)
__device__ __forceinline__ void rows_load(const bf16_t *base, int rows, int kb, int K, int lane, bf16x8_t (&v)[4]) {
  rows_load(base, RowOffsets(0, rows, K, lane), kb, K, lane, v);
}
// between the two: the wavefront's LDS accesses keep their order (the hardware takes them in order)
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// v as the sum of three bf16 values, cut off by truncation; infinities and NaN stay in the first
__device__ __forceinline__ void three_pieces(float v, float (&pc)[3]) {
  const bool finite = (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u;
  pc[0] = finite ? __uint_as_float(__float_as_uint(v) & 0xffff0000u) : v;
  const float rest = finite ? v - pc[0] : 0.f;
  pc[1] = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
  pc[2] = rest - pc[1];
}

}  // namespace mixlora
