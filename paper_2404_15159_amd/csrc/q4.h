// 4-bit frozen matrices: their layout, shared by the kernels and the entry points.
//
// W' [n, K] = scale x level: codes are 4-bit floating-point numbers (sign, two exponent bits, one of
// fraction: 0, 0.5, 1, 1.5, 2, 3, 4, 6), which the hardware widens two per instruction; scales are bf16, one
// per group of 32, 64 or 128 consecutive inputs of a row.  A tile is 16 rows x 128 inputs, tiles of a row
// block follow one another.  In a tile, the 16 bytes at 16 (16 h + i) belong to row i: its bytes 4 b .. 4 b + 3
// hold inputs 32 b + 8 h .. + 7, the even one in the low half of a byte.  So the 16 bytes at 16 * lane are
// what a lane of a wavefront needs for four MFMA 16x16x32 steps, a wavefront reads a tile as one run of 1 KiB,
// and a step meets inputs of one group only.  Scales: [tile][row][group of the tile].  What lies past the
// last row or input is zero.
#pragma once
#include "common.h"

namespace mixlora {

constexpr int Q4_ROWS = 16, Q4_COLS = 128, Q4_TILE_BYTES = Q4_ROWS * Q4_COLS / 2;
__host__ __device__ __forceinline__ int64_t q4_row_blocks(int n) { return (n + Q4_ROWS - 1) / Q4_ROWS; }
__host__ __device__ __forceinline__ int64_t q4_col_blocks(int K) { return (K + Q4_COLS - 1) / Q4_COLS; }
inline size_t q4_code_bytes(int n, int K) { return (size_t)(q4_row_blocks(n) * q4_col_blocks(K)) * Q4_TILE_BYTES; }
inline size_t q4_scale_bytes(int n, int K, int group) {
  return (size_t)(q4_row_blocks(n) * q4_col_blocks(K)) * Q4_ROWS * (Q4_COLS / group) * 2;
}
inline bool q4_group_ok(int g) { return g == 32 || g == 64 || g == 128; }

struct Q4Matrix {
  const unsigned char *codes;
  const bf16_t *scales;
  int n, K, group;
};
// out [n, K] or, transposed, [K, n] in the given storage dtype
hipError_t launch_q4_dequantize(const Q4Matrix &w, bool transposed, int dtype, void *out, hipStream_t st);

}  // namespace mixlora
