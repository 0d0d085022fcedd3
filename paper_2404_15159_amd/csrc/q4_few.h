// Few rows through a LoRA linear on a 4-bit matrix (csrc/q4_few.hip)
#pragma once
#include "q4.h"

namespace mixlora {

constexpr int Q4_FEW_ROWS = 128;
struct Q4Few {
  const bf16_t *x, *A, *B;   // [T, K], [r, K], [n, r]; r a multiple of 8
  int T, r, rank;            // entries from rank on fill up r
  float s;
  bf16_t *y;                 // [T, n]
};
size_t q4_few_scratch_floats(int n, int K, int T, int r);
hipError_t launch_q4_few(const Q4Matrix &w, const Q4Few &a, const DropArgs &drop, float *scratch, size_t floats, hipStream_t st);

// The same for more rows, whose projection is there: S slices [S][T][r], whose sum times f it is.  With PT its three bf16
// pieces are written there, [3][r][ldT].
struct Q4Projection {
  const float *P;
  int S;
  float f;
  bf16_t *PT;
  int ldT;
};
bool q4_mid_ok(int n, int K, int T);
size_t q4_mid_scratch_floats(int n, int K, int T);
hipError_t launch_q4_mid(const Q4Matrix &w, const Q4Few &a, const Q4Projection &P, float *scratch, size_t floats, hipStream_t st);

}  // namespace mixlora
