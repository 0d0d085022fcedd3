// The rank-r projection of a LoRA linear and the operands that its rank-r term and its gradient sums take.
#pragma once
#include "common.h"
#include "dropout.h"

namespace mixlora {

// v as the sum of three bf16 values, cut off by truncation; infinities and NaN stay in the first
__device__ __forceinline__ void three_pieces(float v, float (&pc)[3]) {
  const bool finite = (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u;
  pc[0] = finite ? __uint_as_float(__float_as_uint(v) & 0xffff0000u) : v;
  const float rest = finite ? v - pc[0] : 0.f;
  pc[1] = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
  pc[2] = rest - pc[1];
}

// P[t, q] = sum_c X[t, c] * Wq[q, c]  (r <= 64 columns), in three forms: fp32, transposed bf16 (the
// row factor of the gradient sums) and m * P (s = m 2^e, 1/2 <= |m| < 1) cut into three bf16 pieces by
// truncation, ext[t] = [hi(r) | mid(r) | lo(r)]: their sum is m * P to its last bit, and no piece
// overflows.  Trailing workgroups lay out the other factor of that term, Bx[c] = [B | B' | B'] 2^e with
// B' = B but zeros for infinities: hi alone meets those, or two pieces of opposite signs would make
// NaN of them.
// Bound by reading X once (33 MB at 4096 x 4096: 9 us); a workgroup owns 16 rows, its eight waves every
// eighth 128-column run of them, so that 256 workgroups have 2 waves per SIMD with 4 KB each in flight;
// fragments come straight from memory (whole 128-byte lines over four MFMA steps), Wq from the caches.
// The waves' sums are added in a fixed order.
// DROP: the elements of X that the generator drops count as zeros, and P is multiplied by drop.inv (X row =
// generator row).  PIECES: PT is P in three such pieces of its own, [hi(r) | mid(r) | lo(r)][ldT], so that
// the gradient sums lose none of its bits.
template <int NQ, bool DROP, bool PIECES>
__global__ __launch_bounds__(512) void rank_project_kernel(const bf16_t *__restrict__ X,
                                                           const bf16_t *__restrict__ Wq, int T, int K,
                                                           int r, float m, float *__restrict__ P,
                                                           bf16_t *__restrict__ PT, int ldT,
                                                           bf16_t *__restrict__ ext,
                                                           int32_t *__restrict__ tok_offs,
                                                           const bf16_t *__restrict__ Bm, int cols,
                                                           float b_scale, bf16_t *__restrict__ Bx,
                                                           DropArgs drop) {
  __shared__ float red[8][NQ][64][4];
  const int row_blocks = (T + 15) >> 4;
  if ((int)blockIdx.x >= row_blocks) {   // workgroup-uniform; eight entries of a row of B per thread
    const int per = r >> 3, i = (blockIdx.x - row_blocks) * 512 + threadIdx.x;
    if (i >= cols * per) return;
    const int c = i / per, q0 = i % per * 8;
    bf16x8_t v = *reinterpret_cast<const bf16x8_t *>(Bm + (int64_t)c * r + q0), fin;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      v[e] = (bf16_t)((float)v[e] * b_scale);
      fin[e] = __builtin_isinf((float)v[e]) ? (bf16_t)0.f : v[e];
    }
    bf16_t *o = Bx + (int64_t)c * 3 * r + q0;
    *reinterpret_cast<bf16x8_t *>(o) = v;
    *reinterpret_cast<bf16x8_t *>(o + r) = fin;
    *reinterpret_cast<bf16x8_t *>(o + 2 * r) = fin;
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l15 = lane & 15, hi = lane >> 4;
  const int t0 = blockIdx.x * 16;
  if (blockIdx.x == 0 && threadIdx.x == 0) {   // all tokens are one group of the gradient sums
    tok_offs[0] = 0;
    tok_offs[1] = T;
  }
  const int row = t0 + l15 < T ? t0 + l15 : T - 1;
  const bf16_t *xr = X + (int64_t)row * K;
  const bf16_t *wr[NQ];
#pragma unroll
  for (int j = 0; j < NQ; j++) wr[j] = Wq + (int64_t)(j * 16 + l15 < r ? j * 16 + l15 : r - 1) * K;
  f32x4_t acc[NQ];
#pragma unroll
  for (int j = 0; j < NQ; j++) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  DropKey key;
  if constexpr (DROP) key = drop_key(drop);
  for (int k0 = wave * 128; k0 < K; k0 += 8 * 128) {
    bf16x8_t fx[4], fw[NQ][4];
#pragma unroll
    for (int ks = 0; ks < 4; ks++) {
      const int k = k0 + ks * 32 + hi * 8;
      const int kc = k < K ? k : 0;
      fx[ks] = *reinterpret_cast<const bf16x8_t *>(xr + kc);
#pragma unroll
      for (int j = 0; j < NQ; j++) fw[j][ks] = *reinterpret_cast<const bf16x8_t *>(wr[j] + kc);
    }
#pragma unroll
    for (int ks = 0; ks < 4; ks++) {
      if constexpr (DROP) fx[ks] = drop_mask8(key, (uint32_t)row, (uint32_t)(k0 + ks * 32 + hi * 8) >> 3, fx[ks]);
      if (k0 + ks * 32 + hi * 8 >= K) {   // past the end: zeros on both sides
#pragma unroll
        for (int u = 0; u < 8; u++) fx[ks][u] = (bf16_t)0.f;
#pragma unroll
        for (int j = 0; j < NQ; j++)
#pragma unroll
          for (int u = 0; u < 8; u++) fw[j][ks][u] = (bf16_t)0.f;
      }
#pragma unroll
      for (int j = 0; j < NQ; j++)
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[j][ks], fx[ks], acc[j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int j = 0; j < NQ; j++) *reinterpret_cast<f32x4_t *>(red[wave][j][lane]) = acc[j];
  __syncthreads();
  // acc[j][u] of lane (l15, hi): row l15, q = 16 j + 4 hi + u
  for (int i = threadIdx.x; i < NQ * 256; i += 512) {
    const int j = i >> 8, q = j * 16 + (i & 15), t = t0 + ((i >> 4) & 15);
    if (q >= r || t >= T) continue;
    const int ln = ((i >> 2) & 3) * 16 + ((i >> 4) & 15), u = i & 3;
    float v = red[0][j][ln][u];
#pragma unroll
    for (int w = 1; w < 8; w++) v += red[w][j][ln][u];
    if constexpr (DROP) v *= drop.inv;
    P[(int64_t)t * r + q] = v;
    float pc[3];
    if constexpr (PIECES) {
      three_pieces(v, pc);
#pragma unroll
      for (int i = 0; i < 3; i++) PT[((int64_t)i * r + q) * ldT + t] = (bf16_t)pc[i];
    } else {
      PT[(int64_t)q * ldT + t] = (bf16_t)v;
    }
    three_pieces(m * v, pc);
    bf16_t *o = ext + (int64_t)t * 3 * r + q;
    o[0] = (bf16_t)pc[0];
    o[r] = (bf16_t)pc[1];
    o[2 * r] = (bf16_t)pc[2];
  }
}

}  // namespace mixlora
