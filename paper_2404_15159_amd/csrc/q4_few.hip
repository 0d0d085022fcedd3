// Products of few rows (up to 1024) with a 4-bit frozen matrix, and the rank-r term of a LoRA linear on it:
//   y = x W'^T + s (D(x) A^T) B^T.
// Bound by reading the codes once, and from some tens of rows on by reading x for every 64 columns.  Codes go from memory
// to registers as a wavefront's MFMA operand (q4.h) and are widened there, two per instruction; levels are exact in bf16,
// so x times level is summed in fp32 as it is and a group's sum is multiplied by the group's scale in fp32: nothing is
// rounded before y (but see q4_tile_scaled).  The sum of a group is at most 768 |x|, which fp32 holds for |x| <= 2^118.
#include "q4.h"
#include "q4_few.h"
#include "dropout.h"
#include "rows_stage.h"

#include <type_traits>

namespace mixlora {

typedef bf16_t bf16x2_t __attribute__((ext_vector_type(2)));

// eight codes as an MFMA operand
__device__ __forceinline__ bf16x8_t q4_operand(uint32_t word) {
  bf16x2_t p[4];
  p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.f, 0);
  p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.f, 1);
  p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.f, 2);
  p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.f, 3);
  bf16x8_t v;
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = p[i >> 1][i & 1];
  return v;
}

// the PER = 128 / group scales of a lane's row in a tile
template <int PER> __device__ __forceinline__ void q4_load_scales(const bf16_t *p, float (&s)[PER]);
template <> __device__ __forceinline__ void q4_load_scales<1>(const bf16_t *p, float (&s)[1]) { s[0] = (float)*p; }
template <> __device__ __forceinline__ void q4_load_scales<2>(const bf16_t *p, float (&s)[2]) {
  const uint32_t v = *reinterpret_cast<const uint32_t *>(p);
  s[0] = __uint_as_float(v << 16), s[1] = __uint_as_float(v & 0xffff0000u);
}
template <> __device__ __forceinline__ void q4_load_scales<4>(const bf16_t *p, float (&s)[4]) {
  const uint2 v = *reinterpret_cast<const uint2 *>(p);
  s[0] = __uint_as_float(v.x << 16), s[1] = __uint_as_float(v.x & 0xffff0000u);
  s[2] = __uint_as_float(v.y << 16), s[3] = __uint_as_float(v.y & 0xffff0000u);
}

// a lane's codes and scales of a tile (uniform over the wavefront)
template <int PER>
__device__ __forceinline__ void q4_load(const Q4Matrix &w, int64_t tile, int lane, uint4 &c, float (&s)[PER]) {
  c = *reinterpret_cast<const uint4 *>(w.codes + tile * Q4_TILE_BYTES + (uint32_t)lane * 16u);
  q4_load_scales<PER>(w.scales + tile * (Q4_ROWS * PER) + (uint32_t)(lane & 15) * PER, s);
}

// acc += (sums of x times level over each group of the tile) x scale; MT blocks of 16 rows
template <int MT, int PER>
__device__ __forceinline__ void q4_tile(const bf16x8_t (&fx)[MT][4], const uint4 &c, const float (&s)[PER],
                                        f32x4_t (&acc)[MT]) {
  const uint32_t word[4] = {c.x, c.y, c.z, c.w};
  constexpr int STEPS = 4 / PER;
#pragma unroll
  for (int g = 0; g < PER; g++) {
    f32x4_t part[MT];
#pragma unroll
    for (int m = 0; m < MT; m++) part[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = g * STEPS; st < (g + 1) * STEPS; st++) {
      const bf16x8_t fw = q4_operand(word[st]);
#pragma unroll
      for (int m = 0; m < MT; m++) part[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[m][st], fw, part[m], 0, 0, 0);
    }
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
      for (int u = 0; u < 4; u++) acc[m][u] = fmaf(s[g], part[m][u], acc[m][u]);
  }
}

// ---- up to 64 rows (32 of more than 8192 inputs), rank up to 16, no dropout: one launch ---------------------------------------------
// A workgroup owns NT tiles' rows (16 NT columns of y) over the whole contraction, its eight wavefronts every
// eighth tile of it; MT blocks of 16 rows of x.  Every workgroup makes the projection x A^T itself (128 KB of A at
// 16 x 4096, out of L2): that costs less than a launch in front of this one.  Nothing is requested ahead within a
// wavefront: with the registers that takes, fewer of them fit, and one token 4096 -> 4096 took 6.6 instead of 5.4 us.
// ONE: a single row of x, which every lane can read for itself.
template <int NT, int MT, int PER, bool ONE>
__global__ __launch_bounds__(512) void q4_few_kernel(Q4Matrix w, Q4Few a) {
  static_assert(!ONE || MT == 1, "one row is one block");
  constexpr int WAVES = 8;
  // staging of A, then of x, wavefront by wavefront; sums [8][NT + 1][MT][64][4] (the last: of the projection), and
  // the projection itself
  extern __shared__ __align__(16) unsigned char smem[];
  auto red = reinterpret_cast<float(*)[NT + 1][MT][64][4]>(smem);
  auto sp = reinterpret_cast<float(*)[17]>(smem + WAVES * (NT + 1) * MT * 1024);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hi = lane >> 4;
  const int rb0 = blockIdx.x * NT, row_blocks = (int)q4_row_blocks(w.n), kbs = (int)q4_col_blocks(w.K);
  const int T = a.T, r = a.r, K = w.K;
  // what the end needs of B: column col of tile i for tokens tok, tok + 16, ..
  const int col = tid & 15, tok = (tid >> 4) & 15, half = tid >> 8;
  constexpr int OUT = (NT + 1) / 2;
  bf16x8_t bq[OUT][2];
#pragma unroll
  for (int o = 0; o < OUT; o++) {
    const int n = (rb0 + half + 2 * o) * 16 + col;
#pragma unroll
    for (int h = 0; h < 2; h++)
      bq[o][h] = *reinterpret_cast<const bf16x8_t *>(a.B + (int64_t)(n < w.n ? n : 0) * r + (8 * h < r ? 8 * h : 0));
  }
  unsigned char *stage = smem + wave * MT * STAGE_BYTES;
  int64_t first[NT];   // tiles in front of each row block
#pragma unroll
  for (int i = 0; i < NT; i++) first[i] = (int64_t)(rb0 + i < row_blocks ? rb0 + i : row_blocks - 1) * kbs;
  f32x4_t acc[NT][MT], accp[MT];
#pragma unroll
  for (int m = 0; m < MT; m++) {
    accp[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NT; i++) acc[i][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const RowOffsets oa(0, r, K, lane);
  for (int kb = wave; kb < kbs; kb += WAVES) {
    uint4 c[NT];
    float s[NT][PER];
    bf16x8_t va[4], vx[MT][4], fa[4], fx[MT][4];
    rows_load(a.A, oa, kb, K, lane, va);
#pragma unroll
    for (int i = 0; i < NT; i++) q4_load<PER>(w, first[i] + kb, lane, c[i], s[i]);
    if constexpr (ONE) {
#pragma unroll
      for (int st = 0; st < 4; st++) {
        const int k = st * 32 + hi * 8;
        fx[0][st] = *reinterpret_cast<const bf16x8_t *>(
            a.x + (int64_t)kb * Q4_COLS + (uint32_t)((kb + 1) * Q4_COLS <= K || kb * Q4_COLS + k < K ? k : 0));
      }
      if ((kb + 1) * Q4_COLS > K) {
#pragma unroll
        for (int st = 0; st < 4; st++) fx[0][st] = zero_unless(kb * Q4_COLS + st * 32 + hi * 8 < K, fx[0][st]);
      }
    } else {
#pragma unroll
      for (int m = 0; m < MT; m++) rows_load(a.x, RowOffsets(m * 16, T, K, lane), kb, K, lane, vx[m]);
    }
    wave_order();
    rows_to_lds(stage, va, kb, K, lane);
    wave_order();
    rows_from_lds(stage, lane, fa);
    if constexpr (!ONE) {
      wave_order();
#pragma unroll
      for (int m = 0; m < MT; m++) rows_to_lds(stage + m * STAGE_BYTES, vx[m], kb, K, lane);
      wave_order();
#pragma unroll
      for (int m = 0; m < MT; m++) rows_from_lds(stage + m * STAGE_BYTES, lane, fx[m]);
    }
#pragma unroll
    for (int st = 0; st < 4; st++)
#pragma unroll
      for (int m = 0; m < MT; m++) accp[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[m][st], fa[st], accp[m], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NT; i++) q4_tile<MT, PER>(fx, c[i], s[i], acc[i]);
  }
  __syncthreads();   // the staging is behind everybody
  // lane (l15, hi), register u: row 4 hi + u, column l15
#pragma unroll
  for (int m = 0; m < MT; m++) {
#pragma unroll
    for (int i = 0; i < NT; i++) *reinterpret_cast<f32x4_t *>(red[wave][i][m][lane]) = acc[i][m];
    *reinterpret_cast<f32x4_t *>(red[wave][NT][m][lane]) = accp[m];
  }
  __syncthreads();
  const int ln = (tok >> 2) * 16 + col, u = tok & 3;
#pragma unroll
  for (int m = 0; m < MT; m++) {
    if ((m & 1) != half) continue;   // the halves of the workgroup share the row blocks
    float v = red[0][NT][m][ln][u];
#pragma unroll
    for (int q = 1; q < WAVES; q++) v += red[q][NT][m][ln][u];
    sp[m * 16 + tok][col] = col < a.rank ? v : 0.f;   // (a zero row of A makes NaN beside an infinite row of x)
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MT; m++) {
    const int t = m * 16 + tok;
    if (t >= T) break;
#pragma unroll
    for (int o = 0; o < OUT; o++) {
      const int i = half + 2 * o, n = (rb0 + i) * 16 + col;
      if (i >= NT || n >= w.n) continue;
      float v = red[0][i][m][ln][u], p = 0.f;
#pragma unroll
      for (int q = 1; q < WAVES; q++) v += red[q][i][m][ln][u];
#pragma unroll
      for (int q = 0; q < 8; q++) p = fmaf(sp[t][q], (float)bq[o][0][q], p);
      if (r > 8) {
#pragma unroll
        for (int q = 0; q < 8; q++) p = fmaf(sp[t][8 + q], (float)bq[o][1][q], p);
      }
      a.y[(int64_t)t * w.n + n] = (bf16_t)fmaf(a.s, p, v);
    }
  }
}
template <int NT, int MT> constexpr size_t few_lds() {
  const size_t stage = (size_t)8 * MT * STAGE_BYTES, sums = (size_t)8 * (NT + 1) * MT * 1024 + (size_t)MT * 16 * 17 * 4;
  return stage > sums ? stage : sums;
}
template <int NT, int MT, int PER, bool ONE>
static hipError_t launch_few(const Q4Matrix &w, const Q4Few &a, hipStream_t st) {
  constexpr size_t lds = few_lds<NT, MT>();
  if constexpr (lds > 65536) {
    static const hipError_t e = hipFuncSetAttribute((const void *)q4_few_kernel<NT, MT, PER, ONE>,
                                                    hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((q4_few_kernel<NT, MT, PER, ONE>), dim3((unsigned)((q4_row_blocks(w.n) + NT - 1) / NT)), dim3(512),
                     lds, st, w, a);
  return hipGetLastError();
}
template <int MT, int PER, bool ONE>
static hipError_t launch_few_n(const Q4Matrix &w, const Q4Few &a, hipStream_t st) {
  // as many tiles per workgroup as leave the chip one round of workgroups.  One, two, three of them at 1 | 24 | 64 tokens, us,
  // with the codes in memory, not in a cache:
  //   4096 -> 4096,   256 tiles   6.6  6.9  7.8 |  9.7 10.4 11.8 | 14.9 15.2 17.1
  //   5120 -> 5120,   320 tiles  11.7  8.5  9.7 | 18.4 13.2 14.7 | 29.8 19.8 22.2
  //   4096 -> 8192,   512 tiles  10.0  7.5  8.3 | 15.2 11.0 12.3 | 26.8 17.0 17.7
  //   4096 -> 11008,  688 tiles  13.3 11.6  8.8 | 20.8 18.6 12.8 | 36.9 28.4 18.6
  // More than 768 tiles are more than a round of three, which is where two would be ahead until they need a third round:
  //   4096 -> 14336,  896 tiles  16.8 12.0 14.4 | 26.3 19.6 21.6 | 47.8 29.9 31.5
  const int64_t tiles = q4_row_blocks(w.n);
  if (tiles <= 256) return launch_few<1, MT, PER, ONE>(w, a, st);
  if (tiles <= 512) return launch_few<2, MT, PER, ONE>(w, a, st);
  return launch_few<3, MT, PER, ONE>(w, a, st);
}
template <int PER> static hipError_t launch_few_m(const Q4Matrix &w, const Q4Few &a, hipStream_t st) {
  if (a.T == 1) return launch_few_n<1, PER, true>(w, a, st);
  if (a.T <= 16) return launch_few_n<1, PER, false>(w, a, st);
  if (a.T <= 32) return launch_few_n<2, PER, false>(w, a, st);
  return launch_few_n<4, PER, false>(w, a, st);
}

// The same with the codes as the first operand: a lane has four neighbouring columns of y of one row instead of four rows of a
// column, which is how sums are then added and written 16 bytes at a time.  It takes the scales of its four columns,
// [column][group] as they are held.
template <int PER> struct Q4Scales4 { uint32_t w[2 * PER]; };
template <int PER>
__device__ __forceinline__ void q4_load_scales4(const Q4Matrix &w, int64_t tile, int lane, Q4Scales4<PER> &s) {
  const bf16_t *p = w.scales + tile * (Q4_ROWS * PER) + (uint32_t)(lane >> 4) * (4 * PER);
  if constexpr (PER == 1) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    s.w[0] = v.x, s.w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < PER / 2; i++) {
      const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
      s.w[4 * i] = v.x, s.w[4 * i + 1] = v.y, s.w[4 * i + 2] = v.z, s.w[4 * i + 3] = v.w;
    }
  }
}
template <int MT, int PER>
__device__ __forceinline__ void q4_tile4(const bf16x8_t (&fx)[MT][4], const uint4 &c, const Q4Scales4<PER> &s, f32x4_t (&acc)[MT]) {
  const uint32_t word[4] = {c.x, c.y, c.z, c.w};
  constexpr int STEPS = 4 / PER;
#pragma unroll
  for (int g = 0; g < PER; g++) {
    f32x4_t part[MT];
#pragma unroll
    for (int m = 0; m < MT; m++) part[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = g * STEPS; st < (g + 1) * STEPS; st++) {
      const bf16x8_t fw = q4_operand(word[st]);
#pragma unroll
      for (int m = 0; m < MT; m++) part[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw, fx[m][st], part[m], 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < 4; u++) {
      const int at = u * PER + g;
      const float sc = __uint_as_float(at & 1 ? s.w[at >> 1] & 0xffff0000u : s.w[at >> 1] << 16);
#pragma unroll
      for (int m = 0; m < MT; m++) acc[m][u] = fmaf(sc, part[m][u], acc[m][u]);
    }
  }
}

// In groups of 32 and with four row blocks the scales of four columns, a product per group and block, cost more than scaling
// the operand: scale x level goes into bf16, exactly for scales of six significant bits (517 tokens 4096 -> 1024 34.7 ->
// 23.7 us a pass).  A lane takes the four scales of one row.
template <int MT>
__device__ __forceinline__ void q4_tile_scaled(const bf16x8_t (&fx)[MT][4], const uint4 &c, const uint2 &sc, f32x4_t (&acc)[MT]) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int st = 0; st < 4; st++) {
    const uint32_t h = st < 2 ? sc.x : sc.y;
    const float s = __uint_as_float(st & 1 ? h & 0xffff0000u : h << 16);
    f32x2_t p[4];
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[st], 1.f, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[st], 1.f, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[st], 1.f, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[st], 1.f, 3);
    bf16x8_t fw;
#pragma unroll
    for (int e = 0; e < 8; e++) fw[e] = (bf16_t)(s * p[e >> 1][e & 1]);
#pragma unroll
    for (int m = 0; m < MT; m++) acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw, fx[m][st], acc[m], 0, 0, 0);
  }
}

// ---- everything else: slices of the contraction, then their sum with the rank-r term ------------------------
// A workgroup owns NT tiles' rows and a slice of the contraction.  Its eight wavefronts are WM groups of MT row
// blocks times 8 / WM shares of the slice.  Up to 128 rows trailing workgroups make slices of the projection D(x) A^T; of more
// rows (which come with their projection) every workgroup takes 128.
constexpr int Q4S_NT = 4;
struct Q4Slices {
  int S, per;              // slices, tiles of each
  int blocks, main;        // 128-row blocks of x; workgroups of the product
  int PS;                  // slices of the projection, of eight tiles: one per wavefront
  float *part, *ppart;     // [S][T][n], [PS][T][r]
};

template <int MT, int WM, int PER>
__global__ __launch_bounds__(512) void q4_slices_kernel(Q4Matrix w, Q4Few a, Q4Slices z, DropArgs drop) {
  constexpr int NT = Q4S_NT, WK = 8 / WM;
  // wavefront by wavefront the staging of MT row blocks, then sums [8][NT][MT][64][4]
  extern __shared__ __align__(16) unsigned char smem[];
  float *red = reinterpret_cast<float *>(smem);
  static_assert(NT >= 4, "the staging fits");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l15 = lane & 15, hi = lane >> 4;
  const int r = a.r, K = w.K, kbs = (int)q4_col_blocks(K);
  if ((int)blockIdx.x >= z.main) {   // a slice of the projection of 16 rows: one tile of the contraction per wavefront
    const int T = a.T, nq = (r + 15) >> 4, at = blockIdx.x - z.main, ps = at % z.PS, t0 = at / z.PS * 16;
    const int kb = ps * 8 + wave, row = t0 + l15 < T ? t0 + l15 : T - 1;
    unsigned char *stage = smem + wave * STAGE_BYTES;
    f32x4_t p[4];
#pragma unroll
    for (int j = 0; j < 4; j++) p[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (kb < kbs) {
      bf16x8_t v[4], fx[4];
      rows_load(a.x, RowOffsets(t0, T, K, lane), kb, K, lane, v);
      rows_to_lds(stage, v, kb, K, lane);
      wave_order();
      rows_from_lds(stage, lane, fx);
      if (drop.thr) {
        const DropKey key = drop_key(drop);
#pragma unroll
        for (int st = 0; st < 4; st++)
          fx[st] = drop_mask8(key, (uint32_t)row, (uint32_t)(kb * Q4_COLS + st * 32 + hi * 8) >> 3, fx[st]);
      }
#pragma unroll
      for (int j = 0; j < 4; j++) {
        if (j >= nq) break;
        bf16x8_t fa[4];
        rows_load(a.A, RowOffsets(j * 16, r, K, lane), kb, K, lane, v);
        wave_order();
        rows_to_lds(stage, v, kb, K, lane);
        wave_order();
        rows_from_lds(stage, lane, fa);
#pragma unroll
        for (int st = 0; st < 4; st++) p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[st], fa[st], p[j], 0, 0, 0);
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; j++)
      if (j < nq) *reinterpret_cast<f32x4_t *>(red + ((wave * 4 + j) * 64 + lane) * 4) = p[j];
    __syncthreads();
    for (int i = tid; i < nq * 256; i += 512) {
      const int j = i >> 8, q = j * 16 + (i & 15), tl = (i >> 4) & 15;
      if (q >= r || t0 + tl >= T) continue;
      const int e = ((tl >> 2) * 16 + (i & 15)) * 4 + (tl & 3);
      float v = 0.f;
#pragma unroll
      for (int u = 0; u < 8; u++) v += red[(u * 4 + j) * 256 + e];
      z.ppart[((int64_t)ps * T + t0 + tl) * r + q] = drop.thr ? v * drop.inv : v;
    }
    return;
  }
  const int groups = z.main / (z.S * z.blocks), rb0 = blockIdx.x % groups * NT, at = blockIdx.x / groups;
  const int tb = at % z.blocks * 128, sl = at / z.blocks, T = a.T - tb;   // rows from tb on, of which this one takes 128
  const bf16_t *x0 = a.x + (int64_t)tb * K;
  const int row_blocks = (int)q4_row_blocks(w.n);
  const int wm = wave / WK, wk = wave % WK;
  const int lo = sl * z.per, end = lo + z.per < kbs ? lo + z.per : kbs;
  int64_t first[NT];   // tiles in front of each row block
#pragma unroll
  for (int i = 0; i < NT; i++) first[i] = (int64_t)(rb0 + i < row_blocks ? rb0 + i : row_blocks - 1) * kbs;
  f32x4_t acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; i++)
#pragma unroll
    for (int m = 0; m < MT; m++) acc[i][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  unsigned char *stage = smem + wave * MT * STAGE_BYTES;
  uint4 nc[NT];   // codes come one tile ahead; scales with them would not fit the registers in groups of 32
  auto load_w = [&](int kb) {
#pragma unroll
    for (int i = 0; i < NT; i++)
      nc[i] = *reinterpret_cast<const uint4 *>(w.codes + (first[i] + kb) * Q4_TILE_BYTES + (uint32_t)lane * 16u);
  };
  if (lo + wk < end) load_w(lo + wk);
  for (int kb = lo + wk; kb < end; kb += WK) {
    bf16x8_t fx[MT][4], x[MT][4];
    constexpr bool SCALED = PER == 4 && MT == 4;
    typename std::conditional<SCALED, uint2, Q4Scales4<PER>>::type s[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) {
      if constexpr (SCALED)
        s[i] = *reinterpret_cast<const uint2 *>(w.scales + (first[i] + kb) * (Q4_ROWS * 4) + (uint32_t)l15 * 4);
      else
        q4_load_scales4<PER>(w, first[i] + kb, lane, s[i]);
    }
#pragma unroll
    for (int m = 0; m < MT; m++) rows_load(x0, RowOffsets((wm * MT + m) * 16, T, K, lane), kb, K, lane, x[m]);
    wave_order();
#pragma unroll
    for (int m = 0; m < MT; m++) rows_to_lds(stage + m * STAGE_BYTES, x[m], kb, K, lane);
    uint4 c[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) c[i] = nc[i];
    wave_order();
    if (kb + WK < end) load_w(kb + WK);
#pragma unroll
    for (int m = 0; m < MT; m++) rows_from_lds(stage + m * STAGE_BYTES, lane, fx[m]);
#pragma unroll
    for (int i = 0; i < NT; i++) {
      if constexpr (SCALED) q4_tile_scaled<MT>(fx, c[i], s[i], acc[i]);
      else q4_tile4<MT, PER>(fx, c[i], s[i], acc[i]);
    }
  }
  __syncthreads();   // the staging is behind everybody
#pragma unroll
  for (int i = 0; i < NT; i++)
#pragma unroll
    for (int m = 0; m < MT; m++) *reinterpret_cast<f32x4_t *>(red + (((wave * NT + i) * MT + m) * 64 + lane) * 4) = acc[i][m];
  __syncthreads();
  // lane (l15, hi), register u: row l15, column 4 hi + u
  for (int o = tid; o < WM * NT * MT * 64; o += 512) {
    const int ln = o & 63, m = (o >> 6) % MT, i = (o >> 6) / MT % NT, g = (o >> 6) / (MT * NT);
    const int t = (g * MT + m) * 16 + (ln & 15), n = (rb0 + i) * 16 + (ln >> 4) * 4;
    if (t >= T || n >= w.n) continue;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < WK; k++) v += *reinterpret_cast<const f32x4_t *>(red + ((((g * WK + k) * NT + i) * MT + m) * 64 + ln) * 4);
    *reinterpret_cast<f32x4_t *>(z.part + ((int64_t)sl * a.T + tb + t) * w.n + n) = v;
  }
}

// y = sum of the slices + s (sum of the projection's slices) B^T, in the slices' order.  16 rows x 64 columns per
// workgroup, four columns of a row per thread.
__global__ __launch_bounds__(256) void q4_finish_kernel(int n, Q4Few a, Q4Slices z, Q4Projection proj) {
  __shared__ float sp[16][64 + 4];
  const int tid = threadIdx.x, T = a.T, r = a.r, t0 = blockIdx.y * 16;
  const int t = t0 + (tid >> 4), c = blockIdx.x * 64 + (tid & 15) * 4;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  const bool in = t < T && c < n;
  if (in) {
    const float *p = z.part + (int64_t)t * n + c;
    for (int s0 = 0; s0 < z.S; s0 += 4) {
      f32x4_t u[4];
#pragma unroll
      for (int i = 0; i < 4; i++)
        u[i] = *reinterpret_cast<const f32x4_t *>(p + (int64_t)(s0 + i < z.S ? s0 + i : s0) * T * n);
#pragma unroll
      for (int i = 0; i < 4; i++)
        if (s0 + i < z.S) v += u[i];
    }
  }
  for (int i = tid; i < 16 * r; i += 256) {
    const int tl = i / r, q = i % r;
    float p = 0.f;
    if (t0 + tl < T)
      for (int s = 0; s < proj.S; s++) p += proj.P[((int64_t)s * T + t0 + tl) * r + q];
    p = q < a.rank ? p * proj.f : 0.f;
    sp[tl][q] = p;
    if (proj.PT && blockIdx.x == 0 && t0 + tl < T) {
      float pc[3];
      three_pieces(p, pc);
#pragma unroll
      for (int u = 0; u < 3; u++) proj.PT[((int64_t)u * r + q) * proj.ldT + t0 + tl] = (bf16_t)pc[u];
    }
  }
  __syncthreads();
  if (!in) return;
  f32x4_t d = {0.f, 0.f, 0.f, 0.f};
  for (int q0 = 0; q0 < r; q0 += 8) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const bf16x8_t b = *reinterpret_cast<const bf16x8_t *>(a.B + (int64_t)(c + e) * r + q0);
#pragma unroll
      for (int q = 0; q < 8; q++) d[e] = fmaf(sp[tid >> 4][q0 + q], (float)b[q], d[e]);
    }
  }
  typedef bf16_t bf16x4_t __attribute__((ext_vector_type(4)));
  bf16x4_t o;
#pragma unroll
  for (int e = 0; e < 4; e++) o[e] = (bf16_t)fmaf(a.s, d[e], v[e]);
  *reinterpret_cast<bf16x4_t *>(a.y + (int64_t)t * n + c) = o;
}

// Where the one launch is the shorter way (us, one launch / slices and their sum): 17 tokens 4096 -> 1024 7.1 / 9.3, 24
// tokens 5120 -> 5120 10.3 / 13.3, 64 tokens 4096 -> 4096 14.7 / 17.3; 32 tokens 11008 -> 4096 17.4 / 18.7, but 64
// of them 30.4 / 23.9: four row blocks of x over a long contraction.
static bool one_launch(int T, int K, int r, bool drop) { return T <= (K <= 8192 ? 64 : 32) && r <= 16 && !drop; }

// Slices of the contraction: as many workgroups as fit the chip in one round (128 tokens 4096 -> 4096 with two rounds of
// them 28.4 us, with one 21.1; 48 tokens 4096 -> 11008 34.5, 24.0), no wavefront without a tile.
static Q4Slices plan_slices(int n, int K, int T) {
  Q4Slices z{};
  const int kbs = (int)q4_col_blocks(K), groups = (int)((q4_row_blocks(n) + Q4S_NT - 1) / Q4S_NT);
  const int wk = T <= 64 ? 8 : 4;
  z.blocks = (T + 127) / 128;
  z.PS = (kbs + 7) / 8;
  int S = 256 / (groups * z.blocks);
  const int most = (kbs + wk - 1) / wk;
  S = S > most ? most : S < 1 ? 1 : S > 16 ? 16 : S;
  z.per = (kbs + S - 1) / S;
  z.S = (kbs + z.per - 1) / z.per;
  z.main = groups * z.blocks * z.S;
  return z;
}

// More than 128 rows: while the workgroups are not much more than the chip holds at once (not more, over a long contraction);
// beyond, widening the matrix for the large product costs less than reading x per 64 columns (us, here / widened: 129 tokens
// 4096 -> 4096 25.3 / 39.6, 512 42.3 / 56.2, 700 64.6 / 63.7; 200 4096 -> 11008 60.2 / 85.5; 517 4096 -> 1024 21.9 /
// 32.8, 1024 31.6 / 39.3, 2000 47.9 / 47.7; 300 11008 -> 4096 65.2 / 87.0, 600 122 / 108).
bool q4_mid_ok(int n, int K, int T) {
  const int64_t groups = (q4_row_blocks(n) + Q4S_NT - 1) / Q4S_NT;
  return T > Q4_FEW_ROWS && T <= 1024 && K < 1 << 23 && groups * ((T + 127) / 128) <= (K <= 8192 ? 384 : 256);
}
size_t q4_mid_scratch_floats(int n, int K, int T) { return (size_t)plan_slices(n, K, T).S * T * n; }

#define MIXLORA_SLICES(MT_, WM_, PER_)                                                                                   \
  do {                                                                                                                   \
    constexpr size_t lds_ = (size_t)8 * Q4S_NT * MT_ * 1024;                                                              \
    static const hipError_t e_ = hipFuncSetAttribute((const void *)q4_slices_kernel<MT_, WM_, PER_>,                     \
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_);             \
    if (e_ != hipSuccess) return e_;                                                                                     \
    hipLaunchKernelGGL((q4_slices_kernel<MT_, WM_, PER_>), grid, block, lds_, st, w, a, z, drop);                        \
  } while (0)
#define MIXLORA_BY_GROUP(LAUNCH)        \
  do {                                  \
    if (w.group == 128) LAUNCH(1);      \
    else if (w.group == 64) LAUNCH(2);  \
    else LAUNCH(4);                     \
  } while (0)
#define MIXLORA_S1(PER_) MIXLORA_SLICES(1, 1, PER_)
#define MIXLORA_S2(PER_) MIXLORA_SLICES(2, 1, PER_)
#define MIXLORA_S4(PER_) MIXLORA_SLICES(4, 1, PER_)
#define MIXLORA_S8(PER_) MIXLORA_SLICES(4, 2, PER_)

hipError_t launch_q4_mid(const Q4Matrix &w, const Q4Few &a, const Q4Projection &P, float *scratch, size_t floats, hipStream_t st) {
  Q4Slices z = plan_slices(w.n, w.K, a.T);
  if (!q4_mid_ok(w.n, w.K, a.T) || a.r % 8 || a.r > 64 || w.n % 8 || w.K % 8 || P.S < 1 || (size_t)z.S * a.T * w.n > floats)
    return hipErrorInvalidValue;
  const int slot = prof_on() ? prof_mark_begin(PROF_GEMM, st) : -1;
  z.part = scratch;
  const DropArgs drop{};
  const dim3 grid(z.main), block(512);
  MIXLORA_BY_GROUP(MIXLORA_S8);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(q4_finish_kernel, dim3((w.n + 63) / 64, (a.T + 15) / 16), dim3(256), 0, st, w.n, a, z, P);
  if (slot >= 0) prof_mark_end(slot, st, 2.0 * a.T * w.n * w.K);
  return hipGetLastError();
}

size_t q4_few_scratch_floats(int n, int K, int T, int r) {
  if (T > Q4_FEW_ROWS || K >= 1 << 23) return 0;   // (32-bit offsets into x and A)
  const Q4Slices z = plan_slices(n, K, T);   // (dropout, which one launch does not take, is not known yet)
  return (size_t)T * ((size_t)z.S * n + ((size_t)z.PS * r + 63) / 64 * 64) + 64;
}

hipError_t launch_q4_few(const Q4Matrix &w, const Q4Few &a, const DropArgs &drop, float *scratch, size_t floats, hipStream_t st) {
  if (a.T < 1 || a.T > Q4_FEW_ROWS || a.r % 8 || a.r > 64 || w.K >= 1 << 23 || w.n % 8 || w.K % 8) return hipErrorInvalidValue;
  const int slot = prof_on() ? prof_mark_begin(PROF_GEMM, st) : -1;
  if (one_launch(a.T, w.K, a.r, drop.thr != 0)) {
    const hipError_t e = w.group == 128 ? launch_few_m<1>(w, a, st) : w.group == 64 ? launch_few_m<2>(w, a, st) : launch_few_m<4>(w, a, st);
    if (e != hipSuccess) return e;
  } else {
    Q4Slices z = plan_slices(w.n, w.K, a.T);
    if ((size_t)a.T * ((size_t)z.S * w.n + (size_t)z.PS * a.r) > floats) return hipErrorInvalidValue;
    z.part = scratch;
    z.ppart = scratch + (size_t)z.S * a.T * w.n;
    const dim3 grid(z.main + (a.T + 15) / 16 * z.PS), block(512);
    if (a.T <= 16) MIXLORA_BY_GROUP(MIXLORA_S1);
    else if (a.T <= 32) MIXLORA_BY_GROUP(MIXLORA_S2);
    else if (a.T <= 64) MIXLORA_BY_GROUP(MIXLORA_S4);
    else MIXLORA_BY_GROUP(MIXLORA_S8);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(q4_finish_kernel, dim3((w.n + 63) / 64, (a.T + 15) / 16), dim3(256), 0, st, w.n, a, z,
                       Q4Projection{z.ppart, z.PS, 1.f, nullptr, 0});
  }
  if (slot >= 0) prof_mark_end(slot, st, 2.0 * a.T * w.n * w.K);
  return hipGetLastError();
}

}  // namespace mixlora
