// Products of few rows (up to 128) with a 4-bit frozen matrix, and the rank-r term of a LoRA linear on it:
//   y = x W'^T + s (D(x) A^T) B^T.
// Bound by reading the codes once.  Codes go from memory to registers as a wavefront's MFMA operand (q4.h) and
// are widened there, two per instruction; levels are exact in bf16, so x times level is summed in fp32 as it is
// and a group's sum is multiplied by the group's scale in fp32: nothing is rounded before y.
#include "q4.h"
#include "q4_few.h"
#include "dropout.h"

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

// 32 inputs per step of a row block's operand, zeros past K
__device__ __forceinline__ void load_rows(const bf16_t *row, int k0, int hi, int K, bf16x8_t (&f)[4]) {
#pragma unroll
  for (int st = 0; st < 4; st++) {
    const int k = k0 + st * 32 + hi * 8;
    f[st] = *reinterpret_cast<const bf16x8_t *>(row + (k < K ? k : 0));
  }
}
__device__ __forceinline__ void zero_past(int k0, int hi, int K, bf16x8_t (&f)[4]) {
#pragma unroll
  for (int st = 0; st < 4; st++)
    if (k0 + st * 32 + hi * 8 >= K) {
#pragma unroll
      for (int e = 0; e < 8; e++) f[st][e] = (bf16_t)0.f;
    }
}

// ---- up to 16 rows, rank up to 16, no dropout: one launch ---------------------------------------------
// A workgroup owns NT tiles' rows (16 NT columns of y) over the whole contraction, its eight wavefronts every
// eighth tile of it, two tiles ahead of the one in use.  Every workgroup makes the projection x A^T itself (128
// KB of A at 16 x 4096, out of L2): that costs less than a launch in front of this one.
template <int NT, int PER>
__global__ __launch_bounds__(512) void q4_few_kernel(Q4Matrix w, Q4Few a) {
  constexpr int WAVES = 8, UN = 2;
  __shared__ float red[WAVES][NT + 1][64][4];
  __shared__ float sp[16][17];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l15 = lane & 15, hi = lane >> 4;
  const int rb0 = blockIdx.x * NT, row_blocks = (int)q4_row_blocks(w.n), kbs = (int)q4_col_blocks(w.K);
  const int T = a.T, r = a.r, K = w.K;
  // what the end needs of B: column col of tile i for token tok
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
  const bf16_t *xr = a.x + (int64_t)(l15 < T ? l15 : T - 1) * K;
  const bf16_t *ar = a.A + (int64_t)(l15 < r ? l15 : r - 1) * K;
  const unsigned char *cr[NT];
  const bf16_t *sr[NT];
#pragma unroll
  for (int i = 0; i < NT; i++) {
    const int64_t first = (int64_t)(rb0 + i < row_blocks ? rb0 + i : row_blocks - 1) * kbs;
    cr[i] = w.codes + first * Q4_TILE_BYTES + 16 * lane;
    sr[i] = w.scales + (first * Q4_ROWS + l15) * PER;
  }
  f32x4_t acc[NT][1], accp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NT; i++) acc[i][0] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  struct Block {
    bf16x8_t fx[1][4], fa[4];
    uint4 c[NT];
    float s[NT][PER];
  };
  auto load = [&](int kb, Block &b) {
    const int kc = kb < kbs ? kb : kbs - 1;
#pragma unroll
    for (int i = 0; i < NT; i++) {
      b.c[i] = *reinterpret_cast<const uint4 *>(cr[i] + (int64_t)kc * Q4_TILE_BYTES);
      q4_load_scales<PER>(sr[i] + (int64_t)kc * Q4_ROWS * PER, b.s[i]);
    }
    load_rows(xr, kc * Q4_COLS, hi, K, b.fx[0]);
    load_rows(ar, kc * Q4_COLS, hi, K, b.fa);
  };
  auto use = [&](int kb, Block &b) {
    if (kb >= kbs) return;   // (wavefront-uniform)
    if (kb == kbs - 1) {
      zero_past(kb * Q4_COLS, hi, K, b.fx[0]);
      zero_past(kb * Q4_COLS, hi, K, b.fa);
    }
#pragma unroll
    for (int st = 0; st < 4; st++) accp = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.fx[0][st], b.fa[st], accp, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NT; i++) q4_tile<1, PER>(b.fx, b.c[i], b.s[i], acc[i]);
  };
  Block cur[UN], nxt[UN];
#pragma unroll
  for (int u = 0; u < UN; u++) load(wave + u * WAVES, cur[u]);
  for (int kb = wave; kb < kbs; kb += UN * WAVES) {
#pragma unroll
    for (int u = 0; u < UN; u++) load(kb + (UN + u) * WAVES, nxt[u]);
#pragma unroll
    for (int u = 0; u < UN; u++) use(kb + u * WAVES, cur[u]);
#pragma unroll
    for (int u = 0; u < UN; u++) cur[u] = nxt[u];
  }
  // lane (l15, hi), register u: row 4 hi + u, column l15
#pragma unroll
  for (int i = 0; i < NT; i++) *reinterpret_cast<f32x4_t *>(red[wave][i][lane]) = acc[i][0];
  *reinterpret_cast<f32x4_t *>(red[wave][NT][lane]) = accp;
  __syncthreads();
  const int ln = (tok >> 2) * 16 + col, u = tok & 3;
  if (tid < 256) {
    float v = red[0][NT][ln][u];
#pragma unroll
    for (int q = 1; q < WAVES; q++) v += red[q][NT][ln][u];
    sp[tok][col] = col < r ? v : 0.f;
  }
  __syncthreads();
  if (tok >= T) return;
#pragma unroll
  for (int o = 0; o < OUT; o++) {
    const int i = half + 2 * o, n = (rb0 + i) * 16 + col;
    if (i >= NT || n >= w.n) continue;
    float v = red[0][i][ln][u], p = 0.f;
#pragma unroll
    for (int q = 1; q < WAVES; q++) v += red[q][i][ln][u];
#pragma unroll
    for (int q = 0; q < 8; q++) p = fmaf(sp[tok][q], (float)bq[o][0][q], p);
    if (r > 8) {
#pragma unroll
      for (int q = 0; q < 8; q++) p = fmaf(sp[tok][8 + q], (float)bq[o][1][q], p);
    }
    a.y[(int64_t)tok * w.n + n] = (bf16_t)fmaf(a.s, p, v);
  }
}

// ---- everything else up to 128 rows: slices of the contraction, then their sum with the rank-r term --------
// A workgroup owns NT tiles' rows and a slice of the contraction.  Its eight wavefronts are WM groups of MT row
// blocks times 8 / WM shares of the slice.  Trailing workgroups make slices of the projection D(x) A^T.
constexpr int Q4S_NT = 4;
struct Q4Slices {
  int S, per;              // slices, tiles of each
  int main;                // workgroups of the product
  int PS, pper;            // slices of the projection, in tiles (at most 8: one per wavefront)
  float *part, *ppart;     // [S][T][n], [PS][T][r]
};

template <int MT, int WM, int PER>
__global__ __launch_bounds__(512) void q4_slices_kernel(Q4Matrix w, Q4Few a, Q4Slices z, DropArgs drop) {
  constexpr int NT = Q4S_NT, WK = 8 / WM;
  extern __shared__ __align__(16) float red[];   // [8][NT][MT][64][4]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l15 = lane & 15, hi = lane >> 4;
  const int T = a.T, r = a.r, K = w.K, kbs = (int)q4_col_blocks(K);
  if ((int)blockIdx.x >= z.main) {   // a slice of the projection of 16 rows: one tile of the contraction per wavefront
    const int nq = (r + 15) >> 4, at = blockIdx.x - z.main, ps = at % z.PS, t0 = at / z.PS * 16;
    const int kb = ps * 8 + wave, row = t0 + l15 < T ? t0 + l15 : T - 1;
    bf16x8_t fx[4];
    if (kb < kbs) {
      load_rows(a.x + (int64_t)row * K, kb * Q4_COLS, hi, K, fx);
      if (drop.thr) {
        const DropKey key = drop_key(drop);
#pragma unroll
        for (int st = 0; st < 4; st++)
          fx[st] = drop_mask8(key, (uint32_t)row, (uint32_t)(kb * Q4_COLS + st * 32 + hi * 8) >> 3, fx[st]);
      }
      zero_past(kb * Q4_COLS, hi, K, fx);
    }
    for (int j = 0; j < nq; j++) {
      f32x4_t p = {0.f, 0.f, 0.f, 0.f};
      if (kb < kbs) {
        bf16x8_t fa[4];
        const int q = j * 16 + l15;
        load_rows(a.A + (int64_t)(q < r ? q : r - 1) * K, kb * Q4_COLS, hi, K, fa);
        zero_past(kb * Q4_COLS, hi, K, fa);
#pragma unroll
        for (int st = 0; st < 4; st++) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[st], fa[st], p, 0, 0, 0);
      }
      *reinterpret_cast<f32x4_t *>(red + ((wave * 4 + j) * 64 + lane) * 4) = p;
    }
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
  const int groups = z.main / z.S, rb0 = blockIdx.x % groups * NT, sl = blockIdx.x / groups;
  const int row_blocks = (int)q4_row_blocks(w.n);
  const int wm = wave / WK, wk = wave % WK;
  const int lo = sl * z.per, end = lo + z.per < kbs ? lo + z.per : kbs;
  const bf16_t *xr[MT];
#pragma unroll
  for (int m = 0; m < MT; m++) {
    const int t = (wm * MT + m) * 16 + l15;
    xr[m] = a.x + (int64_t)(t < T ? t : T - 1) * K;
  }
  const unsigned char *cr[NT];
  const bf16_t *sr[NT];
#pragma unroll
  for (int i = 0; i < NT; i++) {
    const int64_t first = (int64_t)(rb0 + i < row_blocks ? rb0 + i : row_blocks - 1) * kbs;
    cr[i] = w.codes + first * Q4_TILE_BYTES + 16 * lane;
    sr[i] = w.scales + (first * Q4_ROWS + l15) * PER;
  }
  f32x4_t acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; i++)
#pragma unroll
    for (int m = 0; m < MT; m++) acc[i][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int kb = lo + wk; kb < end; kb += WK) {
    uint4 c[NT];
    float s[NT][PER];
    bf16x8_t fx[MT][4];
#pragma unroll
    for (int i = 0; i < NT; i++) {
      c[i] = *reinterpret_cast<const uint4 *>(cr[i] + (int64_t)kb * Q4_TILE_BYTES);
      q4_load_scales<PER>(sr[i] + (int64_t)kb * Q4_ROWS * PER, s[i]);
    }
#pragma unroll
    for (int m = 0; m < MT; m++) load_rows(xr[m], kb * Q4_COLS, hi, K, fx[m]);
    if (kb == kbs - 1) {
#pragma unroll
      for (int m = 0; m < MT; m++) zero_past(kb * Q4_COLS, hi, K, fx[m]);
    }
#pragma unroll
    for (int i = 0; i < NT; i++) q4_tile<MT, PER>(fx, c[i], s[i], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < NT; i++)
#pragma unroll
    for (int m = 0; m < MT; m++) *reinterpret_cast<f32x4_t *>(red + (((wave * NT + i) * MT + m) * 64 + lane) * 4) = acc[i][m];
  __syncthreads();
  // four columns of a token per thread: 16 threads write 64 columns of it
  for (int o = tid; o < WM * MT * 16 * (NT * 4); o += 512) {
    const int c4 = o % (NT * 4), t = o / (NT * 4), i = c4 >> 2, c0 = (c4 & 3) * 4;
    const int n = (rb0 + i) * 16 + c0;
    if (t >= T || n >= w.n) continue;
    const int g = t / (16 * MT), m = t / 16 % MT, tl = t & 15;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < WK; k++) {
      const float *p = red + ((((g * WK + k) * NT + i) * MT + m) * 64 + (tl >> 2) * 16 + c0) * 4 + (tl & 3);
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] += p[4 * e];
    }
    *reinterpret_cast<f32x4_t *>(z.part + ((int64_t)sl * T + t) * w.n + n) = v;
  }
}

// y = sum of the slices + s (sum of the projection's slices) B^T, in the slices' order.  16 rows x 64 columns per
// workgroup, four columns of a row per thread.
__global__ __launch_bounds__(256) void q4_finish_kernel(int n, Q4Few a, Q4Slices z) {
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
      for (int s = 0; s < z.PS; s++) p += z.ppart[((int64_t)s * T + t0 + tl) * r + q];
    sp[tl][q] = p;
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

static bool one_launch(int T, int r, bool drop) { return T <= 16 && r <= 16 && !drop; }

// Slices of the contraction: enough workgroups for the chip twice, no wavefront without a tile.
static Q4Slices plan_slices(int n, int K, int T, int r) {
  Q4Slices z{};
  const int kbs = (int)q4_col_blocks(K), groups = (int)((q4_row_blocks(n) + Q4S_NT - 1) / Q4S_NT);
  const int wk = T <= 64 ? 8 : 4;
  int S = (512 + groups - 1) / groups;
  const int most = (kbs + wk - 1) / wk;
  S = S > most ? most : S < 1 ? 1 : S > 16 ? 16 : S;
  z.per = (kbs + S - 1) / S;
  z.S = (kbs + z.per - 1) / z.per;
  z.main = groups * z.S;
  z.PS = (kbs + 7) / 8;
  return z;
}

size_t q4_few_scratch_floats(int n, int K, int T, int r) {
  if (T > Q4_FEW_ROWS) return 0;
  const Q4Slices z = plan_slices(n, K, T, r);   // (dropout, which one launch does not take, is not known yet)
  return (size_t)T * ((size_t)z.S * n + ((size_t)z.PS * r + 63) / 64 * 64) + 64;
}

hipError_t launch_q4_few(const Q4Matrix &w, const Q4Few &a, const DropArgs &drop, float *scratch, size_t floats, hipStream_t st) {
  if (a.T < 1 || a.T > Q4_FEW_ROWS || a.r % 8 || a.r > 64 || w.n % 8 || w.K % 8) return hipErrorInvalidValue;
  const int slot = prof_on() ? prof_mark_begin(PROF_GEMM, st) : -1;
  const int tiles = (int)q4_row_blocks(w.n);
#define MIXLORA_BY_GROUP(LAUNCH)        \
  do {                                  \
    if (w.group == 128) LAUNCH(1);      \
    else if (w.group == 64) LAUNCH(2);  \
    else LAUNCH(4);                     \
  } while (0)
  if (one_launch(a.T, a.r, drop.thr != 0)) {
#define MIXLORA_FEW(NT_, PER_) \
  hipLaunchKernelGGL((q4_few_kernel<NT_, PER_>), dim3((tiles + NT_ - 1) / NT_), dim3(512), 0, st, w, a)
#define MIXLORA_FEW1(PER_) MIXLORA_FEW(1, PER_)
#define MIXLORA_FEW2(PER_) MIXLORA_FEW(2, PER_)
#define MIXLORA_FEW3(PER_) MIXLORA_FEW(3, PER_)
    if (tiles <= 320) MIXLORA_BY_GROUP(MIXLORA_FEW1);
    else if (tiles <= 512) MIXLORA_BY_GROUP(MIXLORA_FEW2);
    else MIXLORA_BY_GROUP(MIXLORA_FEW3);
  } else {
    Q4Slices z = plan_slices(w.n, w.K, a.T, a.r);
    if ((size_t)a.T * ((size_t)z.S * w.n + (size_t)z.PS * a.r) > floats) return hipErrorInvalidValue;
    z.part = scratch;
    z.ppart = scratch + (size_t)z.S * a.T * w.n;
    const dim3 grid(z.main + (a.T + 15) / 16 * z.PS), block(512);
#define MIXLORA_SLICES(MT_, WM_, PER_)                                                                                   \
  do {                                                                                                                   \
    constexpr size_t lds_ = (size_t)8 * Q4S_NT * MT_ * 1024;                                                              \
    static const hipError_t e_ = hipFuncSetAttribute((const void *)q4_slices_kernel<MT_, WM_, PER_>,                     \
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_);             \
    if (e_ != hipSuccess) return e_;                                                                                     \
    hipLaunchKernelGGL((q4_slices_kernel<MT_, WM_, PER_>), grid, block, lds_, st, w, a, z, drop);                        \
  } while (0)
#define MIXLORA_S1(PER_) MIXLORA_SLICES(1, 1, PER_)
#define MIXLORA_S2(PER_) MIXLORA_SLICES(2, 1, PER_)
#define MIXLORA_S4(PER_) MIXLORA_SLICES(4, 1, PER_)
#define MIXLORA_S8(PER_) MIXLORA_SLICES(4, 2, PER_)
    if (a.T <= 16) MIXLORA_BY_GROUP(MIXLORA_S1);
    else if (a.T <= 32) MIXLORA_BY_GROUP(MIXLORA_S2);
    else if (a.T <= 64) MIXLORA_BY_GROUP(MIXLORA_S4);
    else MIXLORA_BY_GROUP(MIXLORA_S8);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(q4_finish_kernel, dim3((w.n + 63) / 64, (a.T + 15) / 16), dim3(256), 0, st, w.n, a, z);
  }
  if (slot >= 0) prof_mark_end(slot, st, 2.0 * a.T * w.n * w.K);
  return hipGetLastError();
}

}  // namespace mixlora
