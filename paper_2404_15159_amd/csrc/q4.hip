// 4-bit frozen matrices: quantization and back (layout: q4.h).
#include "q4.h"

namespace mixlora {

typedef bf16_t bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// ---- to codes ---------------------------------------------------------------------------------------
// scale = the smallest number of six significant bits that is at least most / 6 (most: the group's largest
// magnitude), so that scale x level has at most eight and is exact in bf16, whichever path widens it; 0 where
// most < 2^-100, NaN where most >= 2^127 or is not a number.  A code is the nearest level, ties to the even
// code, found by comparing |w| with (midpoint x scale): those products are exact in fp32, a quotient w / scale
// would be rounded and could cross a midpoint.
__device__ __forceinline__ float q4_scale(uint32_t most_bits) {
  if (most_bits >= 0x7f000000u) return __uint_as_float(0x7fc00000u);
  if (most_bits < 0x0d800000u) return 0.f;
  const float most = __uint_as_float(most_bits);
  constexpr uint32_t LOW = (1u << 18) - 1;
  uint32_t b = (__float_as_uint(most / 6.f) + LOW) & ~LOW;
  if (6.f * __uint_as_float(b) < most) b += LOW + 1;   // (the quotient was rounded down onto such a number)
  return __uint_as_float(b);
}
// (a bisection: the midpoints in order are 1/4, 3/4, 5/4, 7/4, 5/2, 7/2, 5, and a tie goes up at every second one)
__device__ __forceinline__ uint32_t q4_code(float w, float s) {
  const float a = fabsf(w);
  const bool b2 = a >= 1.75f * s;
  const bool b1 = a >= (b2 ? 3.5f * s : 0.75f * s);
  const bool b0 = a > (b2 ? (b1 ? 5.f * s : 2.5f * s) : (b1 ? 1.25f * s : 0.25f * s));
  const uint32_t c = (b2 ? 4u : 0u) + (b1 ? 2u : 0u) + (b0 ? 1u : 0u);
  return s == 0.f ? 0u : c | (w < 0.f && c ? 8u : 0u);
}

// Eight codes of bf16 weights by the hardware's conversion (nearest, ties to even) of the quotients.  It needs them right at
// the midpoints only: w has 8 significant bits and midpoint x scale at most 9, so they differ by 2^-9 or not at all, and in
// that case the corrected quotient is the midpoint itself (w - q s is exact, so q + (w - q s) / s is rounded once, and the
// midpoint needs no rounding).  For 24 bits that does not hold.
__device__ __forceinline__ uint32_t q4_codes_bf16(const float (&w)[8], float s) {
  const float r = __builtin_amdgcn_rcpf(s);
  uint32_t word = 0;
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; e++) {
    const float q0 = w[e] * r;
    q[e] = fmaf(fmaf(-q0, s, w[e]), r, q0);
  }
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[0], q[1], 1.f, 0);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[2], q[3], 1.f, 1);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[4], q[5], 1.f, 2);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[6], q[7], 1.f, 3);
  word &= 0x77777777u | ((word | word >> 1 | word >> 2) & 0x11111111u) << 3;   // a magnitude of 0 has no sign
  return s > 0.f ? word : 0u;
}
template <typename E> __device__ __forceinline__ uint32_t q4_codes(const float (&w)[8], float s) {
  uint32_t word = 0;
#pragma unroll
  for (int e = 0; e < 8; e++) word |= q4_code(w[e], s) << (4 * e);
  return word;
}
template <> __device__ __forceinline__ uint32_t q4_codes<bf16_t>(const float (&w)[8], float s) { return q4_codes_bf16(w, s); }

// Bound by reading W once.  A wavefront owns a tile; four neighbouring lanes have 64 bytes of a row between them (in bf16),
// four times over, and what a lane has is what it writes: the 16 bytes of its row and quarter.
template <typename E, int PER>
__global__ __launch_bounds__(256) void q4_quantize_kernel(const E *__restrict__ W, int n, int K,
                                                          unsigned char *__restrict__ codes,
                                                          bf16_t *__restrict__ scales) {
  const int lane = threadIdx.x & 63, i = lane >> 2, h = lane & 3;
  const int64_t kt = q4_col_blocks(K), tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= q4_row_blocks(n) * kt) return;
  const int row = (int)(tile / kt) * Q4_ROWS + i, k0 = (int)(tile % kt) * Q4_COLS;
  const bool whole = row < n && k0 + Q4_COLS <= K;
  const E *src = W + (int64_t)(row < n ? row : n - 1) * K;
  Vec8<E> v[4];
#pragma unroll
  for (int b = 0; b < 4; b++) {
    const int k = k0 + 32 * b + 8 * h;
    v[b].load(src + (k < K ? k : 0));
  }
  float w[4][8];
  uint32_t most[4];
#pragma unroll
  for (int b = 0; b < 4; b++) {
    const bool in = whole || (row < n && k0 + 32 * b + 8 * h < K);   // K is a multiple of 8
    most[b] = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      w[b][e] = in ? v[b].get(e) : 0.f;
      const uint32_t bits = __float_as_uint(w[b][e]) & 0x7fffffffu;
      most[b] = bits > most[b] ? bits : most[b];
    }
  }
  uint32_t word[4];
#pragma unroll
  for (int g = 0; g < PER; g++) {
    constexpr int STEPS = 4 / PER;
    uint32_t m = most[g * STEPS];
#pragma unroll
    for (int b = 1; b < STEPS; b++) m = most[g * STEPS + b] > m ? most[g * STEPS + b] : m;
    uint32_t o = __builtin_amdgcn_update_dpp(0, m, 0xb1, 0xf, 0xf, true);   // quad_perm 1 0 3 2
    m = o > m ? o : m;
    o = __builtin_amdgcn_update_dpp(0, m, 0x4e, 0xf, 0xf, true);            // quad_perm 2 3 0 1
    m = o > m ? o : m;
    const float s = q4_scale(m);
#pragma unroll
    for (int b = g * STEPS; b < (g + 1) * STEPS; b++) word[b] = q4_codes<E>(w[b], s);
    if (h == 0) scales[(tile * Q4_ROWS + i) * PER + g] = (bf16_t)s;
  }
  *reinterpret_cast<uint4 *>(codes + tile * Q4_TILE_BYTES + 16 * (16 * h + i)) = uint4{word[0], word[1], word[2], word[3]};
}
template <typename E>
static hipError_t launch_quantize(const void *W, int n, int K, const mixlora_q4 &q, hipStream_t st) {
  const int64_t tiles = q4_row_blocks(n) * q4_col_blocks(K);
  const dim3 grid((unsigned)((tiles + 3) / 4)), block(256);
#define MIXLORA_QUANTIZE(PER_)                                                                                 \
  hipLaunchKernelGGL((q4_quantize_kernel<E, PER_>), grid, block, 0, st, (const E *)W, n, K, (unsigned char *)q.codes, \
                     (bf16_t *)q.scales)
  if (q.group == 128) MIXLORA_QUANTIZE(1);
  else if (q.group == 64) MIXLORA_QUANTIZE(2);
  else MIXLORA_QUANTIZE(4);
#undef MIXLORA_QUANTIZE
  return hipGetLastError();
}

// ---- and back ---------------------------------------------------------------------------------------
__device__ __forceinline__ void q4_widen8(uint32_t word, float s, float (&v)[8]) {
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.f, 3);
  v[0] = s * a[0], v[1] = s * a[1], v[2] = s * b[0], v[3] = s * b[1];
  v[4] = s * c[0], v[5] = s * c[1], v[6] = s * d[0], v[7] = s * d[1];
}

// Bound by writing the result.  A wavefront owns a tile.
template <typename E>
__global__ __launch_bounds__(256) void q4_dequantize_kernel(Q4Matrix w, E *__restrict__ out) {
  const int lane = threadIdx.x & 63, i = lane & 15, h = lane >> 4;
  const int64_t kt = q4_col_blocks(w.K), tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= q4_row_blocks(w.n) * kt) return;
  const int row = (int)(tile / kt) * Q4_ROWS + i, k0 = (int)(tile % kt) * Q4_COLS, per = Q4_COLS / w.group;
  const uint4 c = *reinterpret_cast<const uint4 *>(w.codes + tile * Q4_TILE_BYTES + 16 * lane);
  const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int b = 0; b < 4; b++) {
    const int k = k0 + 32 * b + 8 * h;
    const float s = (float)w.scales[(tile * Q4_ROWS + i) * per + 32 * b / w.group];
    float v[8];
    q4_widen8(word[b], s, v);
    Vec8<E> o;
#pragma unroll
    for (int e = 0; e < 8; e++) o.set(e, v[e]);
    if (row < w.n && k < w.K) o.store(out + (int64_t)row * w.K + k);
  }
}

// Transposed: a workgroup widens four tiles of 64 rows, whose columns are then rows of the result, through
// LDS (pitch 64 + 8 elements).
template <typename E>
__global__ __launch_bounds__(256) void q4_dequantize_T_kernel(Q4Matrix w, E *__restrict__ out) {
  constexpr int R = 4 * Q4_ROWS, PITCH = R + 8;
  __shared__ __align__(16) E buf[Q4_COLS][PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, h = lane >> 4;
  const int64_t kt = q4_col_blocks(w.K), nt = q4_row_blocks(w.n), groups = (nt + 3) / 4;
  const int64_t at = blockIdx.x, cb = at / groups, rb = (at % groups) * 4 + wave;
  const int64_t tile = (rb < nt ? rb : nt - 1) * kt + cb;
  const int k0 = (int)cb * Q4_COLS, row0 = (int)(at % groups) * R, per = Q4_COLS / w.group;
  const uint4 c = *reinterpret_cast<const uint4 *>(w.codes + tile * Q4_TILE_BYTES + 16 * lane);
  const uint32_t word[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int b = 0; b < 4; b++) {
    const float s = (float)w.scales[(tile * Q4_ROWS + i) * per + 32 * b / w.group];
    float v[8];
    q4_widen8(word[b], s, v);
#pragma unroll
    for (int e = 0; e < 8; e++) buf[32 * b + 8 * h + e][wave * Q4_ROWS + i] = from_f32<E>(v[e]);
  }
  __syncthreads();
  for (int p = threadIdx.x; p < Q4_COLS * (R / 8); p += 256) {
    const int k = p / (R / 8), n = p % (R / 8) * 8;
    if (k0 + k < w.K && row0 + n < w.n) {   // n is a multiple of 8
      Vec8<E> o;
      o.load(&buf[k][n]);
      o.store(out + (int64_t)(k0 + k) * w.n + row0 + n);
    }
  }
}

hipError_t launch_q4_dequantize(const Q4Matrix &w, bool transposed, int dtype, void *out, hipStream_t st) {
  const int64_t tiles = q4_row_blocks(w.n) * q4_col_blocks(w.K);
  const dim3 grid((unsigned)(transposed ? (q4_row_blocks(w.n) + 3) / 4 * q4_col_blocks(w.K) : (tiles + 3) / 4)), block(256);
  const int slot = prof_on() ? prof_mark_begin(PROF_OTHER, st) : -1;
  if (transposed && dtype == MIXLORA_BF16)
    hipLaunchKernelGGL(q4_dequantize_T_kernel<bf16_t>, grid, block, 0, st, w, (bf16_t *)out);
  else if (transposed)
    hipLaunchKernelGGL(q4_dequantize_T_kernel<float>, grid, block, 0, st, w, (float *)out);
  else if (dtype == MIXLORA_BF16)
    hipLaunchKernelGGL(q4_dequantize_kernel<bf16_t>, grid, block, 0, st, w, (bf16_t *)out);
  else
    hipLaunchKernelGGL(q4_dequantize_kernel<float>, grid, block, 0, st, w, (float *)out);
  if (slot >= 0) prof_mark_end(slot, st, (double)w.n * w.K * (dtype == MIXLORA_BF16 ? 2.5 : 4.5));
  return hipGetLastError();
}

}  // namespace mixlora

using namespace mixlora;

namespace {
inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
int check_matrix(int32_t d_out, int32_t d_in, int32_t group) {
  if (d_out < 8 || d_in < 8 || d_out % 8 || d_in % 8 || !q4_group_ok(group)) return MIXLORA_E_SHAPE;
  if (q4_row_blocks(d_out) * q4_col_blocks(d_in) >= (1ll << 31)) return MIXLORA_E_SHAPE;   // a tile per wavefront
  return MIXLORA_OK;
}
}  // namespace

extern "C" {

size_t mixlora_q4_code_bytes(int32_t d_out, int32_t d_in) {
  return check_matrix(d_out, d_in, 128) ? 0 : q4_code_bytes(d_out, d_in);
}

size_t mixlora_q4_scale_bytes(int32_t d_out, int32_t d_in, int32_t group) {
  return check_matrix(d_out, d_in, group) ? 0 : q4_scale_bytes(d_out, d_in, group);
}

int mixlora_q4_quantize(const void *W, int32_t dtype, int32_t d_out, int32_t d_in, const mixlora_q4 *q4,
                        void *stream) {
  if (!q4 || !W || !q4->codes || !q4->scales) return MIXLORA_E_NULL;
  if (dtype != MIXLORA_F32 && dtype != MIXLORA_BF16) return MIXLORA_E_DTYPE;
  const int rc = check_matrix(d_out, d_in, q4->group);
  if (rc) return rc;
  if (misaligned(W) || misaligned(q4->codes) || misaligned(q4->scales)) return MIXLORA_E_ALIGN;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const hipError_t e = dtype == MIXLORA_BF16 ? launch_quantize<bf16_t>(W, d_out, d_in, *q4, st)
                                             : launch_quantize<float>(W, d_out, d_in, *q4, st);
  return e == hipSuccess ? MIXLORA_OK : MIXLORA_E_HIP;
}

int mixlora_q4_dequantize(const mixlora_q4 *q4, int32_t d_out, int32_t d_in, int32_t transposed, void *W,
                          int32_t dtype, void *stream) {
  if (!q4 || !W || !q4->codes || !q4->scales) return MIXLORA_E_NULL;
  if (dtype != MIXLORA_F32 && dtype != MIXLORA_BF16) return MIXLORA_E_DTYPE;
  const int rc = check_matrix(d_out, d_in, q4->group);
  if (rc) return rc;
  if (transposed != 0 && transposed != 1) return MIXLORA_E_SHAPE;
  if (misaligned(W) || misaligned(q4->codes) || misaligned(q4->scales)) return MIXLORA_E_ALIGN;
  const Q4Matrix m{(const unsigned char *)q4->codes, (const bf16_t *)q4->scales, d_out, d_in, q4->group};
  return launch_q4_dequantize(m, transposed != 0, dtype, W, reinterpret_cast<hipStream_t>(stream)) == hipSuccess
             ? MIXLORA_OK : MIXLORA_E_HIP;
}

}  // extern "C"
