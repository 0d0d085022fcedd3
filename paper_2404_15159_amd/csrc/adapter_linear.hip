// LoRA linear with dropout on the adapter's input, on an ordinary or on a 4-bit frozen matrix:
//   y = x W^T + s (D(x) A^T) B^T,   dx = dy W + D'(s (dy B) A),   dA = s (dy B)^T D(x),   dB = s dy^T (D(x) A^T)
// D drops elements and scales the others (dropout.h makes the mask from counters wherever it is needed), D' drops the
// same ones.  bf16: the projection on the rank-r side is made first and rides in the frozen product as an extra K segment,
// in three bf16 pieces that hold all of its 24 bits; the backward's, which has to be masked with dropout, goes first and is
// masked in the accumulators.  The gradient sums take the rank-r factor in three pieces as well.  A 4-bit matrix is widened
// into the workspace, which rounds nothing with scales of six bits (q4.h), but for the forward of few rows, which multiplies
// with the codes (q4_few.hip).  fp32: the forward makes D(x) in the workspace for both directions, and the products are the fp32 ones.
#include "common.h"
#include "q4.h"
#include "q4_few.h"
#include "dropout.h"
#include "rows_stage.h"

#include <cmath>
#include <initializer_list>

using namespace mixlora;

namespace {

constexpr size_t ALIGN = 256;
inline size_t up(size_t v) { return (v + ALIGN - 1) / ALIGN * ALIGN; }
inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

struct Layout {
  int rp, ldT;                            // rank rounded up to a multiple of 8; pitch of the transposed factors
  size_t padA, padB, P, P_T, offs, xd;    // kept for the backward
  size_t ext, ext_B, proj, gemm_part;     // scratch of either direction
  size_t W, fwd_end;
  size_t W_T, Bt, At, V, V_T, dx32, partials, padgA, padgB, bwd_end;
  size_t few;                             // partial sums of the few-rows product
  size_t gemm_floats, partial_floats, few_floats, mid_floats;
};

size_t project_floats(int T, int K, int r);   // partial sums of a projection

// q4: room for the widened matrix.  The scratch of the two directions overlaps.
Layout make_layout(const mixlora_linear_dims &D, bool q4) {
  Layout L{};
  const size_t T = D.T, di = D.d_in, dn = D.d_out, r = (D.r + 7) & ~7;
  const bool bf16 = D.dtype == MIXLORA_BF16, padded = (int)r != D.r;
  const size_t E = bf16 ? 2 : 4, wide = di > dn ? di : dn;
  size_t o = 0;
  auto take = [&](size_t bytes) { size_t at = o; o = up(o + bytes); return at; };
  L.rp = (int)r;
  L.ldT = (int)((T + 15) / 16 * 16 + 16);
  L.padA = take(padded ? r * di * E : 0);
  L.padB = take(padded ? dn * r * E : 0);
  L.P = take(T * r * 4);
  L.P_T = take(bf16 ? 3 * r * L.ldT * 2 : 0);
  L.offs = take(2 * 4);
  L.xd = take(bf16 ? 0 : T * di * E);
  L.ext = take(bf16 ? T * 3 * r * 2 : 0);
  L.ext_B = take(bf16 ? wide * 3 * r * 2 : 0);
  {
    const size_t fx = project_floats(D.T, D.d_in, (int)r), fdy = project_floats(D.T, D.d_out, (int)r);
    L.proj = take(bf16 ? (fx > fdy ? fx : fdy) * 4 : 0);
  }
  {   // partial tiles of products cut along K: at most one tile per CU
    const size_t slices = wide / 64 / 4, tiles = (T / 192 + 1) * (wide / 256 + 1) * slices;
    L.gemm_floats = bf16 && slices >= 2 ? GEMM_SCRATCH_FLOATS / 256 * (tiles < 256 ? tiles : 256) : 0;
    L.gemm_part = take(L.gemm_floats * 4);
  }
  const size_t scratch = o;
  // few rows in bf16 multiply with the codes themselves
  L.few_floats = q4 && bf16 ? q4_few_scratch_floats((int)dn, (int)di, (int)T, (int)r) : 0;
  L.mid_floats = q4 && bf16 && !L.few_floats && q4_mid_ok((int)dn, (int)di, (int)T) ? q4_mid_scratch_floats((int)dn, (int)di, (int)T) : 0;
  L.few = take((L.few_floats + L.mid_floats) * 4);
  L.W = take(q4 && !L.few_floats && !L.mid_floats ? di * dn * E : 0);
  L.fwd_end = o;
  o = scratch;
  L.W_T = take(di * dn * E);
  L.Bt = take(r * dn * E);
  L.At = take(di * r * E);
  L.V = take(T * r * 4);
  L.V_T = take(bf16 ? 3 * r * L.ldT * 2 : 0);
  L.dx32 = take(bf16 && !gemm_masked_ok(D.T, D.d_in, D.d_out, 3 * (int)r) ? T * di * 4 : 0);
  L.partial_floats = bf16 ? adapter_sums_partial_floats((int)r, (int)di, (int)T) + adapter_sums_partial_floats((int)r, (int)dn, (int)T)
                          : group_outer_partial_floats(1, (int)r, (int)di, (int)T) +
                                group_outer_partial_floats(1, (int)r, (int)dn, (int)T);
  L.partials = take(L.partial_floats * 4);
  L.padgA = take(padded ? r * di * 4 : 0);
  L.padgB = take(padded ? dn * r * 4 : 0);
  L.bwd_end = o > L.fwd_end ? o : L.fwd_end;
  return L;
}

// back: of a backward call.  A factor of 2^31 elements is not laid out anew (launch_relayout), which the backward does with
// both, and the forward where they are padded.
int check_dims(const mixlora_linear_dims *D, bool back) {
  if (!D) return MIXLORA_E_NULL;
  if (D->dtype != MIXLORA_F32 && D->dtype != MIXLORA_BF16) return MIXLORA_E_DTYPE;
  if (D->T < 1 || D->d_in < 8 || D->d_out < 8 || D->r < 1 || D->r > 64) return MIXLORA_E_SHAPE;
  if (D->d_in % 8 || D->d_out % 8 || D->d_in >= 1 << 27 || D->d_out >= 1 << 27) return MIXLORA_E_SHAPE;
  if ((int64_t)D->T >= (1 << 24)) return MIXLORA_E_SHAPE;
  const int64_t r = (D->r + 7) & ~7, wide = D->d_in > D->d_out ? D->d_in : D->d_out;
  if ((back || r != D->r) && r * wide >= (1ll << 31)) return MIXLORA_E_SHAPE;
  return MIXLORA_OK;
}

int check_q4(const mixlora_linear_dims &D, const mixlora_q4 *q4) {
  if (!q4 || !q4->codes || !q4->scales) return MIXLORA_E_NULL;
  if (!mixlora_q4_scale_bytes(D.d_out, D.d_in, q4->group)) return MIXLORA_E_SHAPE;
  return misaligned(q4->codes) || misaligned(q4->scales) ? MIXLORA_E_ALIGN : MIXLORA_OK;
}

// p in [0, 1), held in 16 bits; from 1 - 2^-17 on it would drop everything
int make_drop(const mixlora_dropout *d, DropArgs &out) {
  out = DropArgs{};
  if (!d) return MIXLORA_OK;
  if (!(d->p >= 0.f && d->p < 1.f)) return MIXLORA_E_SHAPE;
  if (d->step && (reinterpret_cast<uintptr_t>(d->step) & 7)) return MIXLORA_E_ALIGN;
  const uint32_t thr = (uint32_t)std::floor((double)d->p * 65536.0 + 0.5);
  if (thr >= 65536) return MIXLORA_E_SHAPE;
  out = DropArgs{thr, (float)(65536.0 / (65536.0 - thr)), (uint32_t)d->seed, (uint32_t)(d->seed >> 32), d->offset, d->step};
  return MIXLORA_OK;
}

#define HIP_TRY(expr)                                   \
  do {                                                  \
    hipError_t e_ = (expr);                             \
    if (e_ != hipSuccess) return MIXLORA_E_HIP;         \
  } while (0)

// fp32 storage: out = D(x), eight elements per thread.  Workgroups in rows of DROP_GRID_X: a grid dimension holds less than 2^32
// threads, 2^35 elements.
constexpr int DROP_GRID_X = 1 << 14;
__global__ __launch_bounds__(256) void dropout_f32_kernel(const float *__restrict__ x, float *__restrict__ out,
                                                          int64_t chunks, int per_row, DropArgs drop) {
  const int64_t i = ((int64_t)blockIdx.y * DROP_GRID_X + blockIdx.x) * 256 + threadIdx.x;
  if (i >= chunks) return;
  const uint32_t keep = drop_keep8(drop_key(drop), (uint32_t)(i / per_row), (uint32_t)(i % per_row));
  Vec8<float> v;
  v.load(x + i * 8);
#pragma unroll
  for (int e = 0; e < 8; e++) v.set(e, keep >> e & 1 ? drop.inv * v.get(e) : 0.f);
  v.store(out + i * 8);
}

// out[t, c] = base[t, c] + (c of row t kept ? f * sum_q V[t, q] At[c, q] : 0), rounded once (fp32 storage: base is out).
// Bound by base and out.  A workgroup owns 64 columns of 32 ROWS rows and holds both factors in LDS: its columns' part of At is one
// run of memory.  Eight columns of ROWS rows per thread, one call of the generator each.  A step of 600 tokens 1024 -> 1024 at
// rank 16 took 95.7 us with At read by every thread in its rows' order, 83.5 so; 3000 2048 -> 2048 at rank 64 909, 764.
// Of V's entries those from `rank` on count as zeros (they fill up a multiple of eight, and are NaN beside an infinite row).
// offs: all tokens are one group of the gradient sums.
constexpr int MLA_COLS = 64, MLA_PITCH = 64 + 4;
template <typename E, int ROWS>
__global__ __launch_bounds__(256) void masked_lowrank_add_kernel(const float *base, const float *__restrict__ V,
                                                                 const E *__restrict__ At, E *out, int T, int C, int r,
                                                                 int rank, float f, DropArgs drop, int32_t *offs) {
  __shared__ __align__(16) float sa[64][MLA_PITCH], sv[32 * ROWS][MLA_PITCH];   // [q][column], [row][q]
  const int tid = threadIdx.x, col_blocks = (C + MLA_COLS - 1) / MLA_COLS;
  if (offs && blockIdx.x == 0 && tid == 0) offs[0] = 0, offs[1] = T;
  const int first_col = blockIdx.x % col_blocks * MLA_COLS, first_row = blockIdx.x / col_blocks * (32 * ROWS);
  const int c0 = first_col + (tid & 7) * 8, t0 = first_row + (tid >> 3), pieces = r >> 3;
  Vec8<float> b[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; i++)
    b[i].load(base + (int64_t)(t0 + 32 * i < T ? t0 + 32 * i : T - 1) * C + (c0 < C ? c0 : 0));
  for (int i = tid; i < MLA_COLS * pieces; i += 256) {
    const int c = i / pieces, q0 = i % pieces * 8;
    Vec8<E> v;
    v.load(At + (int64_t)(first_col + c < C ? first_col + c : C - 1) * r + q0);
#pragma unroll
    for (int e = 0; e < 8; e++) sa[q0 + e][c] = v.get(e);
  }
  for (int i = tid; i < 32 * ROWS * pieces; i += 256) {
    const int t = i / pieces, q0 = i % pieces * 8;
    Vec8<float> v;
    v.load(V + (int64_t)(first_row + t < T ? first_row + t : T - 1) * r + q0);
    if (q0 + 8 > rank) {
#pragma unroll
      for (int e = 0; e < 8; e++) v.set(e, q0 + e < rank ? v.get(e) : 0.f);
    }
    v.store(&sv[t][q0]);
  }
  __syncthreads();
  float acc[ROWS][8];
#pragma unroll
  for (int i = 0; i < ROWS; i++)
#pragma unroll
    for (int j = 0; j < 8; j++) acc[i][j] = 0.f;
  for (int q0 = 0; q0 < r; q0 += 4) {
    f32x4_t p[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; i++) p[i] = *reinterpret_cast<const f32x4_t *>(&sv[(tid >> 3) + 32 * i][q0]);
#pragma unroll
    for (int q = 0; q < 4; q++) {
      Vec8<float> w;
      w.load(&sa[q0 + q][(tid & 7) * 8]);
#pragma unroll
      for (int i = 0; i < ROWS; i++)
#pragma unroll
        for (int j = 0; j < 8; j++) acc[i][j] = fmaf(p[i][q], w.get(j), acc[i][j]);
    }
  }
  if (c0 >= C) return;
  const DropKey key = drop_key(drop);
#pragma unroll
  for (int i = 0; i < ROWS; i++) {
    const int t = t0 + 32 * i;
    if (t >= T) break;
    const uint32_t keep = drop.thr ? drop_keep8(key, (uint32_t)t, (uint32_t)c0 >> 3) : 0xffu;
    Vec8<E> o;
#pragma unroll
    for (int j = 0; j < 8; j++) o.set(j, b[i].get(j) + (keep >> j & 1 ? f * acc[i][j] : 0.f));
    o.store(out + (int64_t)t * C + c0);
  }
}
template <typename E>
hipError_t launch_masked_add(const float *base, const float *V, const void *At, void *out, int T, int C, int r, int rank, float f,
                             const DropArgs &drop, int32_t *offs, hipStream_t st) {
  // four rows per thread read the factors less often; one where that leaves most of the chip without a workgroup
  const int64_t col_blocks = (C + MLA_COLS - 1) / MLA_COLS;
  const bool four = (T + 127) / 128 * col_blocks >= 256;
  const dim3 grid((unsigned)((four ? (T + 127) / 128 : (T + 31) / 32) * col_blocks)), block(256);
  const int slot = prof_on() ? prof_mark_begin(PROF_OTHER, st) : -1;
  if (four)
    hipLaunchKernelGGL((masked_lowrank_add_kernel<E, 4>), grid, block, 0, st, base, V, (const E *)At, (E *)out, T, C, r, rank, f, drop, offs);
  else
    hipLaunchKernelGGL((masked_lowrank_add_kernel<E, 1>), grid, block, 0, st, base, V, (const E *)At, (E *)out, T, C, r, rank, f, drop, offs);
  if (slot >= 0) prof_mark_end(slot, st, (double)T * C * (4 + sizeof(E)));
  return hipGetLastError();
}

GemmProblem problem(int M, int N, void *C, int c_f32, const void *A, const void *B, int K) {
  GemmProblem p{};
  p.M = M; p.N = N; p.C = C; p.ldc = N; p.c_f32 = c_f32; p.nseg = 1;
  p.seg[0].A = A; p.seg[0].lda = K; p.seg[0].B = B; p.seg[0].ldb = K; p.seg[0].K = K;
  return p;
}

// ---- bf16: the projection P = D(X) Wq^T [T, r] in all its forms ------------------------------------------------
// P in fp32; PT, the row factor of the gradient sums, in three bf16 pieces [hi(r) | mid(r) | lo(r)][ldT]; and m P
// (s = m 2^e, 1/2 <= |m| < 1) in three pieces, ext[t] = [hi(r) | mid(r) | lo(r)], whose sum is m P to its last bit.
// The other factor of the rank-r term, from Wr [cols, r], is ext_B[c] = [B | B' | B'] 2^e with B' = B but zeros for
// infinities: hi alone meets those, or two pieces of opposite signs would make NaN of them.
struct Project {
  const bf16_t *X, *Wq, *Wr;
  int T, K, r, cols, ldT, S;   // S slices of the contraction, of `per` tiles
  int per, rank;               // entries from rank on fill up a multiple of eight
  float m, b_scale, *P, *part; // part [S][T][r], S > 1
  bf16_t *PT, *ext, *ext_B;
  int32_t *offs;
  DropArgs drop;
};

__device__ __forceinline__ void store_projection(const Project &a, int t, int q, float v) {
  if (a.drop.thr) v *= a.drop.inv;
  if (q >= a.rank) v = 0.f;   // a zero row of Wq has made NaN beside an infinite row of X
  a.P[(int64_t)t * a.r + q] = v;
  float pc[3];
  three_pieces(v, pc);
#pragma unroll
  for (int i = 0; i < 3; i++) a.PT[((int64_t)i * a.r + q) * a.ldT + t] = (bf16_t)pc[i];
  three_pieces(a.m * v, pc);
  bf16_t *o = a.ext + (int64_t)t * 3 * a.r + q;
#pragma unroll
  for (int i = 0; i < 3; i++) o[i * a.r] = (bf16_t)pc[i];
}

// Bound by reading X once.  A workgroup owns 16 rows and a slice of the contraction, its wavefronts 128-column tiles
// of that in turn; both operands change lanes in LDS (rows_stage.h).  Few rows are cut into slices that fill the chip, which
// project_finish_kernel adds in order; trailing workgroups lay out the other factor.
template <int NQ, bool DROP, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void project_kernel(Project a) {
  __shared__ __align__(16) unsigned char smem[WAVES * STAGE_BYTES];   // then sums [WAVES][NQ][64][4]
  static_assert(NQ * 1024 <= STAGE_BYTES, "the sums fit");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = a.T, K = a.K, r = a.r, row_blocks = (T + 15) >> 4;
  if ((int)blockIdx.x >= row_blocks * a.S) {   // workgroup-uniform; eight entries of a row of Wr per thread
    const int per = r >> 3;
    const int64_t i = (int64_t)(blockIdx.x - row_blocks * a.S) * (WAVES * 64) + tid;
    if (i >= (int64_t)a.cols * per) return;
    const int c = (int)(i / per), q0 = (int)(i % per) * 8;
    bf16x8_t v = *reinterpret_cast<const bf16x8_t *>(a.Wr + (int64_t)c * r + q0), fin;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      v[e] = (bf16_t)((float)v[e] * a.b_scale);
      fin[e] = __builtin_isinf((float)v[e]) ? (bf16_t)0.f : v[e];
    }
    bf16_t *o = a.ext_B + (int64_t)c * 3 * r + q0;
    *reinterpret_cast<bf16x8_t *>(o) = v;
    *reinterpret_cast<bf16x8_t *>(o + r) = fin;
    *reinterpret_cast<bf16x8_t *>(o + 2 * r) = fin;
    return;
  }
  if (blockIdx.x == 0 && tid == 0) {   // all tokens are one group of the gradient sums
    a.offs[0] = 0;
    a.offs[1] = T;
  }
  const int t0 = blockIdx.x % row_blocks * 16, sl = blockIdx.x / row_blocks;
  const int kbs = (K + STAGE_COLS - 1) / STAGE_COLS, lo = sl * a.per, end = lo + a.per < kbs ? lo + a.per : kbs;
  unsigned char *stage = smem + wave * STAGE_BYTES;
  DropKey key;
  if constexpr (DROP) key = drop_key(a.drop);
  f32x4_t acc[NQ];
#pragma unroll
  for (int j = 0; j < NQ; j++) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int kb = lo + wave; kb < end; kb += WAVES) {
    bf16x8_t vx[4], vw[NQ][4], fx[4];
    rows_load(a.X + (int64_t)t0 * K, T - t0, kb, K, lane, vx);
#pragma unroll
    for (int j = 0; j < NQ; j++) rows_load(a.Wq + (int64_t)(j * 16 < r ? j * 16 : 0) * K, j * 16 < r ? r - j * 16 : r, kb, K, lane, vw[j]);
    if constexpr (DROP) {   // a load is eight columns of a row: one call of the generator
#pragma unroll
      for (int p = 0; p < 4; p++)
        vx[p] = drop_mask8(key, (uint32_t)(t0 + p * 4 + (lane >> 4)), (uint32_t)(kb * (STAGE_COLS / 8) + (lane & 15)), vx[p]);
    }
    wave_order();
    rows_to_lds(stage, vx, kb, K, lane);
    wave_order();
    rows_from_lds(stage, lane, fx);
#pragma unroll
    for (int j = 0; j < NQ; j++) {
      bf16x8_t fw[4];
      wave_order();
      rows_to_lds(stage, vw[j], kb, K, lane);
      wave_order();
      rows_from_lds(stage, lane, fw);
#pragma unroll
      for (int st = 0; st < 4; st++) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[st], fx[st], acc[j], 0, 0, 0);
    }
  }
  __syncthreads();   // the staging is behind everybody
  float *red = reinterpret_cast<float *>(smem);
#pragma unroll
  for (int j = 0; j < NQ; j++) *reinterpret_cast<f32x4_t *>(red + ((wave * NQ + j) * 64 + lane) * 4) = acc[j];
  __syncthreads();
  // acc[j][u] of lane (l15, hi): row l15, q = 16 j + 4 hi + u
  for (int i = tid; i < NQ * 256; i += WAVES * 64) {
    const int j = i >> 8, q = j * 16 + (i & 15), t = t0 + ((i >> 4) & 15);
    if (q >= r || t >= T) continue;
    const int e = (((i >> 2) & 3) * 16 + ((i >> 4) & 15)) * 4 + (i & 3);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; w++) v += red[(w * NQ + j) * 256 + e];
    if (a.S == 1) store_projection(a, t, q, v);
    else a.part[((int64_t)sl * T + t) * r + q] = v;
  }
}
__global__ __launch_bounds__(256) void project_finish_kernel(Project a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)a.T * a.r;
  if (i >= n) return;
  float v = 0.f;
  for (int s0 = 0; s0 < a.S; s0 += 8) {
    float u[8];
#pragma unroll
    for (int s = 0; s < 8; s++) u[s] = a.part[(int64_t)(s0 + s < a.S ? s0 + s : s0) * n + i];
#pragma unroll
    for (int s = 0; s < 8; s++)
      if (s0 + s < a.S) v += u[s];
  }
  store_projection(a, (int)(i / a.r), (int)(i % a.r), v);
}

// Slices of the projection: none where the row blocks alone nearly fill the chip, else as many as fill it with eight
// tiles or fewer left to each.
int project_slices(int T, int K) {
  const int rb = (T + 15) / 16, kbs = (K + STAGE_COLS - 1) / STAGE_COLS;
  if (rb >= 160) return 1;
  const int want = 256 / rb, most = (kbs + 7) / 8;
  return want < most ? want : most;
}
size_t project_floats(int T, int K, int r) {
  const int S = project_slices(T, K);
  return S > 1 ? (size_t)S * T * r : 0;
}
// sliced: the slices, where there are several, are left in a.part for another kernel to add, and their number goes there
hipError_t launch_project(Project a, float s, const DropArgs &drop, hipStream_t st, int *sliced = nullptr) {
  int e = 0;   // s = m 2^e
  if (std::isfinite(s)) std::frexp(s, &e);
  e = e < -100 ? -100 : e > 100 ? 100 : e;
  a.m = std::ldexp(s, -e);
  a.b_scale = std::ldexp(1.f, e);
  a.drop = drop;
  const int kbs = (a.K + STAGE_COLS - 1) / STAGE_COLS;
  a.S = project_slices(a.T, a.K);
  a.per = (kbs + a.S - 1) / a.S;
  a.S = (kbs + a.per - 1) / a.per;
  const int slot = prof_on() ? prof_mark_begin(PROF_OTHER, st) : -1;
#define MIXLORA_PROJECT(NQ_, DROP_, WAVES_)                                                                            \
  hipLaunchKernelGGL((project_kernel<NQ_, DROP_, WAVES_>),                                                             \
                     dim3((a.T + 15) / 16 * a.S + ((int64_t)a.cols * (a.r / 8) + WAVES_ * 64 - 1) / (WAVES_ * 64)),    \
                     dim3(WAVES_ * 64), 0, st, a)
#define MIXLORA_PROJECT_W(NQ_, DROP_)                   \
  do {                                                  \
    if (a.S > 1 || NQ_ > 2) MIXLORA_PROJECT(NQ_, DROP_, 8); \
    else MIXLORA_PROJECT(NQ_, DROP_, (NQ_ > 2 ? 8 : 16));  \
  } while (0)
  if (drop.thr) {
    if (a.r <= 16) MIXLORA_PROJECT_W(1, true);
    else if (a.r <= 32) MIXLORA_PROJECT_W(2, true);
    else MIXLORA_PROJECT_W(4, true);
  } else {
    if (a.r <= 16) MIXLORA_PROJECT_W(1, false);
    else if (a.r <= 32) MIXLORA_PROJECT_W(2, false);
    else MIXLORA_PROJECT_W(4, false);
  }
#undef MIXLORA_PROJECT
#undef MIXLORA_PROJECT_W
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  if (sliced) *sliced = a.S;
  else if (a.S > 1)
    hipLaunchKernelGGL(project_finish_kernel, dim3((unsigned)(((int64_t)a.T * a.r + 255) / 256)), dim3(256), 0, st, a);
  if (slot >= 0) prof_mark_end(slot, st, 0.0);
  return hipGetLastError();
}

// the frozen matrix of a call: one of the two
struct Frozen {
  const void *W, *W_T;       // ordinary; W_T may be NULL
  const mixlora_q4 *q4;
  Q4Matrix q4_matrix(const mixlora_linear_dims &D) const {
    return Q4Matrix{(const unsigned char *)q4->codes, (const bf16_t *)q4->scales, D.d_out, D.d_in, q4->group};
  }
};

Project project(const Layout &L, char *ws, const void *X, const void *Wq, const void *Wr, int T,
                int K, int rank, int cols, size_t P, size_t PT) {
  Project a{};
  a.X = (const bf16_t *)X, a.Wq = (const bf16_t *)Wq, a.Wr = (const bf16_t *)Wr;
  a.T = T, a.K = K, a.r = L.rp, a.rank = rank, a.cols = cols, a.ldT = L.ldT;
  a.P = (float *)(ws + P), a.part = (float *)(ws + L.proj);
  a.PT = (bf16_t *)(ws + PT), a.ext = (bf16_t *)(ws + L.ext), a.ext_B = (bf16_t *)(ws + L.ext_B);
  a.offs = (int32_t *)(ws + L.offs);
  return a;
}

int forward(mixlora_linear_dims D, const Frozen &F, const void *A, const void *B, const DropArgs &drop, const void *x,
            void *y, char *ws, size_t ws_bytes, hipStream_t st) {
  const Layout L = make_layout(D, F.q4 != nullptr);
  if (ws_bytes < L.fwd_end) return MIXLORA_E_WORKSPACE;
  const int T = D.T, di = D.d_in, dn = D.d_out, dt = D.dtype;
  if (L.rp != D.r) {   // run on zero-padded banks (they stay in the workspace for the backward)
    const RelayoutJob jobs[2] = {job_rank_resize(A, ws + L.padA, 1, D.r, L.rp, di, true),
                                 job_rank_resize(B, ws + L.padB, 1, D.r, L.rp, dn, false)};
    HIP_TRY(launch_relayout(dt, jobs, 2, st));
    A = ws + L.padA;
    B = ws + L.padB;
  }
  const int r = L.rp;
  float *P = (float *)(ws + L.P);
  const void *W = F.W;
  if (L.few_floats) {   // (the backward makes the projection itself)
    const Q4Few a{(const bf16_t *)x, (const bf16_t *)A, (const bf16_t *)B, T, r, D.r, D.lora_scale, (bf16_t *)y};
    HIP_TRY(launch_q4_few(F.q4_matrix(D), a, drop, (float *)(ws + L.few), L.few_floats, st));
    return MIXLORA_OK;
  }
  if (L.mid_floats) {
    Q4Projection proj{P, 1, 1.f, nullptr, 0};
    HIP_TRY(launch_project(project(L, ws, x, A, B, T, di, D.r, 0, L.P, L.P_T), D.lora_scale, drop, st, &proj.S));
    if (proj.S > 1) proj = Q4Projection{(const float *)(ws + L.proj), proj.S, drop.thr ? drop.inv : 1.f, (bf16_t *)(ws + L.P_T), L.ldT};
    const Q4Few a{(const bf16_t *)x, (const bf16_t *)A, (const bf16_t *)B, T, r, D.r, D.lora_scale, (bf16_t *)y};
    HIP_TRY(launch_q4_mid(F.q4_matrix(D), a, proj, (float *)(ws + L.few), L.mid_floats, st));
    return MIXLORA_OK;
  }
  if (F.q4) {
    HIP_TRY(launch_q4_dequantize(F.q4_matrix(D), false, dt, ws + L.W, st));
    W = ws + L.W;
  }
  if (dt == MIXLORA_F32) {
    const void *xd = x;
    if (drop.thr) {
      const int64_t chunks = (int64_t)T * (di / 8), blocks = (chunks + 255) / 256;
      const dim3 grid(blocks < DROP_GRID_X ? (unsigned)blocks : DROP_GRID_X, (unsigned)((blocks + DROP_GRID_X - 1) / DROP_GRID_X));
      hipLaunchKernelGGL(dropout_f32_kernel, grid, dim3(256), 0, st, (const float *)x, (float *)(ws + L.xd), chunks, di / 8, drop);
      HIP_TRY(hipGetLastError());
      xd = ws + L.xd;
    }
    const GemmProblem p[2] = {problem(T, dn, y, 0, x, W, di), problem(T, r, P, 1, xd, A, di)};
    HIP_TRY(launch_gemm(dt, p, 2, st));
    HIP_TRY(launch_masked_add<float>((const float *)y, P, B, y, T, dn, r, D.r, D.lora_scale, DropArgs{}, nullptr, st));
    return MIXLORA_OK;
  }
  HIP_TRY(launch_project(project(L, ws, x, A, B, T, di, D.r, dn, L.P, L.P_T), D.lora_scale, drop, st));
  GemmProblem p = problem(T, dn, y, 0, x, W, di);
  p.seg[1] = GemmSeg{ws + L.ext, ws + L.ext_B, 3 * r, 3 * r, 3 * r};
  p.nseg = 2;
  HIP_TRY(launch_gemm(dt, &p, 1, st, GemmScratch{L.gemm_floats ? (float *)(ws + L.gemm_part) : nullptr, L.gemm_floats}));
  return MIXLORA_OK;
}

int backward(const mixlora_linear_dims &D, const Frozen &F, const void *A, const void *B, const DropArgs &drop, const void *x,
             const void *dy, char *ws, size_t ws_bytes, void *dx, float *dA, float *dB, hipStream_t st) {
  const Layout L = make_layout(D, F.q4 != nullptr);
  if (ws_bytes < L.bwd_end) return MIXLORA_E_WORKSPACE;
  const int T = D.T, di = D.d_in, dn = D.d_out, dt = D.dtype, r = L.rp;
  const float s = D.lora_scale;
  float *dA_user = dA, *dB_user = dB;
  if (L.rp != D.r) {   // padded banks from the forward pass; padded gradients, cut back at the end
    A = ws + L.padA;
    B = ws + L.padB;
    dA = (float *)(ws + L.padgA);
    dB = (float *)(ws + L.padgB);
  }
  const void *W_T = F.W_T;
  if (F.q4) {
    HIP_TRY(launch_q4_dequantize(F.q4_matrix(D), true, dt, ws + L.W_T, st));
    W_T = ws + L.W_T;
  } else if (!W_T) {
    HIP_TRY(launch_transpose(dt, F.W, ws + L.W_T, dn, di, st));
    W_T = ws + L.W_T;
  }
  {
    const RelayoutJob jobs[2] = {job_bank_T(B, 1, dn, r, ws + L.Bt),     // [d_out, r] -> [r, d_out]
                                 job_bank_T(A, 1, r, di, ws + L.At)};    // [r, d_in]  -> [d_in, r]
    HIP_TRY(launch_relayout(dt, jobs, 2, st));
  }
  float *V = (float *)(ws + L.V), *P = (float *)(ws + L.P), *part = (float *)(ws + L.partials);
  const int32_t *offs = (const int32_t *)(ws + L.offs);
  if (dt == MIXLORA_F32) {
    const void *xd = drop.thr ? ws + L.xd : x;
    const GemmProblem p[2] = {problem(T, di, dx, 0, dy, W_T, dn), problem(T, r, V, 1, dy, ws + L.Bt, dn)};
    HIP_TRY(launch_gemm(dt, p, 2, st));
    HIP_TRY(launch_masked_add<float>((const float *)dx, V, ws + L.At, dx, T, di, r, D.r, drop.thr ? s * drop.inv : s, drop,
                                     (int32_t *)(ws + L.offs), st));
    const GoJob go[2] = {GoJob{offs, nullptr, V, (const float *)xd, dA, 1, r, di, 1, T, 1, s},
                         GoJob{offs, nullptr, P, (const float *)dy, dB, 1, r, dn, 1, T, 0, s}};
    HIP_TRY(launch_group_outer(go, 2, part, L.partial_floats, st));
  } else {
    if (L.few_floats) {   // the forward has not kept the projection
      HIP_TRY(launch_project(project(L, ws, x, A, B, T, di, D.r, 0, L.P, L.P_T), s, drop, st));
    }
    // (the term of dx is masked and scaled, the factor V of dA is not)
    HIP_TRY(launch_project(project(L, ws, dy, ws + L.Bt, ws + L.At, T, dn, D.r, di, L.V, L.V_T),
                           drop.thr ? s * drop.inv : s, DropArgs{}, st));
    const GemmScratch gs{L.gemm_floats ? (float *)(ws + L.gemm_part) : nullptr, L.gemm_floats};
    const GemmSeg frozen{dy, W_T, dn, dn, dn}, term{ws + L.ext, ws + L.ext_B, 3 * r, 3 * r, 3 * r};
    GemmProblem p = problem(T, di, dx, 0, dy, W_T, dn);
    if (!drop.thr) {
      p.seg[1] = term;
      p.nseg = 2;
      HIP_TRY(launch_gemm(dt, &p, 1, st, gs));
    } else if (gemm_masked_ok(T, di, dn, 3 * r)) {
      p.seg[0] = term;
      p.seg[1] = frozen;
      p.nseg = 2;
      HIP_TRY(launch_gemm_masked(p, drop, st, gs));
    } else {   // operands of 4 GiB or more, the term's included
      p.C = ws + L.dx32;
      p.c_f32 = 1;
      HIP_TRY(launch_gemm(dt, &p, 1, st, gs));
      HIP_TRY(launch_masked_add<bf16_t>((const float *)(ws + L.dx32), V, ws + L.At, dx, T, di, r, D.r, s * drop.inv, drop, nullptr, st));
    }
    const GomJob go[2] = {
        GomJob{ws + L.V_T, x, dA, offs, nullptr, 1, r, di, 1, T, L.ldT, 2, 1, drop.thr ? s * drop.inv : s, 0, drop},
        GomJob{ws + L.P_T, dy, dB, offs, nullptr, 1, r, dn, 1, T, L.ldT, 2, 0, s, 0, DropArgs{}}};
    HIP_TRY(launch_adapter_sums(go, 2, part, L.partial_floats, st));
  }
  if (L.rp != D.r) {
    const RelayoutJob jobs[2] = {job_rank_resize(dA, dA_user, 1, L.rp, D.r, di, true),
                                 job_rank_resize(dB, dB_user, 1, L.rp, D.r, dn, false)};
    HIP_TRY(launch_relayout(MIXLORA_F32, jobs, 2, st));
  }
  return MIXLORA_OK;
}

// arguments common to both kinds of matrix; pointers in order of the call
int check_pointers(std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if (!p) return MIXLORA_E_NULL;
  for (const void *p : ps)
    if (misaligned(p)) return MIXLORA_E_ALIGN;
  return MIXLORA_OK;
}

}  // namespace

extern "C" {

size_t mixlora_q4_linear_workspace_bytes(const mixlora_linear_dims *dims, int32_t group, int for_backward) {
  if (check_dims(dims, for_backward != 0) != MIXLORA_OK || !mixlora_q4_scale_bytes(dims->d_out, dims->d_in, group)) return 0;
  const Layout L = make_layout(*dims, true);
  return for_backward ? L.bwd_end : L.fwd_end;
}

int mixlora_q4_linear_forward(const mixlora_linear_dims *dims, const mixlora_q4 *q4, const void *A, const void *B,
                              const mixlora_dropout *dropout, const void *x, void *y, void *workspace,
                              size_t workspace_bytes, void *stream) {
  int rc = check_dims(dims, false);
  if (rc) return rc;
  DropArgs drop;
  if ((rc = check_q4(*dims, q4)) || (rc = make_drop(dropout, drop)) || (rc = check_pointers({A, B, x, y, workspace})))
    return rc;
  return forward(*dims, Frozen{nullptr, nullptr, q4}, A, B, drop, x, y, (char *)workspace, workspace_bytes, (hipStream_t)stream);
}

int mixlora_q4_linear_backward(const mixlora_linear_dims *dims, const mixlora_q4 *q4, const void *A, const void *B,
                               const mixlora_dropout *dropout, const void *x, const void *dy, void *workspace,
                               size_t workspace_bytes, void *dx, float *dA, float *dB, void *stream) {
  int rc = check_dims(dims, true);
  if (rc) return rc;
  DropArgs drop;
  if ((rc = check_q4(*dims, q4)) || (rc = make_drop(dropout, drop)) ||
      (rc = check_pointers({A, B, x, dy, workspace, dx, dA, dB})))
    return rc;
  return backward(*dims, Frozen{nullptr, nullptr, q4}, A, B, drop, x, dy, (char *)workspace, workspace_bytes, dx, dA, dB,
                  (hipStream_t)stream);
}

size_t mixlora_lora_dropout_workspace_bytes(const mixlora_linear_dims *dims, int for_backward) {
  if (check_dims(dims, for_backward != 0) != MIXLORA_OK) return 0;
  const Layout L = make_layout(*dims, false);
  return for_backward ? L.bwd_end : L.fwd_end;
}

int mixlora_lora_dropout_forward(const mixlora_linear_dims *dims, const void *W, const void *A, const void *B,
                                 const mixlora_dropout *dropout, const void *x, void *y, void *workspace,
                                 size_t workspace_bytes, void *stream) {
  int rc = check_dims(dims, false);
  if (rc) return rc;
  DropArgs drop;
  if ((rc = make_drop(dropout, drop)) || (rc = check_pointers({W, A, B, x, y, workspace}))) return rc;
  return forward(*dims, Frozen{W, nullptr, nullptr}, A, B, drop, x, y, (char *)workspace, workspace_bytes, (hipStream_t)stream);
}

int mixlora_lora_dropout_backward(const mixlora_linear_dims *dims, const void *W, const void *W_T, const void *A,
                                  const void *B, const mixlora_dropout *dropout, const void *x, const void *dy,
                                  void *workspace, size_t workspace_bytes, void *dx, float *dA, float *dB, void *stream) {
  int rc = check_dims(dims, true);
  if (rc) return rc;
  DropArgs drop;
  if ((rc = make_drop(dropout, drop)) || (rc = check_pointers({W, A, B, x, dy, workspace, dx, dA, dB}))) return rc;
  if (W_T && misaligned(W_T)) return MIXLORA_E_ALIGN;
  return backward(*dims, Frozen{W, W_T, nullptr}, A, B, drop, x, dy, (char *)workspace, workspace_bytes, dx, dA, dB,
                  (hipStream_t)stream);
}

}  // extern "C"
