// Softmax routing of given logits with Eq. 8-9 and a z-loss over the tokens that a mask keeps:
//   p = softmax(z), the k largest kept (ties to the lower index), w = their p over its sum;
//   n = tokens kept by the mask, F and P of Eq. 9 over them, balance = a N sum_i F_i P_i,
//   z_loss = b / n sum_t lse_t^2 with lse_t = log sum_i exp z_ti;
//   dz_ti = g_b a N / n p_ti (F_i - sum_j F_j p_tj) + g_z b 2 / n lse_t p_ti + [i kept] w_ti (dw_ti - sum_j w_tj dw_tj).
// A token that the mask drops is left out of every sum, whatever its logits are, and gets index -1, weight 0
// and a zero gradient.  Both directions read the logits once and are bound by a launch's latency (1 MB of
// logits at 16384 x 16), so a thread takes a token and keeps its row in registers.  No sum depends on the
// order in which workgroups end: their partial sums are added in a fixed order.
#include "common.h"

#include <cmath>

using namespace mixlora;

namespace {

constexpr int RL_THREADS = 256;
struct RouterArgs {
  const void *logits;
  const unsigned char *mask;
  int T, N, k, top1;
  float balance, zc;
  int32_t *idx;
  float *w;
  float *part;          // [workgroup][2 N + 2]: P sums, counts (all k, as whole numbers), z sum, tokens; counts of slot 0 behind
  float *stats;         // [N + 1]: F, then 1 / n (0 where no token is kept)
  float *loss;
  int32_t *counts;
};

template <typename E, int NR>
__device__ __forceinline__ void load_row(const E *row, int N, float (&z)[NR]) {
#pragma unroll
  for (int i = 0; i < NR; i++) z[i] = i < N ? to_f32(row[i]) : -INFINITY;
}

// softmax of a row in registers: z becomes p; returns lse.  A row of -inf alone gives NaN, as its definition does.
template <int NR>
__device__ __forceinline__ float softmax_row(float (&z)[NR], int N) {
  float top = z[0];
#pragma unroll
  for (int i = 1; i < NR; i++) top = fmaxf(top, z[i]);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NR; i++) {
    z[i] = i < N ? expf(z[i] - top) : 0.f;
    sum += z[i];
  }
  const float inv = 1.f / sum;
#pragma unroll
  for (int i = 0; i < NR; i++) z[i] *= inv;
  return top + logf(sum);
}

template <typename E, int NR>
__global__ __launch_bounds__(RL_THREADS) void router_loss_forward_kernel(RouterArgs a) {
  __shared__ float col[RL_THREADS / 64][NR];
  __shared__ int cnt[NR], first[NR];
  __shared__ float zs[RL_THREADS / 64];
  __shared__ int toks;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, N = a.N, k = a.k;
  for (int i = tid; i < NR; i += RL_THREADS) cnt[i] = first[i] = 0;
  if (tid == 0) toks = 0;
  __syncthreads();
  const int64_t t = (int64_t)blockIdx.x * RL_THREADS + tid;
  const bool on = t < a.T && (!a.mask || a.mask[t]);
  float z[NR], lse = 0.f;
  if (on) {
    load_row<E, NR>((const E *)a.logits + t * N, N, z);
    // the k largest; NaN ranks with -inf
    uint64_t taken = 0;
    float raw[NR];
#pragma unroll
    for (int i = 0; i < NR; i++) raw[i] = isnan(z[i]) ? -INFINITY : z[i];
    lse = softmax_row<NR>(z, N);
    float sum = 0.f;
    int32_t *idx = a.idx + t * k;
    float *w = a.w + t * k;
    for (int j = 0; j < k; j++) {
      int best = -1;
      float bz = 0.f, bp = 0.f;
#pragma unroll
      for (int i = 0; i < NR; i++) {
        if (i < N && !(taken >> i & 1)) {
          if (best < 0 || raw[i] > bz) best = i, bz = raw[i], bp = z[i];
        }
      }
      taken |= 1ull << best;
      idx[j] = best;
      w[j] = bp;
      sum += bp;
      atomicAdd(&cnt[best], 1);          // whole numbers: any order gives the same
      if (j == 0) atomicAdd(&first[best], 1);
    }
    for (int j = 0; j < k; j++) w[j] /= sum;
    atomicAdd(&toks, 1);
  } else {
#pragma unroll
    for (int i = 0; i < NR; i++) z[i] = 0.f;
    if (t < a.T)
      for (int j = 0; j < k; j++) a.idx[t * k + j] = -1, a.w[t * k + j] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < NR; i++) {
    float v = z[i];
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if (lane == 0) col[wave][i] = v;
  }
  float v = lse * lse;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  if (lane == 0) zs[wave] = v;
  __syncthreads();
  float *p = a.part + (int64_t)blockIdx.x * (3 * N + 2);
  for (int i = tid; i < N; i += RL_THREADS) {
    float s = 0.f;
    for (int u = 0; u < RL_THREADS / 64; u++) s += col[u][i];
    p[i] = s;
    p[N + i] = (float)cnt[i];            // at most 256 k: exact
    p[2 * N + i] = (float)first[i];
  }
  if (tid == 0) {
    float s = 0.f;
    for (int u = 0; u < RL_THREADS / 64; u++) s += zs[u];
    p[3 * N] = s;
    p[3 * N + 1] = (float)toks;
  }
}

// Adds the workgroups' sums, in double and in their order.
__global__ __launch_bounds__(256) void router_loss_finish_kernel(RouterArgs a, int blocks) {
  __shared__ double sums[3 * 64 + 2];
  __shared__ double fp[64];
  const int W = 3 * a.N + 2, tid = threadIdx.x;
  for (int i = tid; i < W; i += 256) {
    double s = 0.0;
    for (int b = 0; b < blocks; b++) s += a.part[(int64_t)b * W + i];
    sums[i] = s;
  }
  __syncthreads();
  const double n = sums[3 * a.N + 1], inv = n > 0 ? 1.0 / n : 0.0;
  if (tid < a.N) {
    const double F = (a.top1 ? sums[2 * a.N + tid] : sums[a.N + tid] / a.k) * inv;
    fp[tid] = F * (sums[tid] * inv);
    a.stats[tid] = (float)F;
    a.counts[tid] = (int32_t)sums[a.N + tid];
  }
  __syncthreads();
  if (tid == 0) {
    double s = 0.0;
    for (int i = 0; i < a.N; i++) s += fp[i];
    const double balance = (double)a.balance * a.N * s, z = (double)a.zc * sums[3 * a.N] * inv;
    a.loss[0] = (float)(balance + z);
    a.loss[1] = (float)balance;
    a.loss[2] = (float)z;
    a.stats[a.N] = (float)inv;
  }
}

template <typename E, int NR>
__global__ __launch_bounds__(RL_THREADS) void router_loss_backward_kernel(RouterArgs a, const int32_t *__restrict__ idx,
                                                                          const float *__restrict__ dw, float gb, float gz,
                                                                          void *__restrict__ dz) {
  const int64_t t = (int64_t)blockIdx.x * RL_THREADS + threadIdx.x;
  if (t >= a.T) return;
  const int N = a.N, k = a.k;
  E *out = (E *)dz + t * N;
  if (a.mask && !a.mask[t]) {
    for (int i = 0; i < N; i++) out[i] = from_f32<E>(0.f);
    return;
  }
  float z[NR];
  load_row<E, NR>((const E *)a.logits + t * N, N, z);
  const float lse = softmax_row<NR>(z, N);
  const float inv = a.stats[N];
  float fp = 0.f;
#pragma unroll
  for (int i = 0; i < NR; i++)
    if (i < N) fp = fmaf(a.stats[i], z[i], fp);
  const float cb = gb * a.balance * (float)N * inv, cz = gz * a.zc * 2.f * inv * lse;
  // the kept experts' share: w = p / sum of the kept p
  uint64_t kept = 0;
  float sum = 0.f, dot = 0.f;
  if (dw) {
    for (int j = 0; j < k; j++) {
      const int e = idx[t * k + j];
      if (e >= 0 && e < N) kept |= 1ull << e;
    }
#pragma unroll
    for (int i = 0; i < NR; i++)
      if (i < N && (kept >> i & 1)) sum += z[i];
    for (int j = 0; j < k; j++) {
      const int e = idx[t * k + j];
      float pe = 0.f;
#pragma unroll
      for (int i = 0; i < NR; i++)
        if (i == e) pe = z[i];
      dot = fmaf(pe / sum, dw[t * k + j], dot);
    }
  }
#pragma unroll
  for (int i = 0; i < NR; i++) {
    if (i >= N) continue;
    float g = z[i] * (cb * (a.stats[i] - fp) + cz);
    if (kept >> i & 1) {
      float d = 0.f;
      for (int j = 0; j < k; j++)
        if (idx[t * k + j] == i) d = dw[t * k + j];
      g = fmaf(z[i] / sum, d - dot, g);
    }
    out[i] = from_f32<E>(g);
  }
}

int check(const mixlora_router_dims *D) {
  if (!D) return MIXLORA_E_NULL;
  if (D->dtype != MIXLORA_F32 && D->dtype != MIXLORA_BF16) return MIXLORA_E_DTYPE;
  if (D->aux_mode != MIXLORA_AUX_TOP1 && D->aux_mode != MIXLORA_AUX_TOPK) return MIXLORA_E_DTYPE;
  if (D->T < 1 || D->N < 1 || D->N > 64 || D->k < 1 || D->k > D->N) return MIXLORA_E_SHAPE;
  if ((int64_t)D->T * D->k >= (1 << 24)) return MIXLORA_E_SHAPE;
  return MIXLORA_OK;
}
inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline int blocks_of(int T) { return (T + RL_THREADS - 1) / RL_THREADS; }
inline size_t stats_bytes(int N) { return ((size_t)(N + 1) * 4 + 255) / 256 * 256; }

RouterArgs args_of(const mixlora_router_dims &D, const void *logits, const unsigned char *mask, void *ws) {
  RouterArgs a{};
  a.logits = logits, a.mask = mask, a.T = D.T, a.N = D.N, a.k = D.k, a.top1 = D.aux_mode == MIXLORA_AUX_TOP1;
  a.balance = D.balance_coeff, a.zc = D.z_coeff;
  a.stats = (float *)ws;
  a.part = (float *)((char *)ws + stats_bytes(D.N));
  return a;
}

// one instance per storage type and row length
#define MIXLORA_ROUTER(KERNEL, D, ...)                                                                                \
  do {                                                                                                                \
    const dim3 grid_(blocks_of((D).T)), block_(RL_THREADS);                                                           \
    if ((D).dtype == MIXLORA_BF16) {                                                                                  \
      if ((D).N <= 8) hipLaunchKernelGGL((KERNEL<bf16_t, 8>), grid_, block_, 0, st, __VA_ARGS__);                     \
      else if ((D).N <= 16) hipLaunchKernelGGL((KERNEL<bf16_t, 16>), grid_, block_, 0, st, __VA_ARGS__);              \
      else hipLaunchKernelGGL((KERNEL<bf16_t, 64>), grid_, block_, 0, st, __VA_ARGS__);                               \
    } else {                                                                                                          \
      if ((D).N <= 8) hipLaunchKernelGGL((KERNEL<float, 8>), grid_, block_, 0, st, __VA_ARGS__);                      \
      else if ((D).N <= 16) hipLaunchKernelGGL((KERNEL<float, 16>), grid_, block_, 0, st, __VA_ARGS__);               \
      else hipLaunchKernelGGL((KERNEL<float, 64>), grid_, block_, 0, st, __VA_ARGS__);                                \
    }                                                                                                                 \
  } while (0)

}  // namespace

extern "C" {

size_t mixlora_router_loss_workspace_bytes(const mixlora_router_dims *dims) {
  if (check(dims) != MIXLORA_OK) return 0;
  return stats_bytes(dims->N) + ((size_t)blocks_of(dims->T) * (3 * dims->N + 2) * 4 + 255) / 256 * 256;
}

int mixlora_router_loss_forward(const mixlora_router_dims *dims, const void *logits, const unsigned char *token_mask,
                                float *loss, int32_t *counts, int32_t *topk_idx, float *topk_w, void *workspace,
                                size_t workspace_bytes, void *stream) {
  const int rc = check(dims);
  if (rc) return rc;
  if (!logits || !loss || !counts || !topk_idx || !topk_w || !workspace) return MIXLORA_E_NULL;
  for (const void *p : {logits, (const void *)loss, (const void *)counts, (const void *)topk_idx, (const void *)topk_w,
                        (const void *)workspace})
    if (misaligned(p)) return MIXLORA_E_ALIGN;
  if (workspace_bytes < mixlora_router_loss_workspace_bytes(dims)) return MIXLORA_E_WORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  RouterArgs a = args_of(*dims, logits, token_mask, workspace);
  a.idx = topk_idx, a.w = topk_w, a.loss = loss, a.counts = counts;
  MIXLORA_ROUTER(router_loss_forward_kernel, *dims, a);
  if (hipGetLastError() != hipSuccess) return MIXLORA_E_HIP;
  hipLaunchKernelGGL(router_loss_finish_kernel, dim3(1), dim3(256), 0, st, a, blocks_of(dims->T));
  return hipGetLastError() == hipSuccess ? MIXLORA_OK : MIXLORA_E_HIP;
}

int mixlora_router_loss_backward(const mixlora_router_dims *dims, const void *logits, const unsigned char *token_mask,
                                 const int32_t *topk_idx, const float *d_topk_w, float d_balance, float d_z,
                                 void *workspace, size_t workspace_bytes, void *dlogits, void *stream) {
  const int rc = check(dims);
  if (rc) return rc;
  if (!logits || !dlogits || !workspace || (d_topk_w && !topk_idx)) return MIXLORA_E_NULL;
  for (const void *p : {logits, (const void *)dlogits, (const void *)workspace, (const void *)topk_idx, (const void *)d_topk_w})
    if (misaligned(p)) return MIXLORA_E_ALIGN;
  if (workspace_bytes < mixlora_router_loss_workspace_bytes(dims)) return MIXLORA_E_WORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const RouterArgs a = args_of(*dims, logits, token_mask, workspace);
  MIXLORA_ROUTER(router_loss_backward_kernel, *dims, a, topk_idx, d_topk_w, d_balance, d_z, dlogits);
  return hipGetLastError() == hipSuccess ? MIXLORA_OK : MIXLORA_E_HIP;
}

}  // extern "C"
