// Softmax routing of given logits with Eq. 8-9 and a z-loss over the tokens that a mask keeps:
//   p = softmax(z), the k largest kept (ties to the lower index), w = their p over its sum;
//   n = tokens kept by the mask, F and P of Eq. 9 over them, balance = a N sum_i F_i P_i,
//   z_loss = b / n sum_t lse_t^2 with lse_t = log sum_i exp z_ti;
//   dz_ti = g_b a N / n p_ti (F_i - sum_j F_j p_tj) + g_z b 2 / n lse_t p_ti + [i kept] w_ti (dw_ti - sum_j w_tj dw_tj).
// A token that the mask drops is left out of every sum, whatever its logits are, and gets index -1, weight 0
// and a zero gradient.  Both directions read the logits once and are bound by a launch's latency (1 MB of
// logits at 16384 x 16), so up to 16 experts a thread takes a token and keeps its row in registers (beyond,
// a lane takes an expert).  Sums over tokens are made on the
// vector ALU, counts from ballots.  No sum depends on the order in which workgroups end: their partial sums are added
// in a fixed order, by a launch of its own.
#include "common.h"

#include <cmath>
#include <type_traits>

using namespace mixlora;

namespace {

constexpr int RL_THREADS = 64;   // one wavefront: 16384 tokens are one workgroup per CU
constexpr int RL_ALL = 1024;     // tokens that one workgroup takes
struct RouterArgs {
  const void *logits;
  const unsigned char *mask;
  int T, N, k, top1;
  float balance, zc;
  int32_t *idx;
  float *w;
  float *part;          // [workgroup or wavefront][3 N + 2]: P sums, counts of all slots, of slot 0 (whole numbers), z sum, tokens
  float *stats;         // [N + 1]: F, then 1 / n (0 where no token is kept)
  float *loss;
  int32_t *counts;
};

// A row in registers, -inf past N.  FULL: N == NR, whole 16-byte pieces.
template <typename E, int NR, bool FULL>
__device__ __forceinline__ void load_row(const E *row, int N, float (&z)[NR]) {
  if constexpr (FULL) {
#pragma unroll
    for (int i = 0; i < NR; i += 8) {
      Vec8<E> v;
      v.load(row + i);
#pragma unroll
      for (int e = 0; e < 8; e++) z[i + e] = v.get(e);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NR; i++) z[i] = i < N ? to_f32(row[i]) : -INFINITY;
  }
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

// sum over the wavefront on the vector ALU (lanes exchange with their quad, half row, row, then rows), for all lanes
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_total(float v) {
  v = dpp_add<0xb1>(v);    // quad_perm 1 0 3 2
  v = dpp_add<0x4e>(v);    // quad_perm 2 3 0 1
  v = dpp_add<0x141>(v);   // row_half_mirror
  v = dpp_add<0x140>(v);   // row_mirror: every lane has its row's sum
  const int b = __builtin_bit_cast(int, v);
  auto row = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(b, l)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}

// Adds the wavefronts' sums in double, each thread every G-th of them, then the G sums in order; called by all of a
// workgroup of `threads`, at least 3 N + 2.
__device__ void finish(const RouterArgs &a, int blocks, int threads) {
  __shared__ double part[1024];
  __shared__ double sums[3 * 64 + 2];
  __shared__ double fp[64];
  const int W = 3 * a.N + 2, tid = threadIdx.x, G = threads / W;
  const int i = tid % W, g = tid / W;
  if (g < G) {
    double s = 0.0;
    constexpr int INFLIGHT = 8;
    for (int b = g; b < blocks; b += INFLIGHT * G) {
      float v[INFLIGHT];
#pragma unroll
      for (int u = 0; u < INFLIGHT; u++) v[u] = a.part[(int64_t)(b + u * G < blocks ? b + u * G : b) * W + i];
#pragma unroll
      for (int u = 0; u < INFLIGHT; u++)
        if (b + u * G < blocks) s += v[u];
    }
    part[tid] = s;
  }
  __syncthreads();
  if (tid < W) {
    double s = 0.0;
    for (int u = 0; u < G; u++) s += part[u * W + tid];
    sums[tid] = s;
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
    for (int e = 0; e < a.N; e++) s += fp[e];
    const double balance = (double)a.balance * a.N * s, z = (double)a.zc * sums[3 * a.N] * inv;
    a.loss[0] = (float)(balance + z);
    a.loss[1] = (float)balance;
    a.loss[2] = (float)z;
    a.stats[a.N] = (float)inv;
  }
}

// ALL: one workgroup takes every token and adds its wavefronts' sums itself.
template <typename E, int NR, bool FULL, bool ALL>
__global__ __launch_bounds__(ALL ? RL_ALL : RL_THREADS) void router_loss_forward_kernel(RouterArgs a) {
  const int lane = threadIdx.x & 63, N = FULL ? NR : a.N, k = a.k;
  const int wave = blockIdx.x + (threadIdx.x >> 6);
  const int64_t t = (int64_t)wave * RL_THREADS + lane;
  const bool on = t < a.T && (!a.mask || a.mask[t]);
  float z[NR], lse = 0.f;
  uint64_t taken = 0;
  int first = -1;
  if (on) {
    load_row<E, NR, FULL>((const E *)a.logits + t * N, N, z);
    float raw[NR];   // NaN ranks with -inf
#pragma unroll
    for (int i = 0; i < NR; i++) raw[i] = isnan(z[i]) ? -INFINITY : z[i];
    lse = softmax_row<NR>(z, N);
    constexpr int KEEP = 8;   // weights that wait in registers for their sum; further ones wait in memory
    float sum = 0.f, wk[KEEP];
    int32_t *idx = a.idx + t * k;
    float *w = a.w + t * k;
    auto pick = [&](int &best, float &bp) {   // the largest that is left, the lowest index among equals
      best = -1;
      float bz = 0.f;
#pragma unroll
      for (int i = 0; i < NR; i++) {
        if (i < N && !(taken >> i & 1) && (best < 0 || raw[i] > bz)) best = i, bz = raw[i], bp = z[i];
      }
      taken |= 1ull << best;
      sum += bp;
    };
#pragma unroll
    for (int j = 0; j < KEEP; j++) {
      if (j >= k) break;
      int best;
      pick(best, wk[j]);
      if (j == 0) first = best;
      idx[j] = best;
    }
    for (int j = KEEP; j < k; j++) {
      int best;
      float bp = 0.f;
      pick(best, bp);
      idx[j] = best;
      w[j] = bp;
    }
#pragma unroll
    for (int j = 0; j < KEEP; j++)
      if (j < k) w[j] = wk[j] / sum;
    for (int j = KEEP; j < k; j++) w[j] /= sum;
  } else {
#pragma unroll
    for (int i = 0; i < NR; i++) z[i] = 0.f;
    if (t < a.T)
      for (int j = 0; j < k; j++) a.idx[t * k + j] = -1, a.w[t * k + j] = 0.f;
  }
  // lane i keeps expert i's sums
  float P = 0.f, all = 0.f, slot0 = 0.f;
#pragma unroll
  for (int i = 0; i < NR; i++) {
    if (i < N) {   // (uniform)
      const float s = wave_total(z[i]);
      const int c = __popcll(__ballot(taken >> i & 1)), f = __popcll(__ballot(first == i));
      if (lane == i) P = s, all = (float)c, slot0 = (float)f;
    }
  }
  const float zs = wave_total(lse * lse);
  const float n = (float)__popcll(__ballot(on));
  float *p = a.part + (int64_t)wave * (3 * N + 2);
  if (lane < N) p[lane] = P, p[N + lane] = all, p[2 * N + lane] = slot0;
  if (lane == 0) p[3 * N] = zs, p[3 * N + 1] = n;
  if constexpr (ALL) {
    __threadfence_block();
    __syncthreads();
    finish(a, blockDim.x >> 6, blockDim.x);
  }
}

__global__ __launch_bounds__(1024) void router_loss_finish_kernel(RouterArgs a, int waves) { finish(a, waves, 1024); }

template <typename E, int NR, bool FULL>
__global__ __launch_bounds__(RL_THREADS) void router_loss_backward_kernel(RouterArgs a, const int32_t *__restrict__ idx,
                                                                          const float *__restrict__ dw, float gb, float gz,
                                                                          void *__restrict__ dz) {
  const int64_t t = (int64_t)blockIdx.x * RL_THREADS + threadIdx.x;
  if (t >= a.T) return;
  const int N = FULL ? NR : a.N, k = a.k;
  float g[NR];
  if (a.mask && !a.mask[t]) {
#pragma unroll
    for (int i = 0; i < NR; i++) g[i] = 0.f;
  } else {
    float z[NR];
    load_row<E, NR, FULL>((const E *)a.logits + t * N, N, z);
    // g: the gradient of a kept expert's weight
#pragma unroll
    for (int i = 0; i < NR; i++) g[i] = 0.f;
    uint64_t kept = 0;
    if (dw) {
      for (int j = 0; j < k; j++) {
        const int e = idx[t * k + j];
        const float d = dw[t * k + j];
        if (e >= 0 && e < N) kept |= 1ull << e;
#pragma unroll
        for (int i = 0; i < NR; i++) g[i] = i == e ? d : g[i];
      }
    }
    const float lse = softmax_row<NR>(z, N);
    const float inv = a.stats[N];
    float fp = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < NR; i++) {
      if (i < N) fp = fmaf(a.stats[i], z[i], fp);
      sum += kept >> i & 1 ? z[i] : 0.f;
    }
    const float cb = gb * a.balance * (float)N * inv, cz = gz * a.zc * 2.f * inv * lse;
    // w = p over the kept ones' sum;  dz = w (dw - sum_j w_j dw_j) + the losses' share
    // (divided, not multiplied with a reciprocal: the weight of a single kept expert is 1 and its gradient nothing, beside
    // which the losses' share is small)
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NR; i++) dot = kept >> i & 1 ? fmaf(z[i] / sum, g[i], dot) : dot;
#pragma unroll
    for (int i = 0; i < NR; i++) {
      const float l = i < N ? z[i] * (cb * (a.stats[i] - fp) + cz) : 0.f;
      g[i] = kept >> i & 1 ? fmaf(z[i] / sum, g[i] - dot, l) : l;
    }
  }
  E *out = (E *)dz + t * N;
  if constexpr (FULL) {
#pragma unroll
    for (int i = 0; i < NR; i += 8) {
      Vec8<E> v;
#pragma unroll
      for (int e = 0; e < 8; e++) v.set(e, g[i + e]);
      v.store(out + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NR; i++)
      if (i < N) out[i] = from_f32<E>(g[i]);
  }
}

// ---- more than 16 experts: a lane takes an expert, a wavefront four tokens in turn ---------------------------------
// (with a token per thread, rows of 33 and 64 took 21 and 13 us per direction at 16384 tokens: exponentials and selections of
// one row behind one another, one wavefront per SIMD)
// 16 wavefronts per workgroup, four where that leaves most of the chip idle (more partial sums, but of few tokens)
constexpr int RW_TOKENS = 4, RW_WAVES = 16;
inline int wide_waves(int T) { return T <= 4096 ? 4 : RW_WAVES; }

template <int CTRL> __device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float lane_value(float v, int l) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
}
__device__ __forceinline__ float wave_max(float v) {   // (NaN counts as nothing)
  v = dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4e>(dpp_max<0xb1>(v))));
  return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
// softmax of a row held one element per lane (-inf past N)
__device__ __forceinline__ float wave_softmax(float z, bool in, float &lse) {
  const float top = wave_max(z);
  const float e = in ? expf(z - top) : 0.f;
  const float sum = wave_total(e);
  lse = top + logf(sum);
  return e * (1.f / sum);
}

template <typename E>
__global__ __launch_bounds__(RW_WAVES * 64) void router_loss_forward_wide_kernel(RouterArgs a) {
  __shared__ float sums[RW_WAVES][3][64];
  __shared__ float zn[RW_WAVES][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), N = a.N, k = a.k;
  const int waves = blockDim.x >> 6;
  const int64_t t0 = ((int64_t)blockIdx.x * waves + wave) * RW_TOKENS;
  const bool in = lane < N;
  float zr[RW_TOKENS];
  bool on[RW_TOKENS];
#pragma unroll
  for (int i = 0; i < RW_TOKENS; i++) {   // (a token past the last one: the last one's row, not used)
    const int64_t t = t0 + i < a.T ? t0 + i : a.T - 1;
    on[i] = t0 + i < a.T && (!a.mask || a.mask[t]);
    zr[i] = in ? to_f32(((const E *)a.logits)[t * N + lane]) : -INFINITY;
  }
  float P = 0.f, all = 0.f, slot0 = 0.f, zs = 0.f, n = 0.f;
#pragma unroll
  for (int i = 0; i < RW_TOKENS; i++) {
    const int64_t t = t0 + i;
    if (t >= a.T) break;
    if (!on[i]) {
      if (lane < k) a.idx[t * k + lane] = -1, a.w[t * k + lane] = 0.f;
      continue;
    }
    const float raw = isnan(zr[i]) ? -INFINITY : zr[i];   // NaN ranks with -inf
    float lse;
    const float p = wave_softmax(zr[i], in, lse);
    bool left = in;
    float kept = 0.f, w = 0.f;
    int e = 0;
    for (int j = 0; j < k; j++) {   // the largest that is left, the lowest index among equals
      const float top = wave_max(left ? raw : -INFINITY);
      const int best = __ffsll((unsigned long long)__ballot(left && raw == top)) - 1;
      const float pb = lane_value(p, best);
      kept += pb;
      if (lane == j) e = best, w = pb;
      if (lane == best) left = false;
      if (j == 0 && lane == best) slot0 += 1.f;
    }
    if (lane < k) a.idx[t * k + lane] = e, a.w[t * k + lane] = w / kept;
    P += p;
    all += in && !left ? 1.f : 0.f;
    zs += lse * lse;
    n += 1.f;
  }
  sums[wave][0][lane] = P, sums[wave][1][lane] = all, sums[wave][2][lane] = slot0;
  if (lane == 0) zn[wave][0] = zs, zn[wave][1] = n;
  __syncthreads();
  float *out = a.part + (int64_t)blockIdx.x * (3 * N + 2);
  for (int i = threadIdx.x; i < 3 * N + 2; i += blockDim.x) {
    float s = 0.f;
    for (int u = 0; u < waves; u++) s += i < 3 * N ? sums[u][i / N][i % N] : zn[u][i - 3 * N];
    out[i] = s;
  }
}

template <typename E>
__global__ __launch_bounds__(RW_WAVES * 64) void router_loss_backward_wide_kernel(RouterArgs a, const int32_t *__restrict__ idx,
                                                                                  const float *__restrict__ dw, float gb, float gz,
                                                                                  void *__restrict__ dz) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), N = a.N, k = a.k;
  const int64_t t0 = ((int64_t)blockIdx.x * (blockDim.x >> 6) + wave) * RW_TOKENS;
  const bool in = lane < N;
  const float F = in ? a.stats[lane] : 0.f, inv = a.stats[N];
  float zr[RW_TOKENS], dr[RW_TOKENS];
  int er[RW_TOKENS];
  bool on[RW_TOKENS];
#pragma unroll
  for (int i = 0; i < RW_TOKENS; i++) {
    const int64_t t = t0 + i < a.T ? t0 + i : a.T - 1;
    on[i] = t0 + i < a.T && (!a.mask || a.mask[t]);
    zr[i] = in ? to_f32(((const E *)a.logits)[t * N + lane]) : -INFINITY;
    er[i] = dw && lane < k ? idx[t * k + lane] : -1;
    dr[i] = dw && lane < k ? dw[t * k + lane] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < RW_TOKENS; i++) {
    const int64_t t = t0 + i;
    if (t >= a.T) break;
    float g = 0.f;
    if (on[i]) {
      float lse;
      const float p = wave_softmax(zr[i], in, lse);
      bool kept = false;
      if (dw)
        for (int j = 0; j < k; j++) {   // the gradient of a kept expert's weight to its lane
          const int e = __builtin_amdgcn_readlane(er[i], j);
          if (lane == e) kept = true, g = lane_value(dr[i], j);
        }
      kept = kept && in;
      const float fp = wave_total(F * p), sum = wave_total(kept ? p : 0.f);
      const float w = kept ? p / sum : 0.f;   // (divided: the weight of a single kept expert is 1)
      const float dot = wave_total(kept ? w * g : 0.f);
      const float l = p * (gb * a.balance * (float)N * inv * (F - fp) + gz * a.zc * 2.f * inv * lse);
      g = kept ? fmaf(w, g - dot, l) : l;
    }
    if (in) ((E *)dz)[t * N + lane] = from_f32<E>(g);
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
inline int wide_blocks(int T) { return (T + wide_waves(T) * RW_TOKENS - 1) / (wide_waves(T) * RW_TOKENS); }
inline size_t stats_bytes(int N) { return ((size_t)(N + 1) * 4 + 255) / 256 * 256; }

RouterArgs args_of(const mixlora_router_dims &D, const void *logits, const unsigned char *mask, void *ws) {
  RouterArgs a{};
  a.logits = logits, a.mask = mask, a.T = D.T, a.N = D.N, a.k = D.k, a.top1 = D.aux_mode == MIXLORA_AUX_TOP1;
  a.balance = D.balance_coeff, a.zc = D.z_coeff;
  a.stats = (float *)ws;
  a.part = (float *)((char *)ws + stats_bytes(D.N));
  return a;
}

template <typename E, int NR, bool FULL>
hipError_t launch_forward(const RouterArgs &a, hipStream_t st) {
  const int waves = blocks_of(a.T);
  if (a.T <= RL_ALL) {   // (300 x 8: 2.7 us of a second launch)
    hipLaunchKernelGGL((router_loss_forward_kernel<E, NR, FULL, true>), dim3(1), dim3(waves * 64), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((router_loss_forward_kernel<E, NR, FULL, false>), dim3(waves), dim3(RL_THREADS), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(router_loss_finish_kernel, dim3(1), dim3(1024), 0, st, a, waves);
  return hipGetLastError();
}
template <typename E, int NR, bool FULL>
hipError_t launch_backward(const RouterArgs &a, const int32_t *idx, const float *dw, float gb, float gz, void *dz, hipStream_t st) {
  hipLaunchKernelGGL((router_loss_backward_kernel<E, NR, FULL>), dim3(blocks_of(a.T)), dim3(RL_THREADS), 0, st, a, idx, dw, gb, gz, dz);
  return hipGetLastError();
}
// one instance per storage type and row length up to 16, with whole rows of 8 and 16 apart
template <typename F>
hipError_t by_row(int N, F &&f) {
  if (N == 8) return f(std::integral_constant<int, 8>{}, std::true_type{});
  if (N < 8) return f(std::integral_constant<int, 8>{}, std::false_type{});
  if (N == 16) return f(std::integral_constant<int, 16>{}, std::true_type{});
  return f(std::integral_constant<int, 16>{}, std::false_type{});
}
template <typename E>
hipError_t launch_forward_wide(const RouterArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(router_loss_forward_wide_kernel<E>, dim3(wide_blocks(a.T)), dim3(wide_waves(a.T) * 64), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(router_loss_finish_kernel, dim3(1), dim3(1024), 0, st, a, wide_blocks(a.T));
  return hipGetLastError();
}
template <typename E>
hipError_t launch_backward_wide(const RouterArgs &a, const int32_t *idx, const float *dw, float gb, float gz, void *dz, hipStream_t st) {
  hipLaunchKernelGGL(router_loss_backward_wide_kernel<E>, dim3(wide_blocks(a.T)), dim3(wide_waves(a.T) * 64), 0, st, a, idx, dw, gb, gz, dz);
  return hipGetLastError();
}

}  // namespace

extern "C" {

size_t mixlora_router_loss_workspace_bytes(const mixlora_router_dims *dims) {
  if (check(dims) != MIXLORA_OK) return 0;
  return stats_bytes(dims->N) + ((size_t)(dims->N > 16 ? wide_blocks(dims->T) : blocks_of(dims->T)) * (3 * dims->N + 2) * 4 + 255) / 256 * 256;
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
  const bool bf16 = dims->dtype == MIXLORA_BF16;
  if (dims->N > 16)
    return (bf16 ? launch_forward_wide<bf16_t>(a, st) : launch_forward_wide<float>(a, st)) == hipSuccess ? MIXLORA_OK : MIXLORA_E_HIP;
  const hipError_t e = by_row(dims->N, [&](auto nr, auto full) {
    return bf16 ? launch_forward<bf16_t, nr.value, full.value>(a, st)
                : launch_forward<float, nr.value, full.value>(a, st);
  });
  return e == hipSuccess ? MIXLORA_OK : MIXLORA_E_HIP;
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
  const bool bf16 = dims->dtype == MIXLORA_BF16;
  if (dims->N > 16)
    return (bf16 ? launch_backward_wide<bf16_t>(a, topk_idx, d_topk_w, d_balance, d_z, dlogits, st)
                 : launch_backward_wide<float>(a, topk_idx, d_topk_w, d_balance, d_z, dlogits, st)) == hipSuccess ? MIXLORA_OK : MIXLORA_E_HIP;
  const hipError_t e = by_row(dims->N, [&](auto nr, auto full) {
    return bf16
               ? launch_backward<bf16_t, nr.value, full.value>(a, topk_idx, d_topk_w, d_balance, d_z, dlogits, st)
               : launch_backward<float, nr.value, full.value>(a, topk_idx, d_topk_w, d_balance, d_z, dlogits, st);
  });
  return e == hipSuccess ? MIXLORA_OK : MIXLORA_E_HIP;
}

}  // extern "C"
