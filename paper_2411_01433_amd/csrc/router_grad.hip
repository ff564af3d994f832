// Backward pass of the routing rules (router.hip): from the gradients g of
// the selected experts' weights, and any of the logits themselves, to those
// of x and Wg.  With s the scores, p the shares of the selected scores and c
// the scale, the gradient of the logits is
//
//   renormalised softmax    dl_k = c p_k (g_k - sum_j g_j p_j)
//   renormalised sigmoid    the same times (1 - s_k)
//   softmax of all experts  dl_e = c s_e ([e selected] g_e - sum_j g_j s_j)
//   sigmoid                 dl_k = c g_k s_k (1 - s_k)
//
// and then  d_x = dl Wg,  d_Wg = dl^T x.
#include "moe_internal.h"

namespace moe {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ inline bool finite(float v) { return fabsf(v) <= 3.402823466e38f; }

__device__ inline float wave_max_f(float v) {
  for (int m = 1; m < 64; m <<= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
  return v;
}

// Gradient of one token's logits by one wave: lane k has slot k, lane i the
// experts i, i + 64, ...
template <int C>
__global__ __launch_bounds__(kThreads) void router_dlogits_kernel(
    RouterParams p, int T, const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const float* __restrict__ dw, const float* __restrict__ dl) {
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (t >= T) return;
  const float* lr = logits + (int64_t)t * p.E;
  const float none = -__builtin_inff();
  int e = -1;
  float g = 0.0f, l = none;
  if (lane < p.K) {
    e = idx[(int64_t)t * p.K + lane];
    if (e >= 0 && e < p.E) l = lr[e];
    if (finite(l)) g = p.scale * dw[(int64_t)t * p.K + lane];
    else e = -1;
  }
  const bool have = e >= 0;
  // s (1 - s) = 1 / ((1 + z) (1 + 1/z)); 1 - s = 1 / (1 + exp l)
  const float z = expf(-fabsf(l));
  const float not_s = have ? (l >= 0.0f ? z : 1.0f) / (1.0f + z) : 0.0f;
  const float s = have ? (l >= 0.0f ? 1.0f : z) / (1.0f + z) : 0.0f;
  const bool sig = p.score == SCORE_SIGMOID;
  float row[C], all = 0.0f, mean = 0.0f, slot = 0.0f;
  if (p.renorm) {
    const float ls = !have ? none : sig ? fminf(l, 0.0f) - log1pf(z) : l;
    const float lm = wave_max_f(ls);
    const float ex = have ? expf(ls - lm) : 0.0f;
    const float sum = wave_sum_dpp(ex);
    const float share = have ? ex / sum : 0.0f;
    mean = wave_sum_dpp(g * share);
    slot = share * (g - mean) * (sig ? not_s : 1.0f);
  } else if (sig) {
    slot = g * s * not_s;
  } else {
    float top = none;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int ee = c * 64 + lane;
      row[c] = ee < p.E ? lr[ee] : none;
      if (finite(row[c])) top = fmaxf(top, row[c]);
    }
    top = wave_max_f(top);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      row[c] = finite(row[c]) ? expf(row[c] - top) : 0.0f;
      all += row[c];
    }
    all = wave_sum_dpp(all);
    const float pk = have ? expf(l - top) / all : 0.0f;
    mean = wave_sum_dpp(g * pk);
    slot = g * pk;
  }
  const bool full = !p.renorm && !sig;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int ee = c * 64 + lane;
    float v = full && row[c] > 0.0f ? -mean * (row[c] / all) : 0.0f;
    for (int k = 0; k < p.K; ++k) {
      const int ek = __shfl(e, k, 64);
      const float gk = __shfl(slot, k, 64);
      if (ek == ee) v += gk;
    }
    if (ee < p.E) {
      const int64_t i = (int64_t)t * p.E + ee;
      p.d_logits[i] = dl ? v + dl[i] : v;
    }
  }
}

// d_x[t, c] = sum_e dl[t, e] Wg[e, c]: 16 tokens x 256 columns per block.
constexpr int kDxTokens = 16;
template <class T16>
__global__ __launch_bounds__(kThreads) void router_dx_kernel(RouterParams p, int T, T16* __restrict__ dx) {
  __shared__ float rows[kDxTokens][64];
  const int t0 = blockIdx.y * kDxTokens, c = blockIdx.x * kThreads + threadIdx.x;
  const T16* wg = static_cast<const T16*>(p.wg);
  float acc[kDxTokens];
#pragma unroll
  for (int i = 0; i < kDxTokens; ++i) acc[i] = 0.0f;
  for (int e0 = 0; e0 < p.E; e0 += 64) {
    for (int v = threadIdx.x; v < kDxTokens * 64; v += kThreads) {
      const int i = v >> 6, e = e0 + (v & 63);
      rows[i][v & 63] = t0 + i < T && e < p.E ? p.d_logits[(int64_t)(t0 + i) * p.E + e] : 0.0f;
    }
    __syncthreads();
    if (c < p.d)
      for (int e = e0; e < min(e0 + 64, p.E); ++e) {
        const float w = (float)wg[(int64_t)e * p.d + c];
#pragma unroll
        for (int i = 0; i < kDxTokens; ++i) acc[i] = fmaf(rows[i][e - e0], w, acc[i]);
      }
    __syncthreads();
  }
  if (c < p.d)
    for (int i = 0; i < kDxTokens; ++i)
      if (t0 + i < T) dx[(int64_t)(t0 + i) * p.d + c] = (T16)acc[i];
}

// d_Wg[e, c] = sum_t dl[t, e] x[t, c]: 8 experts x 256 columns per block; the
// tokens in runs of 64 whose sums are added, so that a long sum keeps its bits.
constexpr int kDwExperts = 8;
template <class T16>
__global__ __launch_bounds__(kThreads) void router_dw_kernel(RouterParams p, int T,
                                                             const T16* __restrict__ x,
                                                             float* __restrict__ dwg) {
  __shared__ float rows[64][kDwExperts];
  const int e0 = blockIdx.y * kDwExperts, c = blockIdx.x * kThreads + threadIdx.x;
  float acc[kDwExperts];
#pragma unroll
  for (int i = 0; i < kDwExperts; ++i) acc[i] = 0.0f;
  for (int t0 = 0; t0 < T; t0 += 64) {
    for (int v = threadIdx.x; v < 64 * kDwExperts; v += kThreads) {
      const int t = t0 + v / kDwExperts, e = e0 + v % kDwExperts;
      rows[v / kDwExperts][v % kDwExperts] = t < T && e < p.E ? p.d_logits[(int64_t)t * p.E + e] : 0.0f;
    }
    __syncthreads();
    if (c < p.d) {
      float run[kDwExperts];
#pragma unroll
      for (int i = 0; i < kDwExperts; ++i) run[i] = 0.0f;
      for (int t = t0; t < min(t0 + 64, T); ++t) {
        const float v = (float)x[(int64_t)t * p.d + c];
#pragma unroll
        for (int i = 0; i < kDwExperts; ++i) run[i] = fmaf(rows[t - t0][i], v, run[i]);
      }
#pragma unroll
      for (int i = 0; i < kDwExperts; ++i) acc[i] += run[i];
    }
    __syncthreads();
  }
  if (c < p.d)
    for (int i = 0; i < kDwExperts; ++i)
      if (e0 + i < p.E) dwg[(int64_t)(e0 + i) * p.d + c] = acc[i];
}

template <class T16>
hipError_t products(const RouterParams& p, int T, const T16* x, T16* dx, float* dwg, hipStream_t s) {
  const int cols = (p.d + kThreads - 1) / kThreads;
  if (dx) {
    router_dx_kernel<T16><<<dim3(cols, (T + kDxTokens - 1) / kDxTokens), kThreads, 0, s>>>(p, T, dx);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (dwg)
    router_dw_kernel<T16><<<dim3(cols, (p.E + kDwExperts - 1) / kDwExperts), kThreads, 0, s>>>(p, T, x, dwg);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_router_backward(const RouterParams& p, int T, const void* x, const float* logits,
                                  const int32_t* idx, const float* dw, const float* dl, void* dx,
                                  float* dwg, hipStream_t s) {
  const int grid = (T + kWaves - 1) / kWaves;
  if (p.E <= 64) router_dlogits_kernel<1><<<grid, kThreads, 0, s>>>(p, T, logits, idx, dw, dl);
  else if (p.E <= 128) router_dlogits_kernel<2><<<grid, kThreads, 0, s>>>(p, T, logits, idx, dw, dl);
  else if (p.E <= 256) router_dlogits_kernel<4><<<grid, kThreads, 0, s>>>(p, T, logits, idx, dw, dl);
  else router_dlogits_kernel<8><<<grid, kThreads, 0, s>>>(p, T, logits, idx, dw, dl);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return p.type == TYPE_F16
             ? products(p, T, static_cast<const f16*>(x), static_cast<f16*>(dx), dwg, s)
             : products(p, T, static_cast<const bf16*>(x), static_cast<bf16*>(dx), dwg, s);
}

}  // namespace moe
