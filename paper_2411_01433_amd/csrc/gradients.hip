// Norm of all gradients and their scaling.
//
//   norm = sqrt(sum g^2);  out = g * min(1, max_norm / (norm + 1e-6))
//
// A block per piece of a tensor.  Squares are summed in 64 bits throughout: no
// gradient of fp32 overflows or vanishes in its square, and the sum of 2^38 of
// them is right to fp32.  A piece's sum goes to its own place, and the block
// that ends last adds the places in a fixed order.
#include "moe_internal.h"

namespace moe {

namespace {

constexpr int kThreads = 256;

// Sum over the block, in every thread of wave 0.
__device__ inline double block_sum(double v, double* red) {
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
  for (int i = 0; i < kThreads / 64; ++i) v += red[i];
  return v;
}

template <class T>
__device__ inline double squares(const GradPiece& p) {
  double s = 0.0;
  for (int i = threadIdx.x; i < p.n; i += kThreads) {
    const double v = (double)(float)static_cast<const T*>(p.in)[i];
    s = fma(v, v, s);
  }
  return s;
}

template <class T>
__device__ inline void scaled(const GradPiece& p, float c) {
  for (int i = threadIdx.x; i < p.n; i += kThreads)
    static_cast<T*>(p.out)[i] = (T)((float)static_cast<const T*>(p.in)[i] * c);
}

}  // namespace

__global__ __launch_bounds__(kThreads) void gradients_norm_kernel(GradList g, float* norm) {
  __shared__ double red[2][kThreads / 64];
  __shared__ bool last;
  const GradPiece p = g.pieces[blockIdx.x];
  const double s = block_sum(p.type == TYPE_F32   ? squares<float>(p)
                             : p.type == TYPE_F16 ? squares<f16>(p)
                                                  : squares<bf16>(p),
                             red[0]);
  if (threadIdx.x == 0) {
    __hip_atomic_store(&g.sums[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(g.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
           gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  double t = 0.0;
  for (int i = threadIdx.x; i < g.n; i += kThreads)
    t += __hip_atomic_load(&g.sums[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  t = block_sum(t, red[1]);
  if (threadIdx.x == 0) {
    *norm = (float)sqrt(t);
    __hip_atomic_store(g.done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

__global__ __launch_bounds__(kThreads) void gradients_scale_kernel(GradList g, float max_norm,
                                                                   const float* norm) {
  const GradPiece p = g.pieces[blockIdx.x];
  const float t = *norm;
  // (in 64 bits: the quotient is then right to half a step of fp32)
  float c = (float)fmin((double)max_norm / ((double)t + 1e-6), 1.0);
  if (!__builtin_isfinite(t)) c = 1.0f;
  if (c == 1.0f && p.in == p.out) return;
  if (p.type == TYPE_F32) scaled<float>(p, c);
  else if (p.type == TYPE_F16) scaled<f16>(p, c);
  else scaled<bf16>(p, c);
}

hipError_t launch_gradients_norm(const GradList& g, float* norm, hipStream_t s) {
  gradients_norm_kernel<<<g.n, kThreads, 0, s>>>(g, norm);
  return hipGetLastError();
}

hipError_t launch_gradients_scale(const GradList& g, float max_norm, const float* norm,
                                  hipStream_t s) {
  gradients_scale_kernel<<<g.n, kThreads, 0, s>>>(g, max_norm, norm);
  return hipGetLastError();
}

}  // namespace moe
