// Norm of all gradients and their scaling.
//
//   norm = sqrt(sum g^2);  out = g * min(1, max_norm / (norm + 1e-6))
//
// Squares are summed in 64 bits throughout: no gradient of fp32 overflows or
// vanishes in its square, and the sum of 2^38 of them is right to fp32.  The
// list holds pieces of tensors; a block takes every kBlocks-th one and leaves
// one sum.  Those are added in a fixed order by the block that ends last, or,
// where the scaling follows, by every block of it for itself (a block that
// waits for the last one would hold all of them up).
//
// Bound by memory: the gradients pass twice, and are written once.  The scaling
// takes the pieces from the end of the list on, since what the norm read last
// is still in the caches (405 us instead of 438 below).
//
// Measured: 0.81 GB of fp32 gradients in 6 tensors 405 us, 118 for the norm (6.8
// TB/s) and 288 for the scaling (5.5 TB/s read and written); 2.6 MB in 48 tensors
// 7.9, of which the two kernels take 3.2 and 4.0.  One element at a time they took
// 834 and 35.  Stores pass the caches by: 405, others 454.  In bf16 and fp16 0.81
// GB 400, 0.40 GB 200; with pieces that the unrolled loops below did not fit (16
// KB) 500 and 256, with these half as deep 409 and 203.
#include "moe_internal.h"

namespace moe {

namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 8;   // vectors of 16 bytes that a thread has in flight
static_assert(kPieceBytes >= kVecs * kThreads * 16, "a piece fills the unrolled loops, of any type");

template <class T> struct Vec;
template <> struct Vec<float> { typedef float V __attribute__((ext_vector_type(4))); };
template <> struct Vec<f16> { typedef f16 V __attribute__((ext_vector_type(8))); };
template <> struct Vec<bf16> { typedef bf16 V __attribute__((ext_vector_type(8))); };

// Sum over the block, in every thread.
__device__ inline double block_sum(double v, double* red) {
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) v += red[i];
  return v;
}

// The norm from the blocks' sums, in every thread, always in the same order.
__device__ inline float joined(const GradList& g, double* red) {
  double t = 0.0;
  for (int i = threadIdx.x; i < g.blocks; i += kThreads)
    t += __hip_atomic_load(&g.sums[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return (float)sqrt(block_sum(t, red));
}

// Elements of a piece before its first 16-byte boundary.
template <class T>
__device__ inline int head_of(const void* p, int n) {
  return min(n, (int)((0 - (uintptr_t)p & 15) / sizeof(T)));
}

template <class T>
__device__ inline double squares(const GradPiece& p, double s) {
  typedef typename Vec<T>::V V;
  constexpr int kN = 16 / sizeof(T);
  const T* in = static_cast<const T*>(p.in);
  auto add = [&](T x) {
    const double v = (double)(float)x;
    s = fma(v, v, s);
  };
  const int head = head_of<T>(in, p.n), vecs = (p.n - head) / kN;
  const V* body = reinterpret_cast<const V*>(in + head);
  int i = threadIdx.x;
  for (; i + (kVecs - 1) * kThreads < vecs; i += kVecs * kThreads) {
    V v[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) v[j] = __builtin_nontemporal_load(body + i + j * kThreads);
#pragma unroll
    for (int j = 0; j < kVecs; ++j)
#pragma unroll
      for (int k = 0; k < kN; ++k) add(v[j][k]);
  }
  for (; i < vecs; i += kThreads) {
    const V v = body[i];
#pragma unroll
    for (int k = 0; k < kN; ++k) add(v[k]);
  }
  const int rest = p.n - vecs * kN;  // head and tail
  if ((int)threadIdx.x < rest) add(in[(int)threadIdx.x < head ? threadIdx.x : threadIdx.x + vecs * kN]);
  return s;
}

template <class T>
__device__ inline void scaled(const GradPiece& p, float c) {
  typedef typename Vec<T>::V V;
  constexpr int kN = 16 / sizeof(T);
  const T* in = static_cast<const T*>(p.in);
  T* out = static_cast<T*>(p.out);
  // one element at a time where in and out lie differently on 16 bytes: outs one
  // element off, 0.81 GB of fp32 648 us instead of 403, 0.40 GB of 16 bits 499
  // instead of 200
  const bool together = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
  const int head = together ? head_of<T>(in, p.n) : 0, vecs = together ? (p.n - head) / kN : 0;
  const V* body = reinterpret_cast<const V*>(in + head);
  V* to = reinterpret_cast<V*>(out + head);
  auto times = [&](V v) {
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = (T)((float)v[k] * c);
    return v;
  };
  int i = threadIdx.x;
  for (; i + (kVecs - 1) * kThreads < vecs; i += kVecs * kThreads) {
    V v[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) v[j] = __builtin_nontemporal_load(body + i + j * kThreads);
#pragma unroll
    for (int j = 0; j < kVecs; ++j) __builtin_nontemporal_store(times(v[j]), to + i + j * kThreads);
  }
  for (; i < vecs; i += kThreads) to[i] = times(body[i]);
  const int rest = p.n - vecs * kN;
  for (int j = threadIdx.x; j < rest; j += kThreads) {
    const int at = j < head ? j : j + vecs * kN;
    out[at] = (T)((float)in[at] * c);
  }
}

}  // namespace

template <bool LAST>
__global__ __launch_bounds__(kThreads) void gradients_norm_kernel(GradList g, float* norm) {
  __shared__ double red[2][kThreads / 64];
  __shared__ bool last;
  double s = 0.0;
  for (int i = blockIdx.x; i < g.n; i += gridDim.x) {
    const GradPiece p = g.pieces[i];
    s = p.type == TYPE_F32 ? squares<float>(p, s) : p.type == TYPE_F16 ? squares<f16>(p, s) : squares<bf16>(p, s);
  }
  s = block_sum(s, red[0]);
  if (!LAST) {
    if (threadIdx.x == 0) g.sums[blockIdx.x] = s;
    return;
  }
  if (threadIdx.x == 0) {
    __hip_atomic_store(&g.sums[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(g.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
           gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  const float t = joined(g, red[1]);
  if (threadIdx.x == 0) {
    *norm = t;
    __hip_atomic_store(g.done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

template <bool JOIN>
__global__ __launch_bounds__(kThreads) void gradients_scale_kernel(GradList g, float max_norm,
                                                                   float* norm) {
  __shared__ double red[kThreads / 64];
  const float t = JOIN ? joined(g, red) : *norm;
  if (JOIN && blockIdx.x == 0 && threadIdx.x == 0) *norm = t;
  // (in 64 bits: the quotient is then right to half a step of fp32)
  float c = (float)fmin((double)max_norm / ((double)t + 1e-6), 1.0);
  if (!__builtin_isfinite(t)) c = 1.0f;
  for (int i = g.n - 1 - (int)blockIdx.x; i >= 0; i -= gridDim.x) {
    const GradPiece p = g.pieces[i];
    if (c == 1.0f && p.in == p.out) continue;
    if (p.type == TYPE_F32) scaled<float>(p, c);
    else if (p.type == TYPE_F16) scaled<f16>(p, c);
    else scaled<bf16>(p, c);
  }
}

hipError_t launch_gradients_norm(const GradList& g, float* norm, hipStream_t s) {
  gradients_norm_kernel<true><<<g.blocks, kThreads, 0, s>>>(g, norm);
  return hipGetLastError();
}

hipError_t launch_gradients_scale(const GradList& g, float max_norm, const float* norm,
                                  hipStream_t s) {
  gradients_scale_kernel<false><<<g.blocks, kThreads, 0, s>>>(g, max_norm, const_cast<float*>(norm));
  return hipGetLastError();
}

hipError_t launch_gradients_clip(const GradList& g, float max_norm, float* norm, hipStream_t s) {
  gradients_norm_kernel<false><<<g.blocks, kThreads, 0, s>>>(g, norm);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  gradients_scale_kernel<true><<<g.blocks, kThreads, 0, s>>>(g, max_norm, norm);
  return hipGetLastError();
}

}  // namespace moe
