// Matrix products grouped by expert, forward and backward.
//
//   y[r]   = W[e(r)] x[r]                 r over the rows of expert e(r)
//   d_x[r] = W[e(r)]^T d_y[r]
//   d_W[e] = sum over the rows r of e of d_y[r] x[r]^T
#include "grouped.h"

namespace moe {

namespace {

constexpr int kTile = 64, kDepth = 16;

// c[64, 64] += a[64, n] b[64, n]^T by 256 threads, 4 x 4 each; a(i, k), b(j, k)
// give fp32 elements (0 outside).
template <class A, class B>
__device__ inline void tile(int n, float (&c)[4][4], A a, B b) {
  __shared__ float as[kDepth][kTile + 1], bs[kDepth][kTile + 1];
  const int ti = threadIdx.x >> 4, tj = threadIdx.x & 15;
  for (int k0 = 0; k0 < n; k0 += kDepth) {
    for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
      const int r = i / kDepth, k = i % kDepth;
      as[k][r] = k0 + k < n ? a(r, k0 + k) : 0.0f;
      bs[k][r] = k0 + k < n ? b(r, k0 + k) : 0.0f;
    }
    __syncthreads();
    for (int k = 0; k < kDepth; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) c[i][j] = fmaf(as[k][4 * ti + i], bs[k][4 * tj + j], c[i][j]);
    __syncthreads();
  }
}

template <class T>
__global__ __launch_bounds__(256) void product_kernel(Grouped g, const T* x, const T* w, T* y) {
  const Rows rows = expert_rows(g, blockIdx.z);
  const int n0 = blockIdx.x * kTile;
  const int64_t wb = (int64_t)blockIdx.z * g.d_out + n0;
  for (int r0 = blockIdx.y * kTile; r0 < rows.n; r0 += gridDim.y * kTile) {
    const int64_t xb = rows.first + r0;
    float c[4][4] = {};
    tile(g.d_in, c,
         [&](int i, int k) { return r0 + i < rows.n ? (float)x[(xb + i) * g.d_in + k] : 0.0f; },
         [&](int j, int k) { return (float)w[(wb + j) * g.d_in + k]; });
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const int r = (threadIdx.x >> 4) * 4 + i, n = (threadIdx.x & 15) * 4 + j;
        if (r0 + r < rows.n) y[(xb + r) * g.d_out + n0 + n] = (T)c[i][j];
      }
  }
}

template <class T>
__global__ __launch_bounds__(256) void dx_kernel(Grouped g, const T* dy, const T* w, T* dx) {
  const Rows rows = expert_rows(g, blockIdx.z);
  const int k0 = blockIdx.x * kTile;
  const int64_t wb = (int64_t)blockIdx.z * g.d_out;
  for (int r0 = blockIdx.y * kTile; r0 < rows.n; r0 += gridDim.y * kTile) {
    const int64_t xb = rows.first + r0;
    float c[4][4] = {};
    tile(g.d_out, c,
         [&](int i, int n) { return r0 + i < rows.n ? (float)dy[(xb + i) * g.d_out + n] : 0.0f; },
         [&](int j, int n) { return (float)w[(wb + n) * g.d_in + k0 + j]; });
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const int r = (threadIdx.x >> 4) * 4 + i, k = (threadIdx.x & 15) * 4 + j;
        if (r0 + r < rows.n) dx[(xb + r) * g.d_in + k0 + k] = (T)c[i][j];
      }
  }
}

template <class T>
__global__ __launch_bounds__(256) void dw_kernel(Grouped g, const T* dy, const T* x, float* dw,
                                                 bool accumulate) {
  const Rows rows = expert_rows(g, blockIdx.z);
  const int n0 = blockIdx.y * kTile, k0 = blockIdx.x * kTile;
  const int64_t xb = rows.first;
  float c[4][4] = {};
  tile(rows.n, c, [&](int i, int r) { return (float)dy[(xb + r) * g.d_out + n0 + i]; },
       [&](int j, int r) { return (float)x[(xb + r) * g.d_in + k0 + j]; });
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int n = (threadIdx.x >> 4) * 4 + i, k = (threadIdx.x & 15) * 4 + j;
      float* out = dw + ((int64_t)blockIdx.z * g.d_out + n0 + n) * g.d_in + k0 + k;
      *out = accumulate ? *out + c[i][j] : c[i][j];
    }
}

unsigned row_blocks(const Grouped& g) { return min((g.n + kTile - 1) / kTile, 256); }

}  // namespace

hipError_t launch_grouped_product(const Grouped& g, const void* x, const void* w, void* y,
                                  hipStream_t s) {
  const dim3 grid(g.d_out / kTile, row_blocks(g), g.E);
  if (g.type == TYPE_F16)
    product_kernel<<<grid, 256, 0, s>>>(g, (const f16*)x, (const f16*)w, (f16*)y);
  else
    product_kernel<<<grid, 256, 0, s>>>(g, (const bf16*)x, (const bf16*)w, (bf16*)y);
  return hipGetLastError();
}

hipError_t launch_grouped_dx(const Grouped& g, const void* dy, const void* w, void* dx,
                             hipStream_t s) {
  const dim3 grid(g.d_in / kTile, row_blocks(g), g.E);
  if (g.type == TYPE_F16)
    dx_kernel<<<grid, 256, 0, s>>>(g, (const f16*)dy, (const f16*)w, (f16*)dx);
  else
    dx_kernel<<<grid, 256, 0, s>>>(g, (const bf16*)dy, (const bf16*)w, (bf16*)dx);
  return hipGetLastError();
}

hipError_t launch_grouped_dw(const Grouped& g, const void* dy, const void* x, float* dw,
                             bool accumulate, hipStream_t s) {
  const dim3 grid(g.d_in / kTile, g.d_out / kTile, g.E);
  if (g.type == TYPE_F16)
    dw_kernel<<<grid, 256, 0, s>>>(g, (const f16*)dy, (const f16*)x, dw, accumulate);
  else
    dw_kernel<<<grid, 256, 0, s>>>(g, (const bf16*)dy, (const bf16*)x, dw, accumulate);
  return hipGetLastError();
}

}  // namespace moe
