// Products grouped by expert with weights in MXFP4, and activations of 16 bits
// or in MXFP4 too.
#include "grouped.h"

namespace moe {

namespace {

constexpr int kTile = 64, kDepth = 32;

// (in 64 bits: 6 * 2^127 is beyond fp32, its product with a small partner is not)
__device__ inline double mx_value(const uint8_t* row, const uint8_t* scales, int k) {
  const uint32_t b = scales[k / 32];
  const uint32_t c = row[k / 2] >> (4 * (k & 1)) & 15;
  const uint32_t m = c & 7;
  const float v = m < 2 ? 0.5f * m : (float)(2 + (m & 1)) * (float)(1 << (m >> 1)) * 0.25f;
  const uint64_t s = b == 255 ? 0x7FF8ull << 48 : (uint64_t)(b + 896) << 52;
  return (double)(c & 8 ? -v : v) * __builtin_bit_cast(double, s);
}

template <class T, bool MX>
__global__ __launch_bounds__(256) void mx_product_kernel(Grouped g, const void* x,
                                                         const uint8_t* xs, const uint8_t* w,
                                                         const uint8_t* ws, T* y) {
  __shared__ double as[kDepth][kTile + 1], bs[kDepth][kTile + 1];
  const Rows rows = expert_rows(g, blockIdx.z);
  const int n0 = blockIdx.x * kTile;
  const int64_t wb = (int64_t)blockIdx.z * g.d_out + n0;
  for (int r0 = blockIdx.y * kTile; r0 < rows.n; r0 += gridDim.y * kTile) {
    const int64_t xb = rows.first + r0;
    float c[4][4] = {};
    for (int k0 = 0; k0 < g.d_in; k0 += kDepth) {
      for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
        const int r = i / kDepth, k = i % kDepth;
        double a = 0.0;
        if (r0 + r < rows.n) {
          if (MX)
            a = mx_value(static_cast<const uint8_t*>(x) + (xb + r) * (g.d_in / 2),
                         xs + (xb + r) * (g.d_in / 32), k0 + k);
          else
            a = (double)(float)static_cast<const T*>(x)[(xb + r) * g.d_in + k0 + k];
        }
        as[k][r] = a;
        const double v = mx_value(w + (wb + r) * (g.d_in / 2), ws + (wb + r) * (g.d_in / 32), k0 + k);
        bs[k][r] = MX ? v : (double)(float)(T)(float)v;
      }
      __syncthreads();
      for (int k = 0; k < kDepth; ++k)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j)
            c[i][j] += (float)(as[k][(threadIdx.x >> 4) * 4 + i] * bs[k][(threadIdx.x & 15) * 4 + j]);
      __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const int r = (threadIdx.x >> 4) * 4 + i, n = (threadIdx.x & 15) * 4 + j;
        if (r0 + r < rows.n) y[(xb + r) * g.d_out + n0 + n] = (T)c[i][j];
      }
  }
}

template <class T>
void launch(const Grouped& g, const void* x, const uint8_t* xs, const uint8_t* w,
            const uint8_t* ws, T* y, hipStream_t s) {
  const dim3 grid(g.d_out / kTile, min((g.n + kTile - 1) / kTile, 256), g.E);
  if (xs)
    mx_product_kernel<T, true><<<grid, 256, 0, s>>>(g, x, xs, w, ws, y);
  else
    mx_product_kernel<T, false><<<grid, 256, 0, s>>>(g, x, xs, w, ws, y);
}

}  // namespace

hipError_t launch_mx_product(const Grouped& g, const void* x, const uint8_t* xs,
                             const uint8_t* w, const uint8_t* ws, void* y, hipStream_t s) {
  if (g.type == TYPE_F16)
    launch(g, x, xs, w, ws, (f16*)y, s);
  else
    launch(g, x, xs, w, ws, (bf16*)y, s);
  return hipGetLastError();
}

}  // namespace moe
