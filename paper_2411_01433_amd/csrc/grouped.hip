// Matrix products grouped by expert, forward and backward.
//
//   y[r]   = W[e(r)] x[r]                 r over the rows of expert e(r)
//   d_x[r] = W[e(r)]^T d_y[r]
//   d_W[e] = sum over the rows r of e of d_y[r] x[r]^T
//
// All three on the tiles of tile.h; the operand whose index is contiguous in
// the output is A.
#include "grouped.h"
#include "tile.h"

namespace moe {

namespace {

using namespace tile;

constexpr int kSuper = 8;  // row tiles that alternate fastest

template <int TYPE> struct Elem { typedef f16 T; };
template <> struct Elem<BF16> { typedef bf16 T; };

// Blocks of 64 TA columns and up to M = 64 TA rows, with the LDS of one (TA 4)
// or two (TA 2) blocks per unit.
template <int TA> constexpr int kLds = TA == 4 ? 160 * 1024 : 80 * 1024;
template <int TA> constexpr int kRows = 64 * TA;

template <int TYPE, int TA, int TB>
__device__ __forceinline__ void product_tile(const Grouped& g, const RowTile& t, const void* x,
                                             const void* w, void* y, lds_u8* lds) {
  typedef typename Elem<TYPE>::T T;
  const int col = t.part * 64 * TA;
  const T* wt = static_cast<const T*>(w) + ((int64_t)t.expert * g.d_out + col) * g.d_in;
  const T* xt = static_cast<const T*>(x) + (int64_t)t.row * g.d_in;
  const uint32_t bytes = 2 * g.d_in;
  Acc<TA, TB> acc;
  product<TYPE, ROWS, ROWS, TA, TB, kLds<TA>>({(const uint8_t*)wt, bytes, g.d_out - col},
                                              {(const uint8_t*)xt, bytes, t.n}, g.d_in, lds, acc);
  store_rows<T, TA, TB>(acc, static_cast<T*>(y) + (int64_t)t.row * g.d_out + col, g.d_out, t.n,
                        g.d_out - col);
}

template <int TYPE, int TA, int TB>
__device__ __forceinline__ void dx_tile(const Grouped& g, const RowTile& t, const void* dy,
                                        const void* w, void* dx, lds_u8* lds) {
  typedef typename Elem<TYPE>::T T;
  const int col = t.part * 64 * TA;
  const T* wt = static_cast<const T*>(w) + (int64_t)t.expert * g.d_out * g.d_in + col;
  const T* yt = static_cast<const T*>(dy) + (int64_t)t.row * g.d_out;
  Acc<TA, TB> acc;
  product<TYPE, COLS, ROWS, TA, TB, kLds<TA>>(
      {(const uint8_t*)wt, (uint32_t)(2 * g.d_in), g.d_in - col},
      {(const uint8_t*)yt, (uint32_t)(2 * g.d_out), t.n}, g.d_out, lds, acc);
  store_rows<T, TA, TB>(acc, static_cast<T*>(dx) + (int64_t)t.row * g.d_in + col, g.d_in, t.n,
                        g.d_in - col);
}

template <int TYPE, int TA, int TB>
__device__ __forceinline__ void dw_tile(const Grouped& g, const Rows& rows, int expert, int a0,
                                        int b0, const void* dy, const void* x, float* dw,
                                        bool accumulate, lds_u8* lds) {
  typedef typename Elem<TYPE>::T T;
  const T* xt = static_cast<const T*>(x) + (int64_t)rows.first * g.d_in + a0;
  const T* yt = static_cast<const T*>(dy) + (int64_t)rows.first * g.d_out + b0;
  Acc<TA, TB> acc;
  product<TYPE, COLS, COLS, TA, TB, kLds<TA>>(
      {(const uint8_t*)xt, (uint32_t)(2 * g.d_in), g.d_in - a0},
      {(const uint8_t*)yt, (uint32_t)(2 * g.d_out), g.d_out - b0}, rows.n, lds, acc);
  const int l = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int aw = (wave >> 1) * TA * 32, bw = (wave & 1) * TB * 32;
  float* out = dw + ((int64_t)expert * g.d_out + b0 + bw + (l & 31)) * g.d_in + a0 + aw + 4 * (l >> 5);
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    if (b0 + bw + 32 * j >= g.d_out) continue;
#pragma unroll
    for (int i = 0; i < TA; ++i) {
      if (a0 + aw + 32 * i >= g.d_in) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4* to = reinterpret_cast<f32x4*>(out + (int64_t)32 * j * g.d_in + 32 * i + 8 * q);
        const f32x16& c = acc[i][j];
        f32x4 v = {c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
        if (accumulate) v += *to;
        *to = v;
      }
    }
  }
}

template <int TYPE, int TA>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(TA == 4 ? 1 : 2, TA == 4 ? 1 : 2)))
void product_kernel(Grouped g, const void* x, const void* w, void* y, int parts) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLds<TA>];
  lds_u8* lds = (lds_u8*)smem;
  RowTile t;
  if (!take_row_tile<kRows<TA>>(g, parts, kSuper, t)) return;
  const int n = (t.n + 63) >> 6;
  if (n == 1) product_tile<TYPE, TA, 1>(g, t, x, w, y, lds);
  else if (TA == 2 || n == 2) product_tile<TYPE, TA, 2>(g, t, x, w, y, lds);
  else if (n == 3) product_tile<TYPE, TA, TA == 2 ? 2 : 3>(g, t, x, w, y, lds);
  else product_tile<TYPE, TA, TA>(g, t, x, w, y, lds);
}

template <int TYPE, int TA>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(TA == 4 ? 1 : 2, TA == 4 ? 1 : 2)))
void dx_kernel(Grouped g, const void* dy, const void* w, void* dx, int parts) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLds<TA>];
  lds_u8* lds = (lds_u8*)smem;
  RowTile t;
  if (!take_row_tile<kRows<TA>>(g, parts, kSuper, t)) return;
  const int n = (t.n + 63) >> 6;
  if (n == 1) dx_tile<TYPE, TA, 1>(g, t, dy, w, dx, lds);
  else if (TA == 2 || n == 2) dx_tile<TYPE, TA, 2>(g, t, dy, w, dx, lds);
  else if (n == 3) dx_tile<TYPE, TA, TA == 2 ? 2 : 3>(g, t, dy, w, dx, lds);
  else dx_tile<TYPE, TA, TA>(g, t, dy, w, dx, lds);
}

template <int TYPE, int TA>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(TA == 4 ? 1 : 2, TA == 4 ? 1 : 2)))
void dw_kernel(Grouped g, const void* dy, const void* x, float* dw, bool accumulate) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLds<TA>];
  lds_u8* lds = (lds_u8*)smem;
  constexpr int kM = kRows<TA>;
  const int na = (g.d_in + kM - 1) / kM, nb = (g.d_out + kM - 1) / kM;
  const int item = die_item(g.E * na * nb, blockIdx.x & 7, blockIdx.x >> 3);
  if (item < 0) return;
  const int expert = item / (na * nb), in = item - expert * (na * nb);
  // up to kSuper tiles of d_out alternate fastest
  const int sup = in / (kSuper * na), left = in - sup * (kSuper * na);
  const int width = min(kSuper, nb - sup * kSuper);
  const int ia = left / width, ib = sup * kSuper + left - ia * width;
  const Rows rows = expert_rows(g, expert);
  if (accumulate && rows.n == 0) return;
  const int a0 = ia * kM, b0 = ib * kM, n = min(kM, g.d_out - b0) >> 6;
  if (n == 1) dw_tile<TYPE, TA, 1>(g, rows, expert, a0, b0, dy, x, dw, accumulate, lds);
  else if (TA == 2 || n == 2) dw_tile<TYPE, TA, 2>(g, rows, expert, a0, b0, dy, x, dw, accumulate, lds);
  else if (n == 3) dw_tile<TYPE, TA, TA == 2 ? 2 : 3>(g, rows, expert, a0, b0, dy, x, dw, accumulate, lds);
  else dw_tile<TYPE, TA, TA>(g, rows, expert, a0, b0, dy, x, dw, accumulate, lds);
}

// Whether blocks of 256 columns and rows are enough to fill the chip.
bool large_blocks(const Grouped& g, int cols) {
  const int active = g.E < g.n ? g.E : g.n;
  const int tiles = g.n / 256 + active / 2;
  return (int64_t)(tiles > active ? tiles : active) * ((cols + 255) / 256) >= 256;
}

}  // namespace

hipError_t launch_grouped_product(const Grouped& g, const void* x, const void* w, void* y,
                                  hipStream_t s) {
  const bool large = large_blocks(g, g.d_out);
  const int m = large ? 256 : 128, parts = (g.d_out + m - 1) / m;
  const unsigned blocks = row_tile_blocks(g, m, parts);
  if (g.type == TYPE_F16) {
    if (large) product_kernel<F16, 4><<<blocks, kThreads, 0, s>>>(g, x, w, y, parts);
    else product_kernel<F16, 2><<<blocks, kThreads, 0, s>>>(g, x, w, y, parts);
  } else {
    if (large) product_kernel<BF16, 4><<<blocks, kThreads, 0, s>>>(g, x, w, y, parts);
    else product_kernel<BF16, 2><<<blocks, kThreads, 0, s>>>(g, x, w, y, parts);
  }
  return hipGetLastError();
}

hipError_t launch_grouped_dx(const Grouped& g, const void* dy, const void* w, void* dx,
                             hipStream_t s) {
  const bool large = large_blocks(g, g.d_in);
  const int m = large ? 256 : 128, parts = (g.d_in + m - 1) / m;
  const unsigned blocks = row_tile_blocks(g, m, parts);
  if (g.type == TYPE_F16) {
    if (large) dx_kernel<F16, 4><<<blocks, kThreads, 0, s>>>(g, dy, w, dx, parts);
    else dx_kernel<F16, 2><<<blocks, kThreads, 0, s>>>(g, dy, w, dx, parts);
  } else {
    if (large) dx_kernel<BF16, 4><<<blocks, kThreads, 0, s>>>(g, dy, w, dx, parts);
    else dx_kernel<BF16, 2><<<blocks, kThreads, 0, s>>>(g, dy, w, dx, parts);
  }
  return hipGetLastError();
}

hipError_t launch_grouped_dw(const Grouped& g, const void* dy, const void* x, float* dw,
                             bool accumulate, hipStream_t s) {
  auto tiles = [&](int m) { return (int64_t)g.E * ((g.d_in + m - 1) / m) * ((g.d_out + m - 1) / m); };
  const bool large = tiles(256) >= 256;
  const unsigned blocks = (unsigned)((tiles(large ? 256 : 128) + 7) / 8 + 1) * 8;
  if (g.type == TYPE_F16) {
    if (large) dw_kernel<F16, 4><<<blocks, kThreads, 0, s>>>(g, dy, x, dw, accumulate);
    else dw_kernel<F16, 2><<<blocks, kThreads, 0, s>>>(g, dy, x, dw, accumulate);
  } else {
    if (large) dw_kernel<BF16, 4><<<blocks, kThreads, 0, s>>>(g, dy, x, dw, accumulate);
    else dw_kernel<BF16, 2><<<blocks, kThreads, 0, s>>>(g, dy, x, dw, accumulate);
  }
  return hipGetLastError();
}

}  // namespace moe
