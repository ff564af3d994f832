// Products grouped by expert with weights in MXFP4, and activations of 16 bits
// or in MXFP4 too, on the tiles of tile.h.
//
// With both in MXFP4 the matrix cores take codes and scales as they are.
// With activations of 16 bits a code becomes an activation's type after it was
// read from LDS (v_cvt_scalef32_pk: exact wherever the type holds the value),
// eight for four of these instructions.
//
// Kernels in us, 16 experts of 6400 x 4096: 1024 bf16 rows 113 to 120 (244 MB and
// 54 GF; a stage's chain of reads, conversions and products bounds it, the
// products are a third of the time), 16384 fp16 rows 743 (power), 8192 rows in
// MXFP4 158 to 177 (tile.h).  On few_rows.h one row for two experts of 14336 x
// 4096, 62 MB: 13.7 to 14.1 (4.5 TB/s; what bounds it there).
#include "few_rows.h"

namespace moe {

namespace {

using namespace tile;

template <int TYPE, int TA, int TB, bool CODED>
struct MxJob {
  typedef RowTile Tile;
  typedef typename Elem<TYPE>::T T;
  const Grouped& g;
  const uint8_t *x, *xs, *w, *ws;
  T* y;
  Items<TA>& items;

  __device__ inline bool next(Tile& t) { return items.next(TB, t); }
  __device__ inline int steps(const Tile&) const { return g.d_in; }
  __device__ inline int64_t column(const Tile& t) const { return (int64_t)t.expert * g.d_out + t.part * 64 * TA; }
  __device__ inline Operand a(const Tile& t) const {
    return {w + column(t) * (g.d_in / 2), (uint32_t)(g.d_in / 2), g.d_out - t.part * 64 * TA};
  }
  __device__ inline Operand b(const Tile& t) const {
    const int bytes = CODED ? g.d_in / 2 : g.d_in * 2;
    return {x + (int64_t)t.row * bytes, (uint32_t)bytes, t.n};
  }
  __device__ inline Scales a_scales(const Tile& t) const { return {ws + column(t) * (g.d_in / 32), g.d_in / 32}; }
  __device__ inline Scales b_scales(const Tile& t) const { return {xs + (int64_t)t.row * (g.d_in / 32), g.d_in / 32}; }
  template <int NA, int NB>
  __device__ inline void store(const Tile& t, Acc<NA, NB>& acc) const {
    const int col = t.part * 64 * TA;
    store_rows<T, Waves<CODED ? ROWS : CODES, TA>, NA, NB>(acc, y + (int64_t)t.row * g.d_out + col, g.d_out, t.n, g.d_out - col);
  }
};

template <int TYPE, int TA, bool CODED>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(TA == 4 ? 1 : 2, TA == 4 ? 1 : 2)))
void mx_kernel(Grouped g, const uint8_t* x, const uint8_t* xs, const uint8_t* w, const uint8_t* ws,
               void* y, int parts) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLds<TA>];
  lds_u8* lds = (lds_u8*)smem;
  Items<TA> items;
  items.init(g, parts);
  set_aside(x);
  set_aside(xs);
  set_aside(w);
  set_aside(ws);
  set_aside(y);
  auto take = [&](auto size) {
    constexpr int TB = decltype(size)::value;
    MxJob<TYPE, TA, TB, CODED> job = {g, x, xs, w, ws, (typename Elem<TYPE>::T*)y, items};
    stream<CODED ? F4 : TYPE, CODED ? ROWS : CODES, ROWS, TA, TB, kLds<TA>>(job, lds);
  };
  while (const int n = items.size()) {
    if (n == 1) take(std::integral_constant<int, 1>());
    else if (n == 2) take(std::integral_constant<int, 2>());
    else if (TA == 4 && n == 3) take(std::integral_constant<int, TA == 4 ? 3 : 1>());
    else if (TA == 4) take(std::integral_constant<int, TA == 4 ? 4 : 1>());
  }
}

template <int TYPE, bool CODED>
void launch(const Grouped& g, const uint8_t* x, const uint8_t* xs, const uint8_t* w, const uint8_t* ws,
            void* y, hipStream_t s) {
  if (narrow_blocks(g, g.d_out))
    mx_kernel<TYPE, 1, CODED><<<kBlocks<1>, kThreads, 0, s>>>(g, x, xs, w, ws, y, g.d_out / 64);
  else if (large_blocks(g, g.d_out, CODED ? 0 : 384))
    mx_kernel<TYPE, 4, CODED><<<kBlocks<4>, kThreads, 0, s>>>(g, x, xs, w, ws, y, (g.d_out + 255) / 256);
  else
    mx_kernel<TYPE, 2, CODED><<<kBlocks<2>, kThreads, 0, s>>>(g, x, xs, w, ws, y, (g.d_out + 127) / 128);
}

}  // namespace

hipError_t launch_mx_product(const Grouped& g, const void* x, const uint8_t* xs,
                             const uint8_t* w, const uint8_t* ws, void* y, hipStream_t s) {
  const uint8_t* xb = static_cast<const uint8_t*>(x);
  if (few::takes(g, true, xs != nullptr)) {
    if (g.type == TYPE_F16) {
      if (xs) few::launch<F16, true, true>(g, x, xs, w, ws, y, s);
      else few::launch<F16, true, false>(g, x, xs, w, ws, y, s);
    } else {
      if (xs) few::launch<BF16, true, true>(g, x, xs, w, ws, y, s);
      else few::launch<BF16, true, false>(g, x, xs, w, ws, y, s);
    }
  } else if (g.type == TYPE_F16) {
    if (xs) launch<F16, true>(g, xb, xs, w, ws, y, s);
    else launch<F16, false>(g, xb, xs, w, ws, y, s);
  } else {
    if (xs) launch<BF16, true>(g, xb, xs, w, ws, y, s);
    else launch<BF16, false>(g, xb, xs, w, ws, y, s);
  }
  return hipGetLastError();
}

}  // namespace moe
