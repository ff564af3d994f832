// Matrix products grouped by expert, forward and backward.
//
//   y[r]   = W[e(r)] x[r]                 r over the rows of expert e(r)
//   d_x[r] = W[e(r)]^T d_y[r]
//   d_W[e] = sum over the rows r of e of d_y[r] x[r]^T
//
// All three on the tiles of tile.h, calls of few rows on few_rows.h.  A is the
// operand whose index is contiguous in y and d_x, so that a lane stores 16 bytes
// of a row; for d_W, whose fp32 values go out one by one, the other one (roles
// swapped, and not past the caches, both gradients of the 8192 rows below took 12 %
// longer).
//
// d_W is 4 bytes per 2 rows' products: few rows per expert bound it by its own
// writing.  Added to what is there (ADD) it reads as much: a lane fetches the 16
// values of a tile of 32 x 32 together, since none may pass a store to the same
// array; one at a time 16 experts of 6400 x 4096, 8192 rows, took 3183 us where it
// takes 764 (681 at a copy's rate), 60 of 1472 x 2048, 5348 rows, 1341 where it
// takes 276.  A kernel that can only write takes 531, one that can do both 553.
// Kernels in us (what bounds them):
//   16 experts of 6400 x 4096, fp16: y of 16384 rows 774 to 863 (power: 1.0 to 1.1
//     PF), d_x of 8192 rows 452 to 476 (640 tiles, some hardly filled, in three
//     rounds of 256; 512 rows for every expert, 512 full tiles, 374: 1.15 PF; the
//     forward product of the same sizes takes 374 and 472 on the same two counts),
//     d_W 552 to 579 (tiles of eight stages, whose stores nothing runs beside:
//     0.77 PF, 3.2 TB/s)
//   60 experts of 1472 x 2048, bf16, 5348 rows: y 98 to 105 (W's way from memory,
//     4.1 TB/s), d_x 79 to 86 (5.1 TB/s), d_W 134 to 146 (5.4 TB/s written)
#include "few_rows.h"

namespace moe {

namespace {

using namespace tile;

// Rows of 16 bits: forward (A = W, whose rows are the columns of y) and, with
// BACK, the gradient of x (A = W^T, the reduction over W's rows).
template <int TYPE, int TA, int TB, bool BACK>
struct RowJob {
  typedef RowTile Tile;
  typedef typename Elem<TYPE>::T T;
  const Grouped& g;
  const T *in, *w;
  T* out;
  Items<TA>& items;

  __device__ inline int n_in() const { return BACK ? g.d_out : g.d_in; }
  __device__ inline int n_out() const { return BACK ? g.d_in : g.d_out; }
  __device__ inline bool next(Tile& t) { return items.next(TB, t); }
  __device__ inline int steps(const Tile&) const { return n_in(); }
  __device__ inline Operand a(const Tile& t) const {
    const int col = t.part * 64 * TA;
    const T* at = w + (int64_t)t.expert * g.d_out * g.d_in + (BACK ? col : (int64_t)col * g.d_in);
    return {(const uint8_t*)at, (uint32_t)(2 * g.d_in), n_out() - col};
  }
  __device__ inline Operand b(const Tile& t) const {
    return {(const uint8_t*)(in + (int64_t)t.row * n_in()), (uint32_t)(2 * n_in()), t.n};
  }
  __device__ inline void store(const Tile& t, Acc<TA, TB>& acc) const {
    const int col = t.part * 64 * TA;
    store_rows<T, Waves<BACK ? COLS : ROWS, TA>, TA, TB>(acc, out + (int64_t)t.row * n_out() + col, n_out(), t.n, n_out() - col);
  }
};

template <int TYPE, int TA, bool BACK>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(TA == 4 ? 1 : 2, TA == 4 ? 1 : 2)))
void rows_kernel(Grouped g, const void* in, const void* w, void* out, int parts) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLds<TA>];
  typedef typename Elem<TYPE>::T T;
  constexpr int KA = BACK ? COLS : ROWS;
  lds_u8* lds = (lds_u8*)smem;
  Items<TA> items;
  items.init(g, parts);
  set_aside(in);
  set_aside(w);
  set_aside(out);
  auto take = [&](auto size) {
    constexpr int TB = decltype(size)::value;
    RowJob<TYPE, TA, TB, BACK> job = {g, (const T*)in, (const T*)w, (T*)out, items};
    stream<TYPE, KA, ROWS, TA, TB, kLds<TA>>(job, lds);
  };
  while (const int n = items.size()) {
    if (n == 1) take(std::integral_constant<int, 1>());
    else if (n == 2) take(std::integral_constant<int, 2>());
    else if (TA == 4 && n == 3) take(std::integral_constant<int, TA == 4 ? 3 : 1>());
    else if (TA == 4) take(std::integral_constant<int, TA == 4 ? 4 : 1>());
  }
}

// The gradient of W: A from d_y (rows of d_W), B from x, the reduction over the
// expert's rows.
struct WeightTile {
  int expert, first, n, a0, b0;
};

template <int TA, bool ADD>
struct WeightItems {
  const Grouped& g;
  Counts counts;
  int slot;
  WeightTile t;        // the first one not taken; n < 0: none

  __device__ inline void init() {
    counts.init(g);
    set_aside(counts.per);
    slot = (int)(blockIdx.x >> 3) - kBlocks<TA> / 8;
    set_aside(slot);
    step();
  }
  __device__ inline void step() {
    constexpr int kSuper = 8;  // tiles of d_in that alternate fastest
    const int na = (g.d_out + kRows<TA> - 1) / kRows<TA>, nb = (g.d_in + kRows<TA> - 1) / kRows<TA>;
    const int per = na * nb, n = g.E * per;
    Counts now = counts;
    now.per = __builtin_amdgcn_readfirstlane(counts.per);
    int at = __builtin_amdgcn_readfirstlane(slot);
    WeightTile x = {0, 0, -1, 0, 0};
    while (x.n < 0 && (at += kBlocks<TA> / 8) < die_slots(n)) {
      const int item = die_item(n, blockIdx.x & 7, at);
      if (item < 0) continue;
      const int e = item / per, in = item - e * per;
      const Rows rows = now.rows(e);
      if (ADD && rows.n == 0) continue;
      const int sup = in / (kSuper * na), left = in - sup * (kSuper * na);
      const int width = min(kSuper, nb - sup * kSuper);
      const int ia = left / width, ib = sup * kSuper + left - ia * width;
      x = {e, rows.first, rows.n, ia * kRows<TA>, ib * kRows<TA>};
    }
    t = x;
    slot = at;
    set_aside(slot);
    set_aside(t.expert);
    set_aside(t.first);
    set_aside(t.n);
    set_aside(t.a0);
    set_aside(t.b0);
  }
  // 64s of columns of the tile (0: no tile)
  __device__ inline int size() const {
    const int n = __builtin_amdgcn_readfirstlane(t.n);
    return n < 0 ? 0 : min(kRows<TA>, g.d_in - __builtin_amdgcn_readfirstlane(t.b0)) >> 6;
  }
  __device__ inline bool next(int tb, WeightTile& x) {
    if (size() != tb) return false;
    x = {__builtin_amdgcn_readfirstlane(t.expert), __builtin_amdgcn_readfirstlane(t.first),
         __builtin_amdgcn_readfirstlane(t.n), __builtin_amdgcn_readfirstlane(t.a0),
         __builtin_amdgcn_readfirstlane(t.b0)};
    step();
    return true;
  }
};

template <int TYPE, int TA, int TB, bool ADD>
struct WeightJob {
  typedef WeightTile Tile;
  typedef typename Elem<TYPE>::T T;
  const Grouped& g;
  const T *dy, *x;
  float* dw;
  WeightItems<TA, ADD>& items;

  __device__ inline bool next(Tile& t) { return items.next(TB, t); }
  __device__ inline int steps(const Tile& t) const { return t.n; }
  __device__ inline Operand a(const Tile& t) const {
    return {(const uint8_t*)(dy + (int64_t)t.first * g.d_out + t.a0), (uint32_t)(2 * g.d_out), g.d_out - t.a0};
  }
  __device__ inline Operand b(const Tile& t) const {
    return {(const uint8_t*)(x + (int64_t)t.first * g.d_in + t.b0), (uint32_t)(2 * g.d_in), g.d_in - t.b0};
  }
  // The lanes lie along d_W's rows: each store writes two whole lines, past the
  // caches (nothing here reads them again).
  __device__ inline void store(const Tile& t, Acc<TA, TB>& acc) const {
    const int l = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int aw = (wave >> 1) * TA * 32, bw = (wave & 1) * TB * 32;
    float* out = dw + ((int64_t)t.expert * g.d_out + t.a0 + aw + 4 * (l >> 5)) * g.d_in + t.b0 + bw + (l & 31);
#pragma unroll
    for (int i = 0; i < TA; ++i) {
      if (t.a0 + aw + 32 * i >= g.d_out) continue;
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        if (t.b0 + bw + 32 * j >= g.d_in) continue;
        keep<TA * TB>(acc[i][j]);
        auto to = [&](int q) {
          return global_ptr<float>(out + (int64_t)(32 * i + 8 * (q >> 2) + (q & 3)) * g.d_in + 32 * j);
        };
        float v[16];
        if constexpr (ADD) {
          // (all of them before the first store, which they may not pass)
#pragma unroll
          for (int q = 0; q < 16; ++q) v[q] = __builtin_nontemporal_load(to(q));
        }
#pragma unroll
        for (int q = 0; q < 16; ++q) v[q] = ADD ? v[q] + acc[i][j][q] : acc[i][j][q];
#pragma unroll
        for (int q = 0; q < 16; ++q) __builtin_nontemporal_store(v[q], to(q));
      }
    }
  }
};

template <int TYPE, int TA, bool ADD>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(TA == 4 ? 1 : 2, TA == 4 ? 1 : 2)))
void dw_kernel(Grouped g, const void* dy, const void* x, float* dw) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLds<TA>];
  typedef typename Elem<TYPE>::T T;
  lds_u8* lds = (lds_u8*)smem;
  WeightItems<TA, ADD> items = {g};
  items.init();
  set_aside(dy);
  set_aside(x);
  set_aside(dw);
  auto take = [&](auto size) {
    constexpr int TB = decltype(size)::value;
    WeightJob<TYPE, TA, TB, ADD> job = {g, (const T*)dy, (const T*)x, dw, items};
    stream<TYPE, COLS, COLS, TA, TB, kLds<TA>>(job, lds);
  };
  while (const int n = items.size()) {
    if (n == 1) take(std::integral_constant<int, 1>());
    else if (n == 2) take(std::integral_constant<int, 2>());
    else if (TA == 4 && n == 3) take(std::integral_constant<int, TA == 4 ? 3 : 1>());
    else if (TA == 4) take(std::integral_constant<int, TA == 4 ? 4 : 1>());
  }
}

template <int TYPE, bool BACK>
void launch_rows(const Grouped& g, const void* in, const void* w, void* out, hipStream_t s) {
  const int cols = BACK ? g.d_in : g.d_out;
  if (narrow_blocks(g, cols))
    rows_kernel<TYPE, 1, BACK><<<kBlocks<1>, kThreads, 0, s>>>(g, in, w, out, cols / 64);
  else if (large_blocks(g, cols, BACK ? 0 : 64))
    rows_kernel<TYPE, 4, BACK><<<kBlocks<4>, kThreads, 0, s>>>(g, in, w, out, (cols + 255) / 256);
  else
    rows_kernel<TYPE, 2, BACK><<<kBlocks<2>, kThreads, 0, s>>>(g, in, w, out, (cols + 127) / 128);
}

// Blocks of 256 x 256 where they fill the chip.  Us with them / with 128 x 128,
// and added to what is there: 16 experts of 6400 x 4096, 8192 rows, 534 / 714, 760
// / 849; 60 of 1472 x 2048, 5348 rows, 136 / 130, 277 / 285; one of 4096 x 4096,
// 4096 rows (256 tiles) 119 / 143, 131 / 150; 16 of 1024 x 1024, 2048 rows (256)
// 18 / 17, 31 / 33; 64 tiles (2048 x 2048) 77 / 46, 87 / 49; 128 tiles (8 of 1024 x
// 1024, 2048 rows) 15 / 12, 27 / 20.
template <int TYPE, bool ADD>
void launch_dw(const Grouped& g, const void* dy, const void* x, float* dw, hipStream_t s) {
  if ((int64_t)g.E * ((g.d_in + 255) / 256) * ((g.d_out + 255) / 256) >= 256)
    dw_kernel<TYPE, 4, ADD><<<kBlocks<4>, kThreads, 0, s>>>(g, dy, x, dw);
  else
    dw_kernel<TYPE, 2, ADD><<<kBlocks<2>, kThreads, 0, s>>>(g, dy, x, dw);
}

}  // namespace

hipError_t launch_grouped_product(const Grouped& g, const void* x, const void* w, void* y,
                                  hipStream_t s) {
  if (few::takes(g, false, false)) {
    if (g.type == TYPE_F16) few::launch<F16, false, false>(g, x, nullptr, w, nullptr, y, s);
    else few::launch<BF16, false, false>(g, x, nullptr, w, nullptr, y, s);
  } else {
    if (g.type == TYPE_F16) launch_rows<F16, false>(g, x, w, y, s);
    else launch_rows<BF16, false>(g, x, w, y, s);
  }
  return hipGetLastError();
}

hipError_t launch_grouped_dx(const Grouped& g, const void* dy, const void* w, void* dx,
                             hipStream_t s) {
  if (g.type == TYPE_F16) launch_rows<F16, true>(g, dy, w, dx, s);
  else launch_rows<BF16, true>(g, dy, w, dx, s);
  return hipGetLastError();
}

hipError_t launch_grouped_dw(const Grouped& g, const void* dy, const void* x, float* dw,
                             bool accumulate, hipStream_t s) {
  if (g.type == TYPE_F16) {
    if (accumulate) launch_dw<F16, true>(g, dy, x, dw, s);
    else launch_dw<F16, false>(g, dy, x, dw, s);
  } else {
    if (accumulate) launch_dw<BF16, true>(g, dy, x, dw, s);
    else launch_dw<BF16, false>(g, dy, x, dw, s);
  }
  return hipGetLastError();
}

}  // namespace moe
