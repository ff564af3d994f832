// Grouped products of few rows per expert: the weights stream past them.
//
//   C[a, b] = sum_k W[a, k] x[b, k],  up to 16 rows b
//
// What bounds it is the weights' way from memory.  Every wave streams 16 rows of
// W through a ring of its own in LDS, by direct loads of whole 128-byte lines
// that pass the caches by (64 columns of 16 bits, 256 of MXFP4 a stage), and
// within a slab of columns waits for nothing but its own loads.  Read as matrix
// fragments straight from memory, 16 rows of 64 bytes at a time, a weight matrix
// of 235 MB took 40.4 us at best, in whole lines 35.6 (6.6 TB/s).
//
// The block's rows of x (and the weights' scales) are copied to LDS through
// registers once per slab while the first loads are under way; these are waited
// for with them, and at a slab's end the stream stops until the next one's copy
// is there.  A slab is 512 floor(20 / rows) columns where x has 16 bits (one row
// 10240, 11 to 16 rows 512: eight stages of W in 16 bits, two in MXFP4), 2048
// floor(20 / rows), or 2048, of x in MXFP4, and beside the scales of 64 rows of W
// 4096 at most.
//
// Of MXFP4, whose blocks have a quarter of the stages, that start is what bounds
// few columns: one row for two experts, 71 MB of 1024 columns 24.7 us, 62 MB of
// 4096 15.3, and 12.9 with x in MXFP4 too, which is without conversions.  With 64
// rows of W to a block, 80 KB of loads are in flight on a unit at once, here as in
// 16 bits (125 MB and 250 MB: 4.3 and 4.4 TB/s; 16 bits, 940 MB: 6.7).
//
//  The products are
// v_mfma_f32_16x16x32 (both operands in MXFP4: v_mfma_scale_f32_16x16x128): lane
// l holds 16 bytes of row l % 16, columns 8 (l / 16) and up of a step, and
// C[4 (l / 16) + i][l % 16].  Rows of x that the tile lacks repeat its last; what
// they give is not stored.
//
// A block is 4 waves: 64 rows of W, or, with SPLIT, 16 rows whose columns the
// waves share, for calls of few blocks; their sums are added in wave order.
#pragma once

#include "grouped.h"

namespace moe {
namespace few {

using namespace tile;

constexpr int kRowsMax = 16;
constexpr int kSlots = 6;                          // stages in a wave's ring
constexpr uint32_t kRing = kSlots * 2048;
// A row of x lies in pieces of 1024 bytes, 16 bytes apart so that the rows of a
// fragment cover the banks; rows of scales are 8 bytes apart.
constexpr int kPiece = 1024, kPieceStride = kPiece + 16, kScalePad = 8;
constexpr uint32_t kX = 4 * kRing, kXArea = 20 * kPieceStride;
constexpr uint32_t kWScale = kX + kXArea, kWScaleArea = 64 * (128 + kScalePad);
constexpr uint32_t kXScale = kWScale + kWScaleArea, kXScaleArea = 16 * (128 + kScalePad);
constexpr uint32_t kLdsFew = kXScale + kXScaleArea;  // two blocks per unit
static_assert(2 * kLdsFew <= 160 * 1024, "LDS");

template <int N>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}
__device__ inline void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

template <int TYPE>
__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (TYPE == F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// TYPE: that of y, and of x and W where they are not in MXFP4 (CODED: W,
// BOTH: x too).
template <int TYPE, bool CODED, bool BOTH, bool SPLIT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void few_kernel(Grouped g, const uint8_t* x, const uint8_t* xs, const uint8_t* w, const uint8_t* ws,
                void* y, int parts) {
  static_assert(CODED || !BOTH, "coded weights for coded rows");
  typedef typename Elem<TYPE>::T T;
  constexpr int kCols = CODED ? 256 : 64;           // columns of a stage
  constexpr int kXBits = BOTH ? 4 : 16;
  constexpr int kPieceCols = kPiece * 8 / kXBits;
  constexpr int kBlockRows = SPLIT ? 16 : 64;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kLdsFew];
  lds_u8* lds = (lds_u8*)smem;
  RowTiles<kRowsMax> tiles;
  RowTile t;
  tiles.init(g, parts);
  if (!tiles.get(blockIdx.x & 7, blockIdx.x >> 3, t)) return;

  const int l = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t ring = (uint32_t)(uintptr_t)lds + wave * kRing;
  const int K = g.d_in, c = t.n;
  const uint32_t row_bytes = CODED ? K / 2 : K * 2;
  const int64_t a0 = (int64_t)t.expert * g.d_out + t.part * kBlockRows;   // row of W
  const int64_t row0 = a0 + (SPLIT ? 0 : 16 * wave);
  const uint8_t* wbase = uniform(w + row0 * row_bytes);
  const int nst = (K + kCols - 1) / kCols;
  // the wave's stages: all, or a quarter of each slab's
  const uint32_t chunk = 16 * ((l & 7) ^ (l >> 4));  // of rows l / 8 (and 8 more: ^ 4)
  const uint32_t off0 = (uint32_t)(l >> 3) * row_bytes + chunk;
  const uint32_t off1 = (uint32_t)(8 + (l >> 3)) * row_bytes + (chunk ^ 64);
  auto load = [&](int k, uint32_t slot) {
    const uint8_t* at = wbase + (int64_t)k * 128;
    const uint32_t limit = k < nst ? kMasked - 1 : 0;
    const bool tail = CODED && K % 256 != 0;       // the last line is partial
    const uint32_t m0 = tail && 128 * k + chunk >= row_bytes ? kMasked : 0;
    const uint32_t m1 = tail && 128 * k + (chunk ^ 64) >= row_bytes ? kMasked : 0;
    load_lds<true>(ring + slot * 2048, at, limit, off0 | m0);
    load_lds<true>(ring + slot * 2048 + 1024, at, limit, off1 | m1);
  };

  // Slabs: whole pieces, as many columns as the areas hold.
  int slab = max(1, (int)(kXArea / kPieceStride) / c) * kPieceCols;
  if (CODED) slab = min(slab, (int)(kWScaleArea / kBlockRows - kScalePad) * 32 / kPieceCols * kPieceCols);
  if (BOTH) slab = min(slab, max(1, ((int)kXScaleArea / c - kScalePad) * 32 / kPieceCols) * kPieceCols);
  slab = min(slab, (nst * kCols + kPieceCols - 1) / kPieceCols * kPieceCols);
  const int ld_scales = slab / 32 + kScalePad;

  f32x4 acc[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
  const int tok = min(l & 15, c - 1), q = l >> 4;
  const uint32_t wrow = (l & 15) * 128, sw = (l >> 1) & 7;
  const uint32_t wscale = kWScale + ((SPLIT ? 0 : 16 * wave) + (l & 15)) * ld_scales;
  const uint32_t xscale = kXScale + tok * ld_scales;
  for (int s0 = 0; s0 < K; s0 += slab) {
    // stages of the slab, and the wave's among them
    const int first = s0 / kCols, all = min(nst, (s0 + slab) / kCols) - first;
    const int each = SPLIT ? (all + 3) / 4 : all;
    const int from = first + (SPLIT ? min(all, wave * each) : 0);
    const int n = SPLIT ? max(0, min(each, all - wave * each)) : all;
    auto stage = [&](int i, uint32_t slot) { load(i < n ? from + i : nst, slot); };
#pragma unroll
    for (int i = 0; i < kSlots - 1; ++i) stage(i, i);
    // the rows of x, zeros behind them (what is behind a row's codes is zero
    // too, but zero times NaN is not), and the scales
    {
      const int per = all * kCols * kXBits / 128;   // 16 bytes
      const int64_t bytes = (int64_t)K * kXBits / 8, at = (int64_t)s0 * kXBits / 8;
      for (int i = threadIdx.x; i < c * per; i += kThreads) {
        const int r = i / per, b = (i - r * per) * 16;
        u32x4 v = {0, 0, 0, 0};
        if (at + b < bytes) v = *reinterpret_cast<const u32x4*>(x + (t.row + r) * bytes + at + b);
        lds_write(lds, kX + ((b / kPiece) * c + r) * kPieceStride + b % kPiece, v);
      }
    }
    if constexpr (CODED) {
      const int bytes = K / 32;
      for (int i = threadIdx.x; i < kBlockRows * all; i += kThreads) {
        const int r = i / all, u = i - r * all;
        lds_write(lds, kWScale + r * ld_scales + 8 * u, scale_unit(ws + (a0 + r) * bytes, bytes, first + u));
      }
      if (BOTH)
        for (int i = threadIdx.x; i < c * all; i += kThreads) {
          const int r = i / all, u = i - r * all;
          lds_write(lds, kXScale + r * ld_scales + 8 * u,
                    scale_unit(xs + (int64_t)(t.row + r) * bytes, bytes, first + u));
        }
    }
    __syncthreads();
    uint32_t slot = 0;
    for (int i = 0; i < n; ++i) {
      wait_loads<2 * (kSlots - 2)>();
      const uint32_t at = wave * kRing + slot * 2048 + wrow;
      const int in = from + i - first, col = in * kCols;  // of the slab
      const uint32_t xat = kX + ((col / kPieceCols) * c + tok) * kPieceStride + (col % kPieceCols) * kXBits / 8;
      u32x4 a[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) a[s] = lds_read<u32x4>(lds, at + 16 * ((4 * s + q) ^ sw));
      if constexpr (!CODED) {
        u32x4 b[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) b[s] = lds_read<u32x4>(lds, xat + 64 * s + 16 * q);
        wait_reads();
        stage(i + kSlots - 1, slot == 0 ? kSlots - 1 : slot - 1);
#pragma unroll
        for (int s = 0; s < 2; ++s) acc[s] = mfma16<TYPE>(a[s], b[s], acc[s]);
      } else {
        const u32x2 sw8 = lds_read<u32x2>(lds, wscale + 8 * in);
        if constexpr (BOTH) {
          const u32x2 sx8 = lds_read<u32x2>(lds, xscale + 8 * in);
          u32x4 b[2];
#pragma unroll
          for (int s = 0; s < 2; ++s) b[s] = lds_read<u32x4>(lds, xat + 64 * s + 16 * q);
          wait_reads();
          stage(i + kSlots - 1, slot == 0 ? kSlots - 1 : slot - 1);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const i32x8 u = {(int)a[s].x, (int)a[s].y, (int)a[s].z, (int)a[s].w, 0, 0, 0, 0};
            const i32x8 v = {(int)b[s].x, (int)b[s].y, (int)b[s].z, (int)b[s].w, 0, 0, 0, 0};
            const uint32_t sa = sw8[s], sb = sx8[s];
            acc[s] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v, acc[s], 4, 4, 0, (int)(sa >> (8 * q)), 0,
                                                                       (int)(sb >> (8 * q)));
          }
        } else {
          u32x4 b[8];
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) b[4 * s + j] = lds_read<u32x4>(lds, xat + 256 * s + 64 * q + 16 * j);
          wait_reads();
          stage(i + kSlots - 1, slot == 0 ? kSlots - 1 : slot - 1);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const uint32_t both = sw8[s];
            const float scale = scale_of((both >> (8 * q)) & 255);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j & 1] = mfma16<TYPE>(decode<TYPE>(a[s][j], scale), b[4 * s + j], acc[j & 1]);
          }
        }
      }
      slot = slot + 1 == kSlots ? 0 : slot + 1;
    }
    wait_loads<0>();
    __syncthreads();
  }
  acc[0] += acc[1];
  if constexpr (SPLIT) {
    lds_write(lds, threadIdx.x * 16, acc[0]);
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < 4; ++i) acc[0] += lds_read<f32x4>(lds, i * 1024 + l * 16);
  }
  if ((l & 15) < c) {
    typedef T x4 __attribute__((ext_vector_type(4)));
    const x4 v = {(T)acc[0].x, (T)acc[0].y, (T)acc[0].z, (T)acc[0].w};
    T* to = static_cast<T*>(y) + (int64_t)(t.row + (l & 15)) * g.d_out + t.part * kBlockRows +
            (SPLIT ? 0 : 16 * wave) + 4 * q;
    *reinterpret_cast<x4*>(to) = v;
  }
}

// Whether a call goes this way: up to 8 rows per expert on average.  Us here / on
// tiles of 64 rows and more, 16 experts of 6400 x 4096: 2 rows each 115 / 128, 8
// rows 153 / 169, 16 rows 195 / 168; W in MXFP4 48 / 73, 75 / 85, 118 / 86; x in
// MXFP4 too, 8 rows 54 / 67, 16 rows 71 / 61.
//
// Codes in calls of few tiles, whose blocks there wait for one stage after
// another, up to 16 rows, 24 if x's are in MXFP4 too.  One expert of 4096 x
// 4096: 16 rows 19 / 26, 32 rows 23 / 28, 64 rows 43 / 28, of 14336 x 4096 24 /
// 28, 28 / 28, 53 / 28; x too 16 rows 14 / 21 and 15 / 23, 32 rows 14 / 22 and
// 18 / 23, 64 rows 14 / 22 and 29 / 23; 8 experts of 2048 x 4096, 32 rows each
// 28 / 24.  In 16 bits 8 rows 15 / 21 and 26 / 25, 16 rows 19 / 21 and 31 / 24.
//
// The counts are on the device, so the rule goes by the average over all experts.
// Counts that leave most of them empty send the others this way with many rows
// each, and W streams once per 16 of them: 64 experts of 4096 x 4096, two of which
// have 256 rows each, 512 rows / 520 (which go by tiles): fp16 142 / 42, W in MXFP4
// 118 / 46, x too 55 / 35; of 1472 x 2048 35 / 23, 29 / 21, 13 / 21.  Evenly
// spread, the same calls take 327 / 361, 161 / 168, 115 / 110 and 73 / 76, 35 / 38,
// 26 / 29.
inline bool takes(const Grouped& g, bool coded, bool both) {
  const int rows = !coded || !narrow_blocks(g, g.d_out) ? 8 : both ? 24 : 16;
  return g.n <= rows * (int64_t)g.E;
}

// Whether the waves of a block share its columns: for calls of few blocks, and
// where both operands are in MXFP4 only if the rows are long, as a stage takes
// 256 of their columns at once.  Us with / without, one row for each of 2
// experts: 4096 x 4096 12.9 / 15.8, 6400 x 4096 21.7 / 20.0, 6400 x 1024 10.2 /
// 7.3, 4096 x 16384 44 / 55; W in MXFP4, 4096 x 4096 7.9 / 9.5, 5120 x 4096 11.6
// / 9.6, 4096 x 16384 18 / 29; x too (quantised before: 5), 2048 x 4096 13.2 /
// 12.2, 2048 x 16384 12.9 / 26.3.
inline bool splits(const Grouped& g, bool both) {
  const int active = g.E < g.n ? g.E : g.n;
  return (int64_t)active * (g.d_out / 64) < 160 && (!both || g.d_in >= 8192);
}

template <int TYPE, bool CODED, bool BOTH>
void launch(const Grouped& g, const void* x, const void* xs, const void* w, const void* ws, void* y,
            hipStream_t s) {
  const uint8_t *xb = static_cast<const uint8_t*>(x), *sb = static_cast<const uint8_t*>(xs);
  const uint8_t *wb = static_cast<const uint8_t*>(w), *tb = static_cast<const uint8_t*>(ws);
  const bool split = splits(g, BOTH);
  const int parts = g.d_out / (split ? 16 : 64);
  const unsigned blocks = row_tile_blocks(g, kRowsMax, parts);
  if (split) few_kernel<TYPE, CODED, BOTH, true><<<blocks, kThreads, 0, s>>>(g, xb, sb, wb, tb, y, parts);
  else few_kernel<TYPE, CODED, BOTH, false><<<blocks, kThreads, 0, s>>>(g, xb, sb, wb, tb, y, parts);
}

}  // namespace few
}  // namespace moe
