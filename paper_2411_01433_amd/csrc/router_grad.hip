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
// and then  d_x = dl Wg,  d_Wg = dl^T x,  two matrix products on the matrix
// cores.  Their fp32 operand dl is split into numbers of 16 bits whose
// products are added in fp32: for fp16 two of them (22 bits), scaled by a
// power of two per group of 64 tokens so that the group's largest lies below
// 2^15; for bf16, which has the range, three (24 bits) for d_Wg and the first
// two (16 bits) for d_x, whose own 8 bits are far above.
#include "moe_internal.h"

namespace moe {

namespace {

typedef f16 f16x8v __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T16> struct Split;
template <> struct Split<f16> {
  typedef f16x8v x8;
  static constexpr int kX = 2, kW = 2;  // parts of dl for d_x and d_Wg
};
template <> struct Split<bf16> {
  typedef bf16x8 x8;
  static constexpr int kX = 2, kW = 3;
};

__device__ inline f32x4 mfma(f16x8v a, f16x8v b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <class T>
__device__ inline const __attribute__((address_space(1))) T* global(const void* p) {
  return (const __attribute__((address_space(1))) T*)(const T*)p;
}

__device__ inline bool finite(float v) { return fabsf(v) <= 3.402823466e38f; }

__device__ inline float wave_max_f(float v) {
  for (int m = 1; m < 64; m <<= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
  return v;
}

// Fragments.  A product of 32 terms takes 8 numbers from each of 64 lanes:
// lane l has row (or column) l & 15 and the terms 4 g .. 4 g + 3 and 16 + 4 g
// .. 16 + 4 g + 3 of its group g = l >> 4, which is what two transposing reads
// of LDS give.  dl is written in this order, 1 KiB per fragment, so that a
// fragment is one contiguous load:
//   for d_x   [T/16][E/32][part][64 lanes][8]: rows tokens, terms experts
//   for d_Wg  [T/32][E/16][part][64 lanes][8]: rows experts, terms tokens
// T and E rounded up to 64 and 32, with zeros.
__device__ inline int term(int g, int j) { return j < 4 ? 4 * g + j : 12 + 4 * g + j; }

constexpr int kGroupTokens = 64;   // tokens with one scale

// Part `part` of v: what is left of it after the parts before, in 16 bits.
template <class T16>
__device__ inline T16 next_part(float& left) {
  const T16 h = (T16)left;
  left -= (float)h;
  return h;
}

// Gradient of the logits of 64 tokens, and its fragments.  A wave per token in
// turn: lane k has slot k, lane i the experts i, i + 64, ...
constexpr int kLogitThreads = 1024;
template <class T16, int C>
__global__ __launch_bounds__(kLogitThreads) void router_dlogits_kernel(
    RouterParams p, int T, const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const float* __restrict__ dw, const float* __restrict__ dl, T16* __restrict__ fx,
    T16* __restrict__ fw, float* __restrict__ scales) {
  typedef typename Split<T16>::x8 x8;
  constexpr int LD = C * 64 + 4;
  __shared__ float rows[kGroupTokens][LD];
  __shared__ float tops[kLogitThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int Ep = (p.E + 31) & ~31;
  const bool sig = p.score == SCORE_SIGMOID, full = !p.renorm && !sig;
  const float none = -__builtin_inff();
  float most = 0.0f;
  for (int i = wave; i < kGroupTokens; i += kLogitThreads / 64) {
    const int t = blockIdx.x * kGroupTokens + i;
    float row[C];
    int e = -1;
    float slot = 0.0f, mean = 0.0f, all = 1.0f;
    if (t < T) {
      const float* lr = logits + (int64_t)t * p.E;
      float g = 0.0f, l = none;
      if (lane < p.K) {
        e = idx[(int64_t)t * p.K + lane];
        if (e >= 0 && e < p.E) l = lr[e];
        if (finite(l)) g = p.scale * dw[(int64_t)t * p.K + lane];
        else e = -1;
      }
      const bool have = e >= 0;
      // z = exp(-|l|): s and 1 - s without loss on either side
      const float z = expf(-fabsf(l));
      const float not_s = have ? (l >= 0.0f ? z : 1.0f) / (1.0f + z) : 0.0f;
      const float s = have ? (l >= 0.0f ? 1.0f : z) / (1.0f + z) : 0.0f;
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
        all = 0.0f;
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
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int ee = c * 64 + lane;
      float v = t < T && full && row[c] > 0.0f ? -mean * (row[c] / all) : 0.0f;
      for (int k = 0; k < p.K; ++k) {
        const int ek = __builtin_amdgcn_readlane(e, k);
        const float gk = __builtin_bit_cast(
            float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, slot), k));
        if (ek == ee) v += gk;
      }
      if (dl && t < T && ee < p.E) v += dl[(int64_t)t * p.E + ee];
      if (finite(v)) most = fmaxf(most, fabsf(v));
      rows[i][ee] = v;
    }
  }
  most = wave_max_f(most);
  if (lane == 0) tops[wave] = most;
  __syncthreads();
  float scale = 1.0f;
  if constexpr (sizeof(T16) == 2 && Split<T16>::kW == 2) {
    float top = 0.0f;
#pragma unroll
    for (int w = 0; w < kLogitThreads / 64; ++w) top = fmaxf(top, tops[w]);
    if (top > 0.0f) scale = ldexpf(1.0f, min(max(14 - ilogbf(top), -113), 110));
  }
  if (threadIdx.x == 0) scales[blockIdx.x] = 1.0f / scale;
  const int m = lane & 15, g = lane >> 4;
  const int EB = Ep / 32, ET = Ep / 16;
  if (fx)
    for (int q = wave; q < 4 * EB; q += kLogitThreads / 64) {
      const int tt = q / EB, eb = q - tt * EB;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rows[tt * 16 + m][eb * 32 + term(g, j)] * scale;
      T16* to = fx + (((int64_t)(blockIdx.x * 4 + tt) * EB + eb) * Split<T16>::kX * 64 + lane) * 8;
#pragma unroll
      for (int part = 0; part < Split<T16>::kX; ++part) {
        x8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = next_part<T16>(v[j]);
        *reinterpret_cast<x8*>(to + part * 512) = o;
      }
    }
  if (fw)
    for (int q = wave; q < 2 * ET; q += kLogitThreads / 64) {
      const int tb = q / ET, et = q - tb * ET;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rows[tb * 32 + term(g, j)][et * 16 + m] * scale;
      T16* to = fw + (((int64_t)(blockIdx.x * 2 + tb) * ET + et) * Split<T16>::kW * 64 + lane) * 8;
#pragma unroll
      for (int part = 0; part < Split<T16>::kW; ++part) {
        x8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = next_part<T16>(v[j]);
        *reinterpret_cast<x8*>(to + part * 512) = o;
      }
    }
}

constexpr int kCols = 128;   // columns of d per block of the products

// LDS tile of 16-bit rows of kCols columns, 256 bytes each: 64-byte block b of
// a row r lies at block b ^ (r & 3), so that the four rows that 16 lanes of a
// transposing read touch lie in different banks.
__device__ inline int tile_at(int row, int byte) { return row * 256 + (byte ^ ((row & 3) << 6)); }

typedef __attribute__((address_space(3))) s16x4* LdsRead;

// 8 terms for one of 16 columns per lane from rows `row` + term(g, .) of a
// tile; lanes q = l & 3 read the columns at byte col(q) (8 bytes each), and
// lane l gets column l & 3 of the ones that q = (l & 15) >> 2 points at.
template <class T16>
__device__ inline typename Split<T16>::x8 read_columns(const unsigned char* tile, int row, int byte) {
  const int lane = threadIdx.x & 63;
  const int r = row + 4 * (lane >> 4) + ((lane & 15) >> 2);
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRead)(tile + tile_at(r, byte)));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRead)(tile + tile_at(r + 16, byte)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return __builtin_bit_cast(typename Split<T16>::x8, v);
}

// d_x of kCols columns: the block keeps Wg's columns in LDS (EB * 32 rows) and
// its waves take 32 tokens each in turn.  A wave's fragment of dl is loaded
// once and multiplied with 128 columns.  Rows of the result are columns of
// d, ordered so that a lane has 8 neighbouring ones of a token: tile 2 s + h,
// row 4 q + r is column 32 s + 8 q + 4 h + r.
constexpr int kDxThreads = 256;
template <class T16, int EB>
__global__ __launch_bounds__(kDxThreads) void router_dx_kernel(RouterParams p, int T,
                                                               const T16* __restrict__ fx,
                                                               const float* __restrict__ scales,
                                                               T16* __restrict__ dx) {
  typedef typename Split<T16>::x8 x8;
  constexpr int kX = Split<T16>::kX;
  __shared__ __attribute__((aligned(16))) unsigned char tile[EB * 32 * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * kCols, eb_n = (p.E + 31) / 32;
  for (int v = threadIdx.x; v < eb_n * 32 * 16; v += kDxThreads) {
    const int e = v >> 4, c = v & 15;
    u32x4 w = {0, 0, 0, 0};
    if (e < p.E && n0 + c * 8 < p.d)
      w = *global<u32x4>(static_cast<const T16*>(p.wg) + (int64_t)e * p.d + n0 + c * 8);
    *reinterpret_cast<u32x4*>(tile + tile_at(e, c * 16)) = w;
  }
  __syncthreads();
  const int q = lane & 3, g = lane >> 4;
  for (int w32 = blockIdx.y * 4 + wave; w32 * 32 < T; w32 += gridDim.y * 4) {
    f32x4 acc[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    const auto frag = [&](int i, int eb, int part) {
      return global<x8>(fx)[(((int64_t)(w32 * 2 + i) * eb_n + eb) * kX + part) * 64 + lane];
    };
    x8 b[2][kX];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int part = 0; part < kX; ++part) b[i][part] = frag(i, 0, part);
    for (int eb = 0; eb < eb_n; ++eb) {
      x8 next[2][kX];
      const int en = min(eb + 1, eb_n - 1);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int part = 0; part < kX; ++part) next[i][part] = frag(i, en, part);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const x8 a = read_columns<T16>(tile, eb * 32, (j >> 1) * 64 + q * 16 + (j & 1) * 8);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int part = 0; part < kX; ++part) acc[i][j] = mfma(a, b[i][part], acc[i][j]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int part = 0; part < kX; ++part) b[i][part] = next[i][part];
    }
    const float s = global<float>(scales)[w32 * 32 / kGroupTokens];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = w32 * 32 + i * 16 + (lane & 15);
      if (t >= T) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = n0 + k * 32 + g * 8;
        x8 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          o[r] = (T16)(acc[i][2 * k][r] * s);
          o[r + 4] = (T16)(acc[i][2 * k + 1][r] * s);
        }
        if (c < p.d) *reinterpret_cast<x8*>(dx + (int64_t)t * p.d + c) = o;
      }
    }
  }
}

// d_Wg of kCols columns: WE waves take 32 experts each, and the WT = 8 / WE
// sets of them 64 tokens at a time in turn; x's rows of a set's tokens lie in
// LDS.  Every 64 tokens' sum is scaled and added: their own scale allows it,
// and a long sum keeps its bits.  Sets and blocks over the tokens write a
// partial sum each, part[set][E][d].
constexpr int kDwThreads = 512;
template <class T16, int WE>
__global__ __launch_bounds__(kDwThreads) void router_dw_kernel(RouterParams p, int T,
                                                               const T16* __restrict__ x,
                                                               const T16* __restrict__ fw,
                                                               const float* __restrict__ scales,
                                                               float* __restrict__ part) {
  typedef typename Split<T16>::x8 x8;
  constexpr int WT = 8 / WE, kW = Split<T16>::kW;
  constexpr int kLoads = 16 / WE;   // 16-byte chunks of 64 rows per thread of a set
  __shared__ __attribute__((aligned(16))) unsigned char tiles[WT][kGroupTokens * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int we = wave % WE, wt = wave / WE, set = blockIdx.z * WT + wt, sets = gridDim.z * WT;
  const int n0 = blockIdx.x * kCols;
  const int ET = ((p.E + 31) & ~31) / 16, et = blockIdx.y * 16 + we * 2;
  const int groups = (T + kGroupTokens - 1) / kGroupTokens, turns = (groups + sets - 1) / sets;
  const bool mine = et < ET;
  unsigned char* tile = tiles[wt];
  f32x4 acc[2][8];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  u32x4 ahead[kLoads];
  const auto load = [&](int turn) {
    const int t0 = (turn * sets + set) * kGroupTokens;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int v = (i * WE + we) * 64 + lane, t = t0 + (v >> 4), c = n0 + (v & 15) * 8;
      // (rows past the end as zeros: what lies there may be no number)
      ahead[i] = t < T && c < p.d ? *global<u32x4>(x + (int64_t)t * p.d + c) : u32x4{0, 0, 0, 0};
    }
  };
  load(0);
  for (int turn = 0; turn < turns; ++turn) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int v = (i * WE + we) * 64 + lane;
      *reinterpret_cast<u32x4*>(tile + tile_at(v >> 4, (v & 15) * 16)) = ahead[i];
    }
    __syncthreads();
    if (turn + 1 < turns) load(turn + 1);
    const int group = turn * sets + set;
    if (!mine || group >= groups) continue;
    const float s = global<float>(scales)[group];
    x8 b[2][2][kW];   // [32 tokens][16 experts][part]
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int part = 0; part < kW; ++part)
          b[k][i][part] = global<x8>(fw)[(((int64_t)(group * 2 + k) * ET + et + i) * kW + part) * 64 + lane];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      f32x4 sum[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const x8 a = read_columns<T16>(tile, k * 32, j * 32 + (lane & 3) * 8);
#pragma unroll
        for (int part = 0; part < kW; ++part)
#pragma unroll
          for (int i = 0; i < 2; ++i) sum[i] = mfma(a, b[k][i][part], sum[i]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i][j] += s * sum[i];
    }
  }
  if (!mine) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = (et + i) * 16 + (lane & 15);
    if (e >= p.E) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = n0 + j * 16 + (lane >> 4) * 4;
      if (c < p.d) *reinterpret_cast<f32x4*>(part + ((int64_t)set * p.E + e) * p.d + c) = acc[i][j];
    }
  }
}

// Sum of n partial sums in their order.
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void router_join_kernel(const float* __restrict__ part,
                                                                   int n, int64_t size,
                                                                   float* __restrict__ out) {
  const int64_t i = ((int64_t)blockIdx.x * kJoinThreads + threadIdx.x) * 4;
  if (i >= size) return;
  f32x4 s = *reinterpret_cast<const f32x4*>(part + i);
  for (int k = 1; k < n; ++k) s += *reinterpret_cast<const f32x4*>(part + k * size + i);
  *reinterpret_cast<f32x4*>(out + i) = s;
}

// Waves over the experts of a block of d_Wg, and the blocks over the tokens:
// about one block per compute unit.
int dw_waves(int E) { return E <= 32 ? 1 : E <= 64 ? 2 : E <= 128 ? 4 : 8; }
int dw_splits(int T, int d, int E) {
  const int tiles = ((d + kCols - 1) / kCols) * ((E + 255) / 256);
  const int sets = 8 / dw_waves(E), groups = (T + kGroupTokens - 1) / kGroupTokens;
  const int want = (256 + tiles - 1) / tiles, most = (groups + sets - 1) / sets;
  return want < most ? want : most;
}

size_t up(size_t b) { return (b + 255) & ~(size_t)255; }

struct Plan {
  size_t fx, fw, scales, part, bytes;  // offsets of the workspace
};
template <class T16>
Plan plan(int T, int d, int E) {
  const size_t Tp = ((size_t)T + 63) & ~(size_t)63, Ep = ((size_t)E + 31) & ~(size_t)31;
  const size_t sets = (size_t)dw_splits(T, d, E) * (8 / dw_waves(E));
  Plan q;
  size_t off = 0;
  q.fx = off; off += up(Tp * Ep * Split<T16>::kX * 2);
  q.fw = off; off += up(Tp * Ep * Split<T16>::kW * 2);
  q.scales = off; off += up(Tp / kGroupTokens * sizeof(float));
  q.part = off; off += up(sets * E * d * sizeof(float));
  q.bytes = off;
  return q;
}

template <class T16, int EB>
void dx_launch(const RouterParams& p, int T, const T16* fx, const float* scales, T16* dx, hipStream_t s) {
  // about two blocks per compute unit, 128 tokens a block and turn
  const int cols = (p.d + kCols - 1) / kCols, turns = (T + 127) / 128, want = (512 + cols - 1) / cols;
  router_dx_kernel<T16, EB><<<dim3(cols, want < turns ? want : turns), kDxThreads, 0, s>>>(p, T, fx, scales, dx);
}

template <class T16>
hipError_t run(const RouterParams& p, int T, const T16* x, const float* logits, const int32_t* idx,
               const float* dw, const float* dl, T16* dx, float* dwg, hipStream_t s) {
  const Plan q = plan<T16>(T, p.d, p.E);
  char* base = static_cast<char*>(p.grad_ws);
  T16* fx = dx ? reinterpret_cast<T16*>(base + q.fx) : nullptr;
  T16* fw = dwg ? reinterpret_cast<T16*>(base + q.fw) : nullptr;
  float* scales = reinterpret_cast<float*>(base + q.scales);
  float* part = reinterpret_cast<float*>(base + q.part);
  const int grid = (T + kGroupTokens - 1) / kGroupTokens;
  if (p.E <= 64) router_dlogits_kernel<T16, 1><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, scales);
  else if (p.E <= 128) router_dlogits_kernel<T16, 2><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, scales);
  else if (p.E <= 256) router_dlogits_kernel<T16, 4><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, scales);
  else router_dlogits_kernel<T16, 8><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, scales);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dx) {
    if (p.E <= 32) dx_launch<T16, 1>(p, T, fx, scales, dx, s);
    else if (p.E <= 64) dx_launch<T16, 2>(p, T, fx, scales, dx, s);
    else if (p.E <= 128) dx_launch<T16, 4>(p, T, fx, scales, dx, s);
    else if (p.E <= 256) dx_launch<T16, 8>(p, T, fx, scales, dx, s);
    else dx_launch<T16, 16>(p, T, fx, scales, dx, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!dwg) return hipSuccess;
  const int we = dw_waves(p.E), splits = dw_splits(T, p.d, p.E), sets = splits * (8 / we);
  const dim3 grid_w((p.d + kCols - 1) / kCols, (p.E + 255) / 256, splits);
  float* to = sets == 1 ? dwg : part;
  if (we == 1) router_dw_kernel<T16, 1><<<grid_w, kDwThreads, 0, s>>>(p, T, x, fw, scales, to);
  else if (we == 2) router_dw_kernel<T16, 2><<<grid_w, kDwThreads, 0, s>>>(p, T, x, fw, scales, to);
  else if (we == 4) router_dw_kernel<T16, 4><<<grid_w, kDwThreads, 0, s>>>(p, T, x, fw, scales, to);
  else router_dw_kernel<T16, 8><<<grid_w, kDwThreads, 0, s>>>(p, T, x, fw, scales, to);
  if ((e = hipGetLastError()) != hipSuccess || sets == 1) return e;
  const int64_t size = (int64_t)p.E * p.d;
  router_join_kernel<<<(unsigned)((size / 4 + kJoinThreads - 1) / kJoinThreads), kJoinThreads, 0, s>>>(part, sets, size, dwg);
  return hipGetLastError();
}

}  // namespace

size_t router_backward_bytes(int type, int T, int d, int E) {
  return type == TYPE_F16 ? plan<f16>(T, d, E).bytes : plan<bf16>(T, d, E).bytes;
}

hipError_t launch_router_backward(const RouterParams& p, int T, const void* x, const float* logits,
                                  const int32_t* idx, const float* dw, const float* dl, void* dx,
                                  float* dwg, hipStream_t s) {
  return p.type == TYPE_F16
             ? run(p, T, static_cast<const f16*>(x), logits, idx, dw, dl, static_cast<f16*>(dx), dwg, s)
             : run(p, T, static_cast<const bf16*>(x), logits, idx, dw, dl, static_cast<bf16*>(dx), dwg, s);
}

}  // namespace moe
