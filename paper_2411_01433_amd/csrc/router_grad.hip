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
// products are added in fp32: for fp16 two of them (22 bits, or what is
// above 2^-39 of the largest), scaled by a power of two so that the largest of
// those that one sum takes lies below 2^15: of a token for d_x, of an expert
// and 64 tokens for d_Wg; for bf16, which has the range, three (24 bits).  (Two
// for d_x, whose outputs hold 8 bits, round about one in 500 of them to the
// wrong side.)  With these d_Wg is 1.3e-7 off for both types at 512 to 8192
// tokens, an fp32 product 1.4e-7 to 6.6e-7.
#include "moe_internal.h"

namespace moe {

namespace {

typedef f16 f16x8v __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T16> struct Split;
template <> struct Split<f16> {
  typedef f16x8v x8;
  static constexpr int kParts = 2;
  static constexpr bool kScaled = true;
};
template <> struct Split<bf16> {
  typedef bf16x8 x8;
  static constexpr int kParts = 3;
  static constexpr bool kScaled = false;
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

// Fragments.  A product of 32 terms takes 8 numbers from each of 64 lanes:
// lane l has row (or column) l & 15 and the terms 4 g .. 4 g + 3 and 16 + 4 g
// .. 16 + 4 g + 3 of its group g = l >> 4, which is what two transposing reads
// of LDS give.  dl is written in this order, 1 KiB per fragment, so that a
// fragment is one contiguous load:
//   for d_x   [T/16][E/32][part][64 lanes][8]: rows tokens, terms experts
//   for d_Wg  [T/32][E/16][part][64 lanes][8]: rows experts, terms tokens
// T and E rounded up to 64 and 32, with zeros.
__device__ inline int term(int g, int j) { return j < 4 ? 4 * g + j : 12 + 4 * g + j; }

constexpr int kGroupTokens = 64;   // tokens with one scale per expert

// Power of two that brings a largest magnitude `top` to [2^14, 2^15) (to as
// much as 2^110 allows; zero like the smallest numbers), and its inverse, by
// their exponents.
struct Scale {
  float by, back;
};
__device__ inline Scale scale_of(float top) {
  const int e = min(max(268 - (int)(__builtin_bit_cast(uint32_t, top) >> 23), 14), 237);
  return {__builtin_bit_cast(float, (uint32_t)e << 23), __builtin_bit_cast(float, (uint32_t)(254 - e) << 23)};
}

// Part `part` of v: what is left of it after the parts before, in 16 bits.
template <class T16>
__device__ inline T16 next_part(float& left) {
  const T16 h = (T16)left;
  left -= (float)h;
  return h;
}

// Sum and maximum over the 16 lanes of a row, in each of them.
__device__ inline float row_sum(float v) {
  v += dpp_f<0xB1>(v);
  v += dpp_f<0x4E>(v);
  v += dpp_f<0x141>(v);
  return v + dpp_f<0x140>(v);
}
__device__ inline float row_max(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  return fmaxf(v, dpp_f<0x140>(v));
}
__device__ inline float wave_max_f(float v) {
  v = row_max(v);
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ inline float lane_value(float v, int from) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), from));
}
__device__ inline void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  __builtin_amdgcn_wave_barrier();
}

// Gradient of the logits of 64 tokens, and its fragments.  A wave has four
// tokens: 16 lanes each for their slots, all lanes for their rows of experts.
// Bound by two dependent trips to memory (index, then logit) and the writing of
// the fragments, on a block for 64 tokens: 8192 tokens x 256 experts 13.1 us
// (16.8 MB written, 128 of 256 units), 1337 x 60 of a softmax of all experts 7.2
// us, 512 x 8 5.9 us.
constexpr int kLogitThreads = 1024;
constexpr int kWaveTokens = kGroupTokens / (kLogitThreads / 64);
static_assert(kWaveTokens * 16 == 64 && kRouterMaxTopK <= 16, "a lane per slot");
template <class T16, int C>
__global__ __launch_bounds__(kLogitThreads) void router_dlogits_kernel(
    RouterParams p, int T, const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const float* __restrict__ dw, const float* __restrict__ dl, T16* __restrict__ fx,
    T16* __restrict__ fw, float* __restrict__ scale_x, float* __restrict__ scale_w,
    uint32_t* __restrict__ live) {
  typedef typename Split<T16>::x8 x8;
  constexpr int LD = C * 64 + 4;
  constexpr bool kScaled = Split<T16>::kScaled;
  __shared__ float rows[kGroupTokens][LD];
  __shared__ float by_token[kGroupTokens];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int Ep = (p.E + 31) & ~31;
  const bool sig = p.score == SCORE_SIGMOID, full = !p.renorm && !sig;
  const float none = -__builtin_inff();
  const int t0 = blockIdx.x * kGroupTokens + wave * kWaveTokens;   // the wave's first token
  const int mi = lane >> 4, k = lane & 15;                         // this lane's token and slot
  // rows of the logits (a softmax of all experts) and of their gradient: on
  // their way first
  float ex[kWaveTokens][C], more[kWaveTokens][C];
#pragma unroll
  for (int i = 0; i < kWaveTokens; ++i)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int ee = c * 64 + lane;
      const int64_t at = (int64_t)(t0 + i) * p.E + ee;
      const bool in = t0 + i < T && ee < p.E;
      ex[i][c] = full && in ? logits[at] : none;
      more[i][c] = dl && in ? dl[at] : 0.0f;
    }
  // slots
  int e = -1;
  float up = 0.0f, l = none;
  if (t0 + mi < T && k < p.K) {
    const int64_t at = (int64_t)(t0 + mi) * p.K + k;
    e = idx[at];
    if (e >= 0 && e < p.E) l = logits[(int64_t)(t0 + mi) * p.E + e];
    if (finite(l)) up = p.scale * dw[at];
    else e = -1;
  }
  const bool have = e >= 0;
  // softmax of all experts: the rows' exponentials and sums
  float top = 0.0f, all = 1.0f;
  if (full) {
#pragma unroll
    for (int i = 0; i < kWaveTokens; ++i) {
      float most = none, sum = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (finite(ex[i][c])) most = fmaxf(most, ex[i][c]);
      most = wave_max_f(most);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        ex[i][c] = finite(ex[i][c]) ? expf(ex[i][c] - most) : 0.0f;
        sum += ex[i][c];
      }
      sum = wave_sum_dpp(sum);
      if (mi == i) {
        top = most;
        all = sum;
      }
    }
  }
  // z = exp(-|l|): s and 1 - s without loss on either side
  const float z = expf(-fabsf(l));
  const float not_s = have ? (l >= 0.0f ? z : 1.0f) / (1.0f + z) : 0.0f;
  const float sc = have ? (l >= 0.0f ? 1.0f : z) / (1.0f + z) : 0.0f;
  float slot, mean = 0.0f;
  if (p.renorm) {
    const float ls = !have ? none : sig ? fminf(l, 0.0f) - log1pf(z) : l;
    const float lm = row_max(ls);
    const float v = have ? expf(ls - lm) : 0.0f;
    const float sum = row_sum(v);
    const float share = have ? v / sum : 0.0f;
    mean = row_sum(up * share);
    slot = share * (up - mean) * (sig ? not_s : 1.0f);
  } else if (sig) {
    slot = up * sc * not_s;
  } else {
    slot = have ? up * (expf(l - top) / all) : 0.0f;
    mean = row_sum(slot);
  }
  // rows: what every expert gets, then the slots on top
#pragma unroll
  for (int i = 0; i < kWaveTokens; ++i) {
    const float by = full ? -lane_value(mean, 16 * i) / lane_value(all, 16 * i) : 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int ee = c * 64 + lane;
      float v = full && ex[i][c] > 0.0f ? by * ex[i][c] : 0.0f;
      v += more[i][c];
      rows[wave * kWaveTokens + i][ee] = v;
    }
  }
  wave_lds_fence();
  float* row = rows[wave * kWaveTokens + mi];
  bool twice = false;  // an expert in two slots of a token: these in their order
  for (int j = 0; j < p.K; ++j) {
    const int ej = __shfl(e, (lane & 48) + j, 64);
    twice |= j < k && have && ej == e;
  }
  if (!__ballot(twice)) {
    if (have) row[e] += slot;
  } else {
    for (int j = 0; j < p.K; ++j) {
      if (have && k == j) row[e] += slot;
      wave_lds_fence();
    }
  }
  wave_lds_fence();
  if (fw) {
    // tokens that have a gradient at all, a bit each: the others' x may hold
    // anything (a padded row; one of no finite logit)
    uint32_t on = 0;
#pragma unroll
    for (int i = 0; i < kWaveTokens; ++i) {
      bool any = false;
#pragma unroll
      for (int c = 0; c < C; ++c) any |= !(rows[wave * kWaveTokens + i][c * 64 + lane] == 0.0f);
      on |= (__ballot(any) != 0 ? 1u : 0u) << i;
    }
    if (lane == 0) live[blockIdx.x * (kLogitThreads / 64) + wave] = on;
  }
  if (kScaled && fx) {
#pragma unroll
    for (int i = 0; i < kWaveTokens; ++i) {
      float most = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const float v = rows[wave * kWaveTokens + i][c * 64 + lane];
        if (finite(v)) most = fmaxf(most, fabsf(v));
      }
      const Scale s = scale_of(wave_max_f(most));
      if (lane == 0) {
        by_token[wave * kWaveTokens + i] = s.by;
        scale_x[t0 + i] = s.back;
      }
    }
  }
  __syncthreads();
  const int m = lane & 15, g = lane >> 4;
  const int EB = Ep / 32, ET = Ep / 16;
  if (fx)
    for (int q = wave; q < 4 * EB; q += kLogitThreads / 64) {
      const int tt = q / EB, eb = q - tt * EB;
      const float by = kScaled ? by_token[tt * 16 + m] : 1.0f;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rows[tt * 16 + m][eb * 32 + term(g, j)] * by;
      T16* to = fx + (((int64_t)(blockIdx.x * 4 + tt) * EB + eb) * Split<T16>::kParts * 64 + lane) * 8;
#pragma unroll
      for (int part = 0; part < Split<T16>::kParts; ++part) {
        x8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = next_part<T16>(v[j]);
        *reinterpret_cast<x8*>(to + part * 512) = o;
      }
    }
  if (fw)
    for (int et = wave; et < ET; et += kLogitThreads / 64) {
      float v[2][8];
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[tb][j] = rows[tb * 32 + term(g, j)][et * 16 + m];
      if constexpr (kScaled) {
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (finite(v[j >> 3][j & 7])) most = fmaxf(most, fabsf(v[j >> 3][j & 7]));
        most = fmaxf(most, __shfl_xor(most, 16, 64));
        const Scale s = scale_of(fmaxf(most, __shfl_xor(most, 32, 64)));
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j >> 3][j & 7] *= s.by;
        if (g == 0) scale_w[blockIdx.x * Ep + et * 16 + m] = s.back;
      }
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        T16* to = fw + (((int64_t)(blockIdx.x * 2 + tb) * ET + et) * Split<T16>::kParts * 64 + lane) * 8;
#pragma unroll
        for (int part = 0; part < Split<T16>::kParts; ++part) {
          x8 o;
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = next_part<T16>(v[tb][j]);
          *reinterpret_cast<x8*>(to + part * 512) = o;
        }
      }
    }
}

constexpr int kCols = 128;   // columns of d per block of the products

// LDS tile of 16-bit rows of kCols columns, 256 bytes each.  A transposing
// read takes 8 bytes of four rows in each of 16 lanes.  64-byte block b of a
// row r lies at block b ^ (r & 3), so that the four rows are in different
// banks; and so that the next 16 lanes, four rows on, are in others again,
// where r & 4 the halves of `kHalf` bytes are exchanged: of 16 bytes for
// columns read 8 bytes in 16, of 64 for columns in a row.
template <int kHalf>
__device__ inline int tile_at(int row, int byte) {
  return row * 256 + (byte ^ ((row & 3) << 6) ^ (row & 4 ? kHalf : 0));
}
template <int kHalf>
__device__ inline void tile_put(unsigned char* tile, int row, int byte, u32x4 v) {
  if (kHalf == 8 && (row & 4)) v = u32x4{v.z, v.w, v.x, v.y};
  *reinterpret_cast<u32x4*>(tile + tile_at<kHalf == 8 ? 0 : kHalf>(row, byte)) = v;
}

typedef __attribute__((address_space(3))) s16x4* LdsRead;

// 8 terms for one of 16 columns per lane from rows `row` + term(g, .) of a
// tile; lanes q = l & 3 read the columns at byte col(q) (8 bytes each), and
// lane l gets column l & 3 of the ones that q = (l & 15) >> 2 points at.
template <class T16, int kHalf>
__device__ inline typename Split<T16>::x8 read_columns(const unsigned char* tile, int row, int byte) {
  const int lane = threadIdx.x & 63;
  const int r = row + 4 * (lane >> 4) + ((lane & 15) >> 2);
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRead)(tile + tile_at<kHalf>(r, byte)));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRead)(tile + tile_at<kHalf>(r + 16, byte)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return __builtin_bit_cast(typename Split<T16>::x8, v);
}

// d_x of kCols columns: the block keeps Wg's columns in LDS (EB * 32 rows) and
// its waves take 32 tokens each in turn.  A wave's fragment of dl is loaded
// once and multiplied with 128 columns.  Blocks that follow one another, which
// the eight dies take in turn, have different tokens, so that a die's L2 holds
// its tokens' dl for all columns.  Rows of the result are columns of
// d, ordered so that a lane has 8 neighbouring ones of a token: tile 2 s + h,
// row 4 q + r is column 32 s + 8 q + 4 h + r.
// 8192 tokens x 256 experts, d 4096: 36 us (0.95 PFLOP/s of the split products,
// whose operands a wave reads from L2 and LDS in turn; a library product of the
// unsplit operands takes 32).
constexpr int kDxThreads = 256;
template <class T16, int EB>
__global__ __launch_bounds__(kDxThreads, 2) void router_dx_kernel(RouterParams p, int T,
                                                               const T16* __restrict__ fx,
                                                               const float* __restrict__ scale_x,
                                                               T16* __restrict__ dx) {
  typedef typename Split<T16>::x8 x8;
  constexpr int kParts = Split<T16>::kParts;
  __shared__ __attribute__((aligned(16))) unsigned char tile[EB * 32 * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.y * kCols, eb_n = (p.E + 31) / 32;
  constexpr int kAhead = EB < 4 ? EB * 2 : 8;   // rows of a thread on their way
  const int c16 = threadIdx.x & 15;
  for (int e0 = threadIdx.x >> 4; e0 < eb_n * 32; e0 += kAhead * 16) {
    u32x4 w[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int e = e0 + i * 16;
      const bool in = e < p.E && n0 + c16 * 8 < p.d;
      w[i] = in ? *global<u32x4>(static_cast<const T16*>(p.wg) + (int64_t)e * p.d + n0 + c16 * 8)
                : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (e0 + i * 16 < eb_n * 32) tile_put<8>(tile, e0 + i * 16, c16 * 16, w[i]);
  }
  __syncthreads();
  const int q = lane & 3, g = lane >> 4;
  // steps of 32 experts through the wave's tiles of 32 tokens, one after
  // another; dl's fragments three steps ahead, Wg's one
  const int first = blockIdx.x * 4 + wave, every = gridDim.x * 4, all = (T + 31) / 32;
  const int steps = first < all ? ((all - first + every - 1) / every) * eb_n : 0;
  f32x4 acc[2][8];
  x8 a[2][8], b[4][2][kParts];
  float scale[2];   // of this lane's two tokens
  const auto start = [&](int w32) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      scale[i] = Split<T16>::kScaled ? global<float>(scale_x)[w32 * 32 + i * 16 + (lane & 15)] : 1.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  };
  int load_at = first, load_eb = 0;
  const auto load_dl = [&](x8 (&bv)[2][kParts]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int part = 0; part < kParts; ++part)
        bv[i][part] = global<x8>(fx)[(((int64_t)(load_at * 2 + i) * eb_n + load_eb) * kParts + part) * 64 + lane];
    if (++load_eb == eb_n) {
      load_eb = 0;
      if (load_at + every < all) load_at += every;  // (past the last tile: that one again)
    }
  };
  const auto load_wg = [&](int eb, x8 (&av)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      av[j] = read_columns<T16, 8>(tile, eb * 32, (j >> 1) * 64 + q * 16 + (j & 1) * 8);
  };
  const auto write = [&](int w32) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = w32 * 32 + i * 16 + (lane & 15);
      const float s = scale[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = n0 + k * 32 + g * 8;
        x8 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          o[r] = (T16)(acc[i][2 * k][r] * s);
          o[r + 4] = (T16)(acc[i][2 * k + 1][r] * s);
        }
        if (t < T && c < p.d) *reinterpret_cast<x8*>(dx + (int64_t)t * p.d + c) = o;
      }
    }
  };
  if (steps == 0) return;
#pragma unroll
  for (int u = 0; u < 3; ++u) load_dl(b[u]);
  load_wg(0, a[0]);
  start(first);
  int w32 = first, eb = 0;
  for (int s0 = 0; s0 < steps; s0 += 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (s0 + u < steps) {
        const int next = eb + 1 < eb_n ? eb + 1 : 0;
        load_dl(b[(u + 3) & 3]);
        load_wg(next, a[(u + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i][j] = mfma(a[u & 1][j], b[u][i][part], acc[i][j]);
        if (next == 0) {
          write(w32);
          if (w32 + every < all) w32 += every;
          start(w32);
        }
        eb = next;
      }
    }
  }
}

// d_Wg of kCols columns: a block's WE waves take 32 experts each, of 64 tokens
// at a time, whose rows of x lie in LDS.  Every 64 tokens' sum is scaled and
// added: a long sum keeps its bits, and an expert whose gradients are far below
// the others' in these tokens (a softmax of all experts) its own.  Blocks over
// the tokens write a partial sum each, part[block][E][d].
// 8192 tokens x 256 experts, d 4096: 41 us (a library product of the unsplit
// operands 59), of which x comes from memory at 1.8 TB/s; the rest is the
// transposing reads of x's tile, each for 32 experts' products.
template <class T16, int WE>
__global__ __launch_bounds__(WE * 64, 2) void router_dw_kernel(RouterParams p, int T,
                                                               const T16* __restrict__ x,
                                                               const T16* __restrict__ fw,
                                                               const float* __restrict__ scale_w,
                                                               const uint32_t* __restrict__ live,
                                                               float* __restrict__ part) {
  typedef typename Split<T16>::x8 x8;
  constexpr int kParts = Split<T16>::kParts;
  constexpr int kLoads = 16 / WE;   // 16-byte chunks of 64 rows per thread
  // a turn's loads during the turn before, where registers allow
  constexpr bool kDlAhead = WE >= (kParts == 2 ? 4 : 8), kXAhead = WE >= 2;
  constexpr int kTiles = WE >= 2 ? 2 : 1;  // two tiles in turn where a unit's LDS holds them
  __shared__ __attribute__((aligned(16))) unsigned char tiles[kTiles][kGroupTokens * 256];
  const int lane = threadIdx.x & 63, we = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int set = blockIdx.x, sets = gridDim.x;
  const int n0 = blockIdx.y * kCols;
  const int ET = ((p.E + 31) & ~31) / 16, et = blockIdx.z * 16 + we * 2;
  const int groups = (T + kGroupTokens - 1) / kGroupTokens, turns = (groups + sets - 1) / sets;
  const bool mine = et < ET;
  f32x4 acc[2][8];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  u32x4 ahead[kLoads];
  uint32_t on[kLoads];   // which of a chunk's four tokens have a gradient
  static_assert(kWaveTokens == 4, "four tokens per word of live");
  x8 b[2][2][kParts];   // [32 tokens][16 experts][part]
  float s[2] = {1.0f, 1.0f};   // scales of this lane's two experts
  const auto load_x = [&](int turn) {
    const int t0 = (turn * sets + set) * kGroupTokens;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int v = (i * WE + we) * 64 + lane, t = t0 + (v >> 4), c = n0 + (v & 15) * 8;
      on[i] = global<uint32_t>(live)[min(turn * sets + set, groups - 1) * 16 + i * WE + we];
      // (rows past the end as zeros: what lies there may be no number)
      ahead[i] = t < T && c < p.d ? *global<u32x4>(x + (int64_t)t * p.d + c) : u32x4{0, 0, 0, 0};
    }
  };
  const auto load_dl = [&](int turn) {
    const int group = min(turn * sets + set, groups - 1), tile_e = min(et, ET - 2);
    if constexpr (Split<T16>::kScaled) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        s[i] = global<float>(scale_w)[(group * ET + tile_e + i) * 16 + (lane & 15)];
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int part = 0; part < kParts; ++part)
          b[k][i][part] = global<x8>(fw)[(((int64_t)(group * 2 + k) * ET + tile_e + i) * kParts + part) * 64 + lane];
  };
  if (kXAhead) load_x(0);
  if (kDlAhead) load_dl(0);
  for (int turn = 0; turn < turns; ++turn) {
    unsigned char* tile = tiles[turn % kTiles];
    if (!kXAhead) load_x(turn);
    if (kTiles == 1) __syncthreads();   // (the last turn's reads)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int v = (i * WE + we) * 64 + lane;
      const bool has = on[i] >> (lane >> 4) & 1;
      tile_put<32>(tile, v >> 4, (v & 15) * 16, has ? ahead[i] : u32x4{0, 0, 0, 0});
    }
    if (kXAhead) load_x(turn + 1);
    if (!kDlAhead) load_dl(turn);
    __syncthreads();
    x8 now[2][2][kParts];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int part = 0; part < kParts; ++part) now[k][i][part] = b[k][i][part];
    const float by[2] = {s[0], s[1]};
    if (kDlAhead) load_dl(turn + 1);
    __builtin_amdgcn_sched_barrier(0);
    if (!mine || turn * sets + set >= groups) continue;
    // two tiles of 16 columns at a time, four sums that do not wait for one
    // another; the next two's fragments of x are read meanwhile, and the last
    // two's sums added
    x8 a[2][2][2];   // [turn][tile][32 tokens]
    f32x4 sum[2][2][2];
    const auto read = [&](int j, x8 (&av)[2][2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          av[h][k] = read_columns<T16, 32>(tile, k * 32, (j * 2 + h) * 32 + (lane & 3) * 8);
    };
    read(0, a[0]);
#pragma unroll
    for (int j = 0; j < 5; ++j) {
      if (j < 3) read(j + 1, a[(j + 1) & 1]);
      if (j < 4) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int i = 0; i < 2; ++i)
                sum[j & 1][h][i] = mfma(a[j & 1][h][k], now[k][i][part],
                                        k == 0 && part == 0 ? f32x4{0, 0, 0, 0} : sum[j & 1][h][i]);
      }
      if (j > 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 2; ++i) acc[i][(j - 1) * 2 + h] += by[i] * sum[(j - 1) & 1][h][i];
      }
      __builtin_amdgcn_sched_barrier(0);
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

// Sum of n partial sums: a wave each for every fourth of them, then theirs in
// order.  Bound by memory: 8 parts of 256 x 4096 in 6.8 us (5.5 TB/s).
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void router_join_kernel(const float* __restrict__ part,
                                                                   int n, int64_t size,
                                                                   float* __restrict__ out) {
  __shared__ f32x4 sums[3][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = ((int64_t)blockIdx.x * 64 + lane) * 4;
  f32x4 s = {0, 0, 0, 0};
  if (i < size) {
#pragma unroll 4
    for (int k = wave; k < n; k += 4) s += *reinterpret_cast<const f32x4*>(part + k * size + i);
  }
  if (wave) sums[wave - 1][lane] = s;
  __syncthreads();
  if (wave == 0 && i < size)
    *reinterpret_cast<f32x4*>(out + i) = s + sums[0][lane] + sums[1][lane] + sums[2][lane];
}

// Waves over the experts of a block of d_Wg, and the blocks over the tokens:
// eight waves per compute unit above 128 experts, else four.  us of product and
// sum at d 4096 with half / these / twice as many: 8192 tokens x 256 experts
// 69.4 47.4 59.6, 1000 x 256 24.7 25.2 37.6, 8192 x 100 50.6 33.4 30.2, 1000 x
// 100 16.3 17.6 20.8, 8192 x 60 40.6 30.5 29.4, 8192 x 8 30.3 24.0 22.6 (twice
// as many are also twice the workspace).
int dw_waves(int E) { return E <= 32 ? 1 : E <= 64 ? 2 : E <= 128 ? 4 : 8; }
int dw_splits(int T, int d, int E) {
  const int tiles = ((d + kCols - 1) / kCols) * ((E + 255) / 256);
  const int groups = (T + kGroupTokens - 1) / kGroupTokens;
  const int we = dw_waves(E), want = ((we == 8 ? 256 : 1024 / we) + tiles - 1) / tiles;
  return want < groups ? want : groups;
}

size_t up(size_t b) { return (b + 255) & ~(size_t)255; }

struct Plan {
  size_t fx, fw, scale_x, scale_w, live, part, bytes;  // offsets of the workspace
};
template <class T16>
Plan plan(int T, int d, int E) {
  const size_t Tp = ((size_t)T + 63) & ~(size_t)63, Ep = ((size_t)E + 31) & ~(size_t)31;
  const size_t sets = (size_t)dw_splits(T, d, E);
  Plan q;
  size_t off = 0;
  q.fx = off; off += up(Tp * Ep * Split<T16>::kParts * 2);
  q.fw = off; off += up(Tp * Ep * Split<T16>::kParts * 2);
  q.scale_x = off; off += up(Split<T16>::kScaled ? Tp * sizeof(float) : 0);
  q.scale_w = off; off += up(Split<T16>::kScaled ? Tp / kGroupTokens * Ep * sizeof(float) : 0);
  q.live = off; off += up(Tp / kWaveTokens * sizeof(uint32_t));
  q.part = off; off += up(sets * E * d * sizeof(float));
  q.bytes = off;
  return q;
}

template <class T16, int EB>
void dx_launch(const RouterParams& p, int T, const T16* fx, const float* sx, T16* dx, hipStream_t s) {
  // about two blocks per compute unit, 128 tokens a block and turn.  us at 8192
  // tokens, d 4096, with one / two / four blocks: 8 experts 16.0 15.9 16.5, 60
  // 19.8 18.2 19.0, 256 42.6 35.4 37.2
  const int cols = (p.d + kCols - 1) / kCols, turns = (T + 127) / 128, want = (512 + cols - 1) / cols;
  router_dx_kernel<T16, EB><<<dim3(want < turns ? want : turns, cols), kDxThreads, 0, s>>>(p, T, fx, sx, dx);
}

template <class T16>
hipError_t run(const RouterParams& p, int T, const T16* x, const float* logits, const int32_t* idx,
               const float* dw, const float* dl, T16* dx, float* dwg, hipStream_t s) {
  const Plan q = plan<T16>(T, p.d, p.E);
  char* base = static_cast<char*>(p.grad_ws);
  T16* fx = dx ? reinterpret_cast<T16*>(base + q.fx) : nullptr;
  T16* fw = dwg ? reinterpret_cast<T16*>(base + q.fw) : nullptr;
  float* sx = reinterpret_cast<float*>(base + q.scale_x);
  float* sw = reinterpret_cast<float*>(base + q.scale_w);
  uint32_t* live = reinterpret_cast<uint32_t*>(base + q.live);
  float* part = reinterpret_cast<float*>(base + q.part);
  const int grid = (T + kGroupTokens - 1) / kGroupTokens;
  if (p.E <= 64) router_dlogits_kernel<T16, 1><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, sx, sw, live);
  else if (p.E <= 128) router_dlogits_kernel<T16, 2><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, sx, sw, live);
  else if (p.E <= 256) router_dlogits_kernel<T16, 4><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, sx, sw, live);
  else router_dlogits_kernel<T16, 8><<<grid, kLogitThreads, 0, s>>>(p, T, logits, idx, dw, dl, fx, fw, sx, sw, live);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dx) {
    if (p.E <= 32) dx_launch<T16, 1>(p, T, fx, sx, dx, s);
    else if (p.E <= 64) dx_launch<T16, 2>(p, T, fx, sx, dx, s);
    else if (p.E <= 128) dx_launch<T16, 4>(p, T, fx, sx, dx, s);
    else if (p.E <= 256) dx_launch<T16, 8>(p, T, fx, sx, dx, s);
    else dx_launch<T16, 16>(p, T, fx, sx, dx, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!dwg) return hipSuccess;
  const int we = dw_waves(p.E), sets = dw_splits(T, p.d, p.E);
  const dim3 grid_w(sets, (p.d + kCols - 1) / kCols, (p.E + 255) / 256);
  float* to = sets == 1 ? dwg : part;
  if (we == 1) router_dw_kernel<T16, 1><<<grid_w, 64, 0, s>>>(p, T, x, fw, sw, live, to);
  else if (we == 2) router_dw_kernel<T16, 2><<<grid_w, 128, 0, s>>>(p, T, x, fw, sw, live, to);
  else if (we == 4) router_dw_kernel<T16, 4><<<grid_w, 256, 0, s>>>(p, T, x, fw, sw, live, to);
  else router_dw_kernel<T16, 8><<<grid_w, 512, 0, s>>>(p, T, x, fw, sw, live, to);
  if ((e = hipGetLastError()) != hipSuccess || sets == 1) return e;
  const int64_t size = (int64_t)p.E * p.d;
  router_join_kernel<<<(unsigned)((size / 4 + 63) / 64), kJoinThreads, 0, s>>>(part, sets, size, dwg);
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
