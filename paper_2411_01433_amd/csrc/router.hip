// Routing rules: scores of the gate's logits, a bias that steers the balance,
// groups of experts, top-k and the weights.
//
//   l = x Wg^T;  s = sigmoid(l) or softmax(l);  key = s + b, or l without a b
//   group score = sum of the group's one or two best keys (scores without b)
//   top-k of the keys in the groups that count most, ties to the lower index
//   w = scale s, or scale s / sum of the selected s
//
// The logits are a matrix product on the matrix cores, in fp32 sums; another
// kernel takes a wave per token for everything else.
//
// Which of two near keys is larger decides what is selected, and fp32 sums
// differ in their last bits with the split of the sum.  So the first kernel
// also gives the norms of the rows of x and Wg, whose product bounds the
// error of a logit, and the selection knows how near two keys may be to be in
// order for certain.  Where two keys (or groups) that decide something are
// nearer - for a few tokens in a hundred - the logits in question are summed
// again in 64 bits, and those decide.
#include "moe_internal.h"

namespace moe {

namespace {

typedef f16 f16x8v __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Pointers that come in a struct would be loaded from as generic ones.
template <class T>
using Global = const __attribute__((address_space(1))) T*;
template <class T>
__device__ inline Global<T> global(const void* p) {
  return (Global<T>)(const T*)p;
}

template <class T16> struct Vec;
template <> struct Vec<f16> { typedef f16x8v x8; };
template <> struct Vec<bf16> { typedef bf16x8 x8; };

__device__ inline f32x4 mfma(f16x8v a, f16x8v b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// acc + the squares of a piece of a row
__device__ inline float squares(f16x8v v, float acc) {
  const u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = u[i];
    acc = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), __builtin_bit_cast(f16x2, w), acc, false);
  }
  return acc;
}
__device__ inline float squares(bf16x8 v, float acc) {
  const u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = u[i];
    acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, w), acc, false);
  }
  return acc;
}
// Whether a piece has a number other than a zero of either sign.
__device__ inline bool any_bits(u32x4 u) {
  return (((u.x | u.y) | (u.z | u.w)) & 0x7FFF7FFFu) != 0;
}

// Error of a logit.  A step of the matrix cores takes its 32 columns in four
// groups of 8, one after another.  A group's products are cut at 2^-24 of 2^e,
// the largest sum of two factors' exponents (subnormals have the least normal
// one), and so is the sum up to there, unless it is so large that the group's
// sum is cut at 2^-31 of it; then the two are added and rounded.  (Measured, as
// documents do not say it: 1.2 million sums of all kinds equal this bit for
// bit.)  So with u = 2^-24 a group costs at most 8 u 2^e and u (1 + 2^-7) of the
// sum S_g that it leaves.  A sum starts with every piece of 64 columns, so that
// S_g is at most |x_g| |w_g|, the norms of the piece's columns up to it; adding
// the piece to the wave's others costs u of their sum, by norms |x_i| |w_i| of
// the wave's columns so far, and the join of the waves' sums u of each.  2^e is
// at most the product of the group's largest |x| and |w|, or 2^-14 for fp16
// where that is more.  With both norms taken apart, all of it is at most
// u q(x) q(w),
//   q(x)^2 = 1.01 (sum over groups |x_g|^2 + sum over pieces |x_i|^2)
//            + (waves + 7) |x|^2 + d 2^-28 (fp16).
// (A sum over all of a wave's columns at once would have a bound 2 to 3 times as
// large at d 4096: 8192 x 256 in groups 81 us instead of 76, for the tokens that
// it leaves open.)
// The squares of fp16 do not underflow in fp32; those of bf16 do below 1e-19,
// and then count as the largest norm that can go with so small a sum (and with
// subnormals).  A row of zeros has q 0, and its logits are exact.
template <class T16>
__device__ inline float error_norm(float q2, bool some, int d) {
  if (!some) return 0.0f;
  if constexpr (__is_same(T16, f16)) q2 += (float)d * 0x1p-28f;
  return fmaxf(sqrtf(q2) * 1.0001f, 1e-13f);
}
constexpr float kSumError = 0x1p-24f;
__device__ inline float logit_error(float qx, float qw) {
  // (rounding to fp32 of the smallest numbers adds to a bound; sums that stay
  // finite have no product of 2^128, and are off by less than the upper one,
  // ten times 2^103 in each of at most 2048 groups)
  return qx > 0.0f && qw > 0.0f ? fminf(kSumError * qx * qw + 1e-33f, 1e36f) : 0.0f;
}

// ---- selection ------------------------------------------------------------

constexpr float kLargest = 3.402823466e38f;
__device__ inline bool finite(float v) { return fabsf(v) <= kLargest; }

// Sum and maximum of doubles over a wave in registers (see wave_sum_dpp).
template <int CTRL>
__device__ inline double dpp_d(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL>
__device__ inline double dpp_of(double v) { return dpp_d<CTRL>(v); }
template <int CTRL>
__device__ inline float dpp_of(float v) { return dpp_f<CTRL>(v); }
// The value that lane `from` (the same for all) has.
__device__ inline float lane_value(float v, int from) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), from));
}
__device__ inline double lane_value(double v, int from) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, from);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), from);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// (exp(-v) leaves the range below -709, before its inverse does)
__device__ inline double sigmoid(double v) {
  const double z = exp(-fabs(v));
  return (v < 0.0 ? z : 1.0) / (1.0 + z);
}
__device__ inline double pair_d(uint32_t lo, uint32_t hi) {
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ inline double wave_sum(double v) {
  v += dpp_d<0xB1>(v);
  v += dpp_d<0x4E>(v);
  v += dpp_d<0x141>(v);
  v += dpp_d<0x140>(v);
  uint64_t u = __builtin_bit_cast(uint64_t, v);
  auto l = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
  auto h = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  v = pair_d(l[0], h[0]) + pair_d(l[1], h[1]);
  u = __builtin_bit_cast(uint64_t, v);
  l = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
  h = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return pair_d(l[0], h[0]) + pair_d(l[1], h[1]);
}
__device__ inline double wave_max(double v) {
  // order-preserving key, its upper half first
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t k = u >> 63 ? ~u : u | 1ull << 63;
  const uint32_t hi = wave_max_u32((uint32_t)(k >> 32));
  const uint32_t lo = wave_max_u32((uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  const uint64_t m = (uint64_t)hi << 32 | lo;
  return __builtin_bit_cast(double, m >> 63 ? m & ~(1ull << 63) : ~m);
}
__device__ inline float key_float(uint32_t k) {
  return __builtin_bit_cast(float, (k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
__device__ inline float wave_max(float v) { return key_float(wave_max_u32(float_key(v))); }

// LDS of one wave is written and read by that wave alone.
__device__ inline void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  __builtin_amdgcn_wave_barrier();
}

// The same order for the compiler alone, which may take a lane's address as not
// another's: a wave's LDS operations are done in their order, so that nothing
// has to be waited for, least of all global loads on their way.
__device__ inline void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

// x . w for two rows w over d columns by one wave, in 64 bits (a product of two
// 16-bit numbers is exact there).  Every lane gets the sums.
template <class T16>
__device__ inline void exact_dots(const T16* x, const T16* w0, const T16* w1, int d, double& s0,
                                  double& s1) {
  typedef typename Vec<T16>::x8 x8;
  constexpr int B = 4;  // pieces whose loads are in flight together
  s0 = s1 = 0.0;
  for (int c0 = (threadIdx.x & 63) * 8; c0 < d; c0 += 512 * B) {
    x8 a[B], b[B], e[B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int c = min(c0 + 512 * i, d - 8);
      a[i] = *global<x8>(x + c);
      b[i] = *global<x8>(w0 + c);
      e[i] = *global<x8>(w1 + c);
    }
#pragma unroll
    for (int i = 0; i < B; ++i)
      if (c0 + 512 * i < d) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const double v = (double)(float)a[i][j];
          s0 = fma(v, (double)(float)b[i][j], s0);
          s1 = fma(v, (double)(float)e[i][j], s1);
        }
      }
  }
  s0 = wave_sum(s0);
  s1 = wave_sum(s1);
}

// Two best values of each group and what decides about it: 64 / G lanes per
// group (G the groups rounded up to a power of two) scan its members and join.
template <class F>
struct GroupBest {
  F sum;   // of the group's best one or two; -inf for a group without any
  F low;   // the least value that counts in it
};
template <class F>
__device__ inline GroupBest<F> group_best(const RouterParams& p, const F* row, int lane, int per, int g) {
  const F none = -__builtin_inff();
  const int size = p.E / p.n_groups;
  F best = none, second = none;
  if (g < p.n_groups)
    for (int i = lane & (per - 1); i < size; i += per) {
      const F v = row[g * size + i];
      second = v > best ? best : v > second ? v : second;
      best = v > best ? v : best;
    }
  const auto join = [&](F ob, F os) {
    const F lo = ob > best ? best : ob;
    second = os > second ? os : second;
    second = lo > second ? lo : second;
    best = ob > best ? ob : best;
  };
  // lane ^ 1, lane ^ 2, mirrors in 8 and 16, then the other row of 16 and half
  if (per > 1) join(dpp_of<0xB1>(best), dpp_of<0xB1>(second));
  if (per > 2) join(dpp_of<0x4E>(best), dpp_of<0x4E>(second));
  if (per > 4) join(dpp_of<0x141>(best), dpp_of<0x141>(second));
  if (per > 8) join(dpp_of<0x140>(best), dpp_of<0x140>(second));
  if (per > 16) join(__shfl_xor(best, 16, 64), __shfl_xor(second, 16, 64));
  if (per > 32) join(__shfl_xor(best, 32, 64), __shfl_xor(second, 32, 64));
  const bool two = p.group_best == 2 && second > none;
  F sum = two ? best + second : best;
  // two of the type's lowest are not the infinity of a group without any
  if constexpr (sizeof(F) == 4) sum = two ? fminf(fmaxf(sum, -kLargest), kLargest) : sum;
  return {sum, two ? second : best};
}

// One token's fp32 selection, by one wave: lane i has the experts i, i + 64,
// ... (C of them), lane k slot k.
template <int C>
struct Token {
  float l[C], b[C], key[C], kerr[C];
  float val[C];       // what groups count
  float err[C];       // bound of l's error; 0 where a row is all zeros
  bool fit[C];        // can be selected at all
  bool kept[C];       // ... and lies in a group that stays
  // lanes of group g (lanes_per_group of them): its best members, whether it
  // stays, the least sum that does and the largest that does not
  GroupBest<float> group;
  bool stays;
  float in, out, group_err;
  float top, z, zrel; // softmax: largest logit, denominator, its relative error
  float margin;       // keys further apart are certainly in order
  bool vague;         // scores whose errors are no small part of them
  bool groups_open, slots_open;
  int sel;
  float sl;           // its logit
};

__device__ inline int lanes_per_group(const RouterParams& p) {
  int per = 64;
  while (64 / per < p.n_groups) per >>= 1;
  return per;
}

// Group of expert e < 512: size_inv is 2^20 / size rounded up, which is off by
// less than 2^-11 for such e, below the 1/size by which e / size can miss a
// whole number.
__device__ inline int group_of(const RouterParams& p, int e) { return (int)((uint32_t)(e * p.size_inv) >> 20); }

// Error of a group's sum.
template <int C>
__device__ inline float group_margin(const Token<C>& tk) {
  return tk.group_err + 5e-7f * fmaxf(fabsf(tk.in), fabsf(tk.out));
}

// Whether this lane's group may be on the other side within `room`.
template <int C>
__device__ inline bool contested(const RouterParams& p, const Token<C>& tk, float room) {
  return (int)(threadIdx.x & 63) / lanes_per_group(p) < p.n_groups && tk.group.sum > -__builtin_inff() &&
         (tk.stays ? tk.group.sum - tk.out <= room : tk.in - tk.group.sum <= room);
}

// The experts of the groups that stay.
template <int C>
__device__ inline void keep_groups(const RouterParams& p, Token<C>& tk) {
  const int lane = threadIdx.x & 63, per = lanes_per_group(p);
  const uint64_t at = __ballot(tk.stays);
#pragma unroll
  for (int c = 0; c < C; ++c)
    tk.kept[c] = tk.fit[c] && (at >> min(group_of(p, c * 64 + lane) * per, 63) & 1);
}

// The waves that work on one open token: a block of TW, or one wave by itself.
// All of a team make the same selection and share the sums in 64 bits.
template <int TW>
struct Team {
  static __device__ void sync() {
    if constexpr (TW == 1) wave_lds_fence();
    else __syncthreads();
  }
  static __device__ bool lead() { return TW == 1 || threadIdx.x < 64; }
  static __device__ int wave() { return TW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
};

// LDS of a team that works on a token whose selection is open.
template <int C>
struct OpenLds {
  double row[C * 64];    // logits, then keys or scores for the groups' scan
  double dots[C * 64];   // logits summed again
  int32_t list[C * 64];  // ... and their experts
};

// Sums the logits of the experts of `want` again, in 64 bits, the team's
// waves in turn: n of them, in lds.list and lds.dots.  Every wave has the same
// `want` and calls this.
template <class T16, int C, int TW>
__device__ inline int sum_again(const RouterParams& p, const T16* xr, const bool (&want)[C], OpenLds<C>& lds) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint64_t m = __ballot(want[c]);
    if (want[c] && Team<TW>::lead())
      lds.list[n + __popcll(m & ((1ull << lane) - 1ull))] = c * 64 + lane;
    n += __popcll(m);
  }
  Team<TW>::sync();
  // two of them at a time, unless the team has a wave for each
  const int step = n > TW ? 2 : 1;
  for (int i = Team<TW>::wave() * step; i < n; i += TW * step) {
    const int last = min(i + step, n) - 1;
    const int e0 = __builtin_amdgcn_readfirstlane(lds.list[i]);
    const int e1 = __builtin_amdgcn_readfirstlane(lds.list[last]);
    const T16* wg = static_cast<const T16*>(p.wg);
    double s0, s1;
    exact_dots(xr, wg + (int64_t)e0 * p.d, wg + (int64_t)e1 * p.d, p.d, s0, s1);
    if (lane == 0) {
      lds.dots[last] = s1;
      lds.dots[i] = s0;
    }
  }
  Team<TW>::sync();
  return n;
}

// The whole selection in 64 bits: every logit that enters it is summed again.
template <class T16, int C, int TW>
__device__ void select_all(const RouterParams& p, const T16* xr, Token<C>& tk, OpenLds<C>& lds) {
  const int lane = threadIdx.x & 63;
  const double none = -__builtin_inf();
  const bool biased = p.bias != nullptr, soft = p.score == SCORE_SOFTMAX;
  bool want[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    want[c] = finite(tk.l[c]) && (soft || tk.fit[c]) && tk.err[c] > 0.0f;
    if (Team<TW>::lead()) lds.row[c * 64 + lane] = tk.l[c];
  }
  const int n = sum_again<T16, C, TW>(p, xr, want, lds);
  if (Team<TW>::lead())
    for (int i = lane; i < n; i += 64) lds.row[lds.list[i]] = lds.dots[i];
  Team<TW>::sync();
  double key[C], top = none, z = 0.0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    key[c] = lds.row[c * 64 + lane];
    if (finite(tk.l[c])) top = fmax(top, key[c]);
  }
  if (soft) {
    top = wave_max(top);
#pragma unroll
    for (int c = 0; c < C; ++c) z += finite(tk.l[c]) ? exp(key[c] - top) : 0.0;
    z = wave_sum(z);
    tk.top = (float)top;   // (for the weights)
    tk.z = (float)z;
  }
  Team<TW>::sync();
#pragma unroll
  for (int c = 0; c < C; ++c) {
    tk.l[c] = finite(tk.l[c]) ? (float)key[c] : tk.l[c];
    const double sc = !tk.fit[c] ? 0.0 : soft ? exp(key[c] - top) / z : sigmoid(key[c]);
    if (biased) key[c] = sc + tk.b[c];
    if (Team<TW>::lead()) lds.row[c * 64 + lane] = !tk.fit[c] ? none : biased ? key[c] : sc;
    tk.kept[c] = tk.fit[c];
  }
  Team<TW>::sync();
  if (p.n_groups > 1) {
    const int per = lanes_per_group(p), g = lane / per;
    const GroupBest<double> gb = group_best(p, lds.row, lane, per, g);
    int rank = 0;
#pragma unroll 1
    for (int h = 0; h < p.n_groups; ++h) {
      const double v = lane_value(gb.sum, h * per);
      rank += v > gb.sum || (v == gb.sum && h < g);
    }
    tk.stays = g < p.n_groups && rank < p.top_groups;
    keep_groups(p, tk);
  }
  tk.sel = -1;
  for (int k = 0; k < p.K; ++k) {
    double best = none;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (tk.kept[c]) best = fmax(best, key[c]);
    best = wave_max(best);
    int e = -1;
    float l = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint64_t m = __ballot(tk.kept[c] && key[c] == best);
      if (e < 0 && m) {
        const int at = __ffsll((unsigned long long)m) - 1;
        e = c * 64 + at;
        l = lane_value(tk.l[c], at);
      }
    }
    e = __builtin_amdgcn_readfirstlane(e);
    if (e < 0) break;  // nobody left
#pragma unroll
    for (int c = 0; c < C; ++c) tk.kept[c] = tk.kept[c] && c * 64 + lane != e;
    if (lane == k) {
      tk.sel = e;
      tk.sl = l;
    }
  }
  Team<TW>::sync();
}

// Descending order of a lane's C keys, each with its number c.
template <int C>
__device__ inline void sort_lane(uint32_t (&k)[C], int (&e)[C]) {
  const auto step = [&](int i, int j) {
    const bool swap = k[j] > k[i];
    const uint32_t kt = swap ? k[j] : k[i];
    k[j] = swap ? k[i] : k[j];
    k[i] = kt;
    const int et = swap ? e[j] : e[i];
    e[j] = swap ? e[i] : e[j];
    e[i] = et;
  };
  // odd-even merging: pairs, fours, eights
#pragma unroll
  for (int n = 1; n < C; n *= 2)
#pragma unroll
    for (int m = n; m >= 1; m /= 2)
#pragma unroll
      for (int j = m % n; j + m < C; j += 2 * m)
#pragma unroll
        for (int i = 0; i < m; ++i)
          if (i + j + m < C && (i + j) / (2 * n) == (i + j + m) / (2 * n)) step(i + j, i + j + m);
}

// Logits of one token and the bounds of their errors.
template <int C>
__device__ inline void load_token(const RouterParams& p, Global<float> lg, Global<float> wn, float xn,
                                  Token<C>& tk) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int e = c * 64 + lane;
    const bool in = e < p.E;
    tk.l[c] = in ? lg[e] : -__builtin_inff();
    tk.b[c] = in && p.bias ? global<float>(p.bias)[e] : 0.0f;
    tk.err[c] = in ? logit_error(xn, wn[e]) : 0.0f;
  }
}

// Scores, keys and groups of a token in fp32.  Keys are compared with one
// margin, twice the largest bound of their errors.  For the slots each lane
// sorts its keys, and a slot takes the largest of the lanes' first ones
// (take_slots).  row: C * 64 floats of LDS of the wave's own.
template <int C>
__device__ inline void score_token(const RouterParams& p, float* row, Token<C>& tk) {
  const int lane = threadIdx.x & 63;
  const float none = -__builtin_inff();
  const bool biased = p.bias != nullptr, soft = p.score == SCORE_SOFTMAX;
  float sc[C];
  float worst = 0.0f;
  tk.top = none;
  tk.z = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    tk.fit[c] = finite(tk.l[c]);
    if (tk.fit[c]) tk.top = fmaxf(tk.top, tk.l[c]);
    worst = fmaxf(worst, tk.fit[c] ? tk.err[c] : 0.0f);
  }
  // The scores by the fast exponential and reciprocal: within 1e-6 of a
  // score, of a sigmoid 1.2e-7 more for each unit below 0 (the exponent's
  // rounding), and of a softmax's term 1e-6 for each unit below the largest.
  tk.zrel = soft ? wave_max(worst) + 4e-6f : 0.0f;
  // A relative error r of a term counts as 1.01 r, which holds for its
  // exponential up to 0.015; logits known less well, of thousands, leave all to
  // 64 bits where scores enter the selection.
  tk.vague = soft && (biased || p.n_groups > 1) && tk.zrel > 0.007f;
  if (soft) {
    tk.top = wave_max(tk.top);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      sc[c] = tk.fit[c] ? __expf(tk.l[c] - tk.top) : 0.0f;
      tk.z += sc[c];
    }
    tk.z = wave_sum_dpp(tk.z);
  }
  float verr[C];      // errors of what groups count
  float most = 0.0f;
  worst = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float e1;
    if (soft) {
      sc[c] = tk.fit[c] ? sc[c] * __builtin_amdgcn_rcpf(tk.z) : 0.0f;
      e1 = tk.fit[c] ? sc[c] * 1.01f * (tk.err[c] + tk.zrel + 1e-6f * (tk.top - tk.l[c])) : 0.0f;
    } else {
      sc[c] = tk.fit[c] ? __builtin_amdgcn_rcpf(1.0f + __expf(-tk.l[c])) : 0.0f;
      // (the sigmoid's slope here, and what it may change by within the bound)
      e1 = tk.err[c] * (1.001f * sc[c] * (1.0f - sc[c]) + 0.1f * tk.err[c]) +
           (1e-6f + 1.2e-7f * fmaxf(-tk.l[c], 0.0f)) * sc[c];
    }
    tk.key[c] = tk.l[c];
    if (biased) {
      tk.fit[c] = tk.fit[c] && finite(tk.b[c]);
      tk.key[c] = sc[c] + tk.b[c];
      e1 += 1e-7f * fabsf(tk.key[c]);
    }
    verr[c] = e1;
    most = fmaxf(most, tk.fit[c] ? e1 : 0.0f);
    tk.kerr[c] = biased ? e1 : tk.err[c];
    worst = fmaxf(worst, tk.fit[c] ? tk.kerr[c] : 0.0f);
    tk.kept[c] = tk.fit[c];
  }
  tk.margin = 2.0f * wave_max(worst);
  tk.group_err = p.group_best * wave_max(most);
  tk.groups_open = false;
  if (p.n_groups > 1) {
    const int per = lanes_per_group(p);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      tk.val[c] = tk.fit[c] ? (biased ? tk.key[c] : sc[c]) : none;
      row[c * 64 + lane] = tk.val[c];
    }
    wave_lds_fence();
    const int g = lane / per;
    tk.group = group_best(p, row, lane, per, g);
    // a group's rank, in all of its lanes
    int rank = 0;
    for (int h = 0; h < p.n_groups; ++h) {
      const float v = lane_value(tk.group.sum, h * per);
      rank += v > tk.group.sum || (v == tk.group.sum && h < g);
    }
    const bool is = g < p.n_groups;
    tk.stays = is && rank < p.top_groups;
    // the least kept group against the best of the others
    tk.in = -wave_max(tk.stays ? -tk.group.sum : none);
    tk.out = wave_max(is && !tk.stays ? tk.group.sum : none);
    tk.groups_open = tk.out > none && tk.in - tk.out <= 2.0f * group_margin(tk);
    if (tk.groups_open) {
      // again by the errors of those that may count in a group whose place is
      // open: a bias that masks has the largest, and counts nowhere
      const float room = 2.0f * group_margin(tk);
      const uint64_t cm = __ballot(contested(p, tk, room));
      most = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = min(group_of(p, c * 64 + lane) * per, 63);
        const float low = __shfl(tk.group.low, at, 64);
        const bool counts = tk.fit[c] && (cm >> at & 1) && tk.val[c] >= low - room;
        most = fmaxf(most, counts ? verr[c] : 0.0f);
      }
      tk.group_err = p.group_best * wave_max(most);
      tk.groups_open = tk.in - tk.out <= 2.0f * group_margin(tk);
    }
    keep_groups(p, tk);
    wave_lds_fence();
  }
}

// Slots of the kept experts by their fp32 keys.
template <int C>
__device__ inline void take_slots(const RouterParams& p, float* row, Token<C>& tk) {
  const int lane = threadIdx.x & 63;
  uint32_t hk[C];
  int he[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    row[c * 64 + lane] = tk.l[c];
    hk[c] = tk.kept[c] ? float_key(tk.key[c] + 0.0f) : 0u;  // (one zero)
    he[c] = c * 64 + lane;
  }
  sort_lane(hk, he);
  tk.sel = -1;
  uint64_t near = 0;
  float last = 0.0f;
  for (int k = 0; k < p.K; ++k) {
    const uint32_t m = __builtin_amdgcn_readfirstlane(wave_max_u32(hk[0]));
    if (m == 0) break;  // nobody left
    last = key_float(m);
    const int from = __ffsll((unsigned long long)__ballot(hk[0] == m)) - 1;
    const int e = __builtin_amdgcn_readlane(he[0], from);
    if (lane == k) tk.sel = e;
    const bool mine = lane == from;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      hk[c] = mine ? (c + 1 < C ? hk[c + 1] : 0u) : hk[c];
      he[c] = mine ? (c + 1 < C ? he[c + 1] : 0) : he[c];
    }
    near |= __ballot(hk[0] >= float_key(last - tk.margin));
  }
  if (near) {
    // again by the margin of those that count: the slots and what comes near
    float worst = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
      worst = fmaxf(worst, tk.kept[c] && tk.key[c] >= last - tk.margin ? tk.kerr[c] : 0.0f);
    tk.margin = 2.0f * wave_max(worst);
    near = 0;
    for (int k = 0; k < p.K; ++k) {
      const int e = __builtin_amdgcn_readlane(tk.sel, k);
      if (e < 0) break;
      float ke = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (e >> 6 == c) ke = lane_value(tk.key[c], e & 63);
#pragma unroll
      for (int c = 0; c < C; ++c)
        near |= __ballot(tk.kept[c] && c * 64 + lane != e && fabsf(tk.key[c] - ke) <= tk.margin);
    }
  }
  tk.slots_open = near != 0;
  wave_lds_fence();
  tk.sl = tk.sel >= 0 ? row[tk.sel] : 0.0f;
  wave_lds_fence();
}

// The groups that stay where fp32 sums leave it open: those certainly in or
// out keep their place (for each, all of the others or enough of them are
// certainly on the other side of it), and the rest are ranked by the sums of
// their members that may count, in 64 bits.  False where a softmax's
// denominator beside biases, which stays that of the fp32 sums, is not known
// well enough for it.
template <class T16, int C, int TW>
__device__ bool settle_groups(const RouterParams& p, const T16* xr, Token<C>& tk, OpenLds<C>& lds) {
  const int lane = threadIdx.x & 63;
  const int per = lanes_per_group(p), g = lane / per;
  const bool biased = p.bias != nullptr, soft = p.score == SCORE_SOFTMAX;
  const double none = -__builtin_inf();
  const float room = 2.0f * group_margin(tk);
  const bool near = contested(p, tk, room);
  const uint64_t cm = __ballot(near), sure = __ballot(tk.stays && !near);
  const int left = p.top_groups - __popcll(sure) / per;
  bool want[C], again[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = min(group_of(p, c * 64 + lane) * per, 63);
    const float low = __shfl(tk.group.low, at, 64);
    want[c] = tk.fit[c] && (cm >> at & 1) && tk.val[c] >= low - room;
    again[c] = want[c] && tk.err[c] > 0.0f;
  }
  double l[C];
#pragma unroll
  for (int c = 0; c < C; ++c) l[c] = tk.l[c];
  const int n = sum_again<T16, C, TW>(p, xr, again, lds);
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    const int e = __builtin_amdgcn_readfirstlane(lds.list[i]);
    const double v = lds.dots[i];
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (c * 64 + lane == e) l[c] = v;
  }
  float most = 0.0f;   // of the scores that may count
#pragma unroll
  for (int c = 0; c < C; ++c) {
    // (a softmax's denominator is common to all groups without a bias)
    const double sc = soft ? exp(l[c] - tk.top) / tk.z : sigmoid(l[c]);
    if (Team<TW>::lead()) lds.row[c * 64 + lane] = want[c] ? (biased ? sc + tk.b[c] : sc) : none;
    most = fmaxf(most, want[c] ? (float)sc : 0.0f);
  }
  Team<TW>::sync();
  const GroupBest<double> gb = group_best(p, lds.row, lane, per, g);
  int rank = 0;
#pragma unroll 1
  for (int h = 0; h < p.n_groups; ++h) {
    if (!(cm >> (h * per) & 1)) continue;
    const double v = lane_value(gb.sum, h * per);
    rank += v > gb.sum || (v == gb.sum && h < g);
  }
  tk.stays = (sure >> lane & 1) || (near && rank < left);
  keep_groups(p, tk);
  Team<TW>::sync();
  if (!soft || !biased) return true;
  // (scores of two groups differ by less than they come to)
  const double in = -wave_max(near && tk.stays ? -gb.sum : none);
  const double out = wave_max(near && !tk.stays ? gb.sum : none);
  return in - out > 1.01 * tk.zrel * p.group_best * wave_max(most);
}

// The order of the slots where only neighbours of it are open: the experts
// within the margin of a slot's key are summed again, and those and the other
// slots ranked anew, a lane each.  Every expert outside is certainly below
// all slots.  False where this does not decide: too many experts, or a
// softmax's denominator that is not known well enough.
template <class T16, int C, int TW>
__device__ bool select_slots(const RouterParams& p, const T16* xr, Token<C>& tk, OpenLds<C>& lds) {
  const int lane = threadIdx.x & 63;
  const bool biased = p.bias != nullptr, soft = p.score == SCORE_SOFTMAX;
  bool want[C], slot[C];
#pragma unroll
  for (int c = 0; c < C; ++c) want[c] = slot[c] = false;
  for (int k = 0; k < p.K; ++k) {
    const int e = __builtin_amdgcn_readlane(tk.sel, k);
    if (e < 0) break;
    float ke = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (e >> 6 == c) ke = lane_value(tk.key[c], e & 63);
    uint64_t near = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const bool self = c * 64 + lane == e;
      const bool n = tk.kept[c] && !self && fabsf(tk.key[c] - ke) <= tk.margin;
      want[c] |= n;
      slot[c] |= self;
      near |= __ballot(n);
    }
    if (near) {
#pragma unroll
      for (int c = 0; c < C; ++c) want[c] |= c * 64 + lane == e;
    }
  }
  int n = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) n += __popcll(__ballot(want[c] || slot[c]));
  if (n > 32) return false;
  bool again[C];
#pragma unroll
  for (int c = 0; c < C; ++c) again[c] = want[c] && tk.err[c] > 0.0f;
  // lane u: member u, its logit and bias
  int me = -1, at = 0;
  double ml = 0.0;
  float mb = 0.0f;
  const auto add = [&](int c, int j, double v) {
    float bj = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i)
      if (i == c) bj = lane_value(tk.b[i], j);
    if (lane == at) {
      me = c * 64 + j;
      ml = v;
      mb = bj;
    }
    ++at;
  };
#pragma unroll
  for (int c = 0; c < C; ++c) {
    uint64_t m = __ballot((slot[c] || want[c]) && !again[c]);
    for (; m; m &= m - 1) {
      const int j = __ffsll((unsigned long long)m) - 1;
      add(c, j, lane_value(tk.l[c], j));
    }
  }
  const int summed = sum_again<T16, C, TW>(p, xr, again, lds);
#pragma unroll 1
  for (int i = 0; i < summed; ++i) {
    const int e = __builtin_amdgcn_readfirstlane(lds.list[i]);
    add(e >> 6, e & 63, lds.dots[i]);
  }
  Team<TW>::sync();
  double s = 0.0, k = ml;
  if (biased) {
    s = soft ? exp(ml - tk.top) / tk.z : sigmoid(ml);
    k = s + mb;
  }
  const bool in = lane < n;
  int rank = 0;
  bool unsure = false;
#pragma unroll 1
  for (int u = 0; u < n; ++u) {
    const double ku = lane_value(k, u), su = lane_value(s, u);
    const int eu = __builtin_amdgcn_readlane(me, u);
    rank += ku > k || (ku == k && eu < me);
    unsure |= soft && biased && u != lane && fabs(ku - k) <= 1.01 * tk.zrel * fabs(su - s);
  }
  if (__ballot(in && unsure)) return false;
  const int K = min(p.K, n);
  tk.sel = -1;
  for (int r = 0; r < K; ++r) {
    const int u = __ffsll((unsigned long long)__ballot(in && rank == r)) - 1;
    const int e = __builtin_amdgcn_readlane(me, u);
    const float v = (float)lane_value(ml, u);
    if (lane == r) {
      tk.sel = e;
      tk.sl = v;
    }
  }
  return true;
}

// Weights and outputs of token t from its selection, by one wave.  counts: the
// block's, in LDS.
template <int C>
__device__ inline void finish(const RouterParams& p, int t, const Token<C>& tk, const RouterOut& o,
                              int32_t* counts) {
  const int lane = threadIdx.x & 63;
  const float none = -__builtin_inff();
  const bool soft = p.score == SCORE_SOFTMAX;
  // The weights are those of the logits' fp32 sums (of the 64-bit ones where
  // the token was open), whose error is theirs: 9e-8 on average at 1337 tokens x
  // 60 experts, d 2048, the denominator's fast exponential among it.
  // Shares of the selected scores, so that scores that underflow still have
  // their ratios.
  const int sel = tk.sel;
  const bool have = sel >= 0;
  const float lm = wave_max(have ? tk.sl : none);  // (by every lane of the wave)
  float ex = 0.0f;
  if (soft || lm < -60.0f) {
    // (the logarithm of a sigmoid that far out is its logit to all bits)
    ex = have ? expf(tk.sl - lm) : 0.0f;
  } else {
    ex = have ? 1.0f / (1.0f + expf(-tk.sl)) : 0.0f;
  }
  const float sum = wave_sum_dpp(ex);
  const float share = have ? ex / sum : 0.0f;
  float w = share;
  if (!p.renorm) w = !have ? 0.0f : soft ? ex * expf(lm - tk.top) / tk.z : 1.0f / (1.0f + expf(-tk.sl));
  w *= p.scale;
  // Eq. 2 over the shares: the score of a slot is the sum of those above it
  int prec = PREC_SKIP;
  if (o.table) {
    float above = 0.0f;
    bool first = true;
    for (int j = 0; j < p.K; ++j) {
      const float sj = lane_value(share, j);
      if (sj > share || (sj == share && j < lane)) {
        above += sj;
        first = false;
      }
    }
    if (have) {
      const int tag = o.table[sel].tag;
      if (tag == TAG_FP16 || tag == TAG_INT8) prec = PREC_HIGH;
      else if (tag == TAG_INT4 || tag == TAG_INT2) prec = PREC_LOW;
      else prec = first || above <= o.t1 ? PREC_HIGH : above <= o.t2 ? PREC_LOW : PREC_SKIP;
    }
  }
  if (lane < p.K) {
    const int64_t i = (int64_t)t * p.K + lane;
    o.idx[i] = sel;
    o.w[i] = w;
    if (o.prec) o.prec[i] = (int8_t)prec;
    if (o.user_idx) o.user_idx[i] = sel;
    if (o.user_w) o.user_w[i] = w;
    if (o.user_prec) o.user_prec[i] = (int8_t)prec;
    if (o.count && have) atomicAdd(&counts[sel], 1);
  }
}

// Selection of a token whose logits are loaded.
template <class T16, int C, int TW>
__device__ inline void select_token(const RouterParams& p, const T16* xr, float* row, Token<C>& tk,
                                    OpenLds<C>& lds) {
  score_token(p, row, tk);
  bool open = tk.vague;
  if (!open && tk.groups_open) open = !settle_groups<T16, C, TW>(p, xr, tk, lds);
  if (!open) {
    take_slots(p, row, tk);
    if (tk.slots_open) open = !select_slots<T16, C, TW>(p, xr, tk, lds);
  }
  if (open) select_all<T16, C, TW>(p, xr, tk, lds);
}

// The block's counts into the call's, by neighbouring lanes: one request per
// line.  (An atomic per slot on these few lines took 21 us for 1337 tokens of
// 4 slots.)
__device__ inline void add_counts(const RouterParams& p, const RouterOut& o, const int32_t* counts) {
  if (!o.count) return;
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += blockDim.x)
    if (counts[e]) atomicAdd(o.count + e, counts[e]);
}

// Many tokens: one per wave in turn; those that fp32 leaves open go on a list.
// Few blocks of many waves, so that few of them add to the counts.  Bound by
// the issue of about 1100 vector instructions per token: 8192 tokens x 256
// experts in groups 23.6 us.
constexpr int kManyThreads = 1024;
constexpr int kManyWaves = kManyThreads / 64;
constexpr int kManyBlocks = 256;
template <int C>
__global__ __launch_bounds__(kManyThreads) void router_select_many_kernel(RouterParams p, int T,
                                                                          const float* __restrict__ lg,
                                                                          RouterOut o) {
  __shared__ float rows[kManyWaves][C * 64];
  __shared__ int32_t counts[C * 64];
  __shared__ int32_t n_open, first_open, opens[kManyThreads];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (threadIdx.x == 0) n_open = 0;
  if (o.count)
    for (int e = threadIdx.x; e < C * 64; e += kManyThreads) counts[e] = 0;
  __syncthreads();
  // (at most 65536 / (16 * 256) = 16 tokens a wave, one slot of opens each)
  for (int t = blockIdx.x * kManyWaves + wave; t < T; t += gridDim.x * kManyWaves) {
    Token<C> tk;
    load_token(p, global<float>(lg + (int64_t)t * p.E), global<float>(p.w_norm), global<float>(p.x_norm)[t], tk);
    score_token(p, rows[wave], tk);
    take_slots(p, rows[wave], tk);
    if (!tk.vague && !tk.groups_open && !tk.slots_open) finish(p, t, tk, o, counts);
    else if ((threadIdx.x & 63) == 0) opens[atomicAdd(&n_open, 1)] = t;
  }
  __syncthreads();
  if (threadIdx.x == 0 && n_open) first_open = atomicAdd(p.open, n_open);
  __syncthreads();
  if ((int)threadIdx.x < n_open) p.open[1 + first_open + threadIdx.x] = opens[threadIdx.x];
  add_counts(p, o, counts);
}

// Tokens of a call or of the list, a team of TW waves each.  Bound by its
// longest chain, an open token's: scores, then two or three rounds of sums in
// 64 bits of a microsecond or two (32 tokens x 256 experts in groups 9 to 16 us,
// as the inputs leave some open, the list of 8192 20 us).
constexpr int team_threads(int tw) { return tw < 4 ? 256 : tw * 64; }
template <class T16, int C, int TW>
__global__ __launch_bounds__(team_threads(TW)) void router_select_kernel(RouterParams p, int T, int listed,
                                                                     const T16* __restrict__ x,
                                                                     const float* __restrict__ lg,
                                                                     RouterOut o) {
  constexpr int kThreads = team_threads(TW), kTeams = kThreads / 64 / TW;
  __shared__ float rows[kThreads / 64][C * 64];
  __shared__ OpenLds<C> lds[kTeams];
  __shared__ int32_t counts[C * 64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / TW;
  const int n = listed ? __builtin_amdgcn_readfirstlane(global<int32_t>(p.open)[0]) : T;
  if ((int)blockIdx.x * kTeams >= n) return;
  if (o.count) {
    for (int e = threadIdx.x; e < C * 64; e += kThreads) counts[e] = 0;
    __syncthreads();
  }
#pragma unroll 1
  for (int i = blockIdx.x * kTeams + team; i < n; i += gridDim.x * kTeams) {
    const int t = listed ? __builtin_amdgcn_readfirstlane(global<int32_t>(p.open)[1 + i]) : i;
    Token<C> tk;
    load_token(p, global<float>(lg + (int64_t)t * p.E), global<float>(p.w_norm), global<float>(p.x_norm)[t], tk);
    select_token<T16, C, TW>(p, x + (int64_t)t * p.d, rows[wave], tk, lds[team]);
    if (TW == 1 || Team<TW>::lead()) finish(p, t, tk, o, counts);
  }
  add_counts(p, o, counts);
}

// ---- logits ---------------------------------------------------------------

// Logits [T, E] of MT * 16 tokens and NT * 16 experts per block.  Every wave
// takes its share of the columns for the whole tile, 64 columns (a line of
// 128 bytes of each row) at a time, so that each byte is loaded once per
// block and no wave waits for another; the waves' sums are joined in LDS in a
// fixed order.  A piece is loaded into registers while the last one is
// multiplied.
//
// What bounds it is the load path of a compute unit.  Loads in the layout
// that the matrix products take put neighbouring lanes on different rows and
// reach 15 bytes a cycle per unit, from L2 as from HBM; eight lanes along a
// line reach 47 (256 units, 16-byte loads, 2 MiB that stay in L2).  So a
// piece is loaded by lines, 8 rows an instruction, and turned through LDS of
// the wave's own: 16-byte chunk k of a row r lies at slot k ^ (r & 7), where
// neither the writes nor the products' reads conflict.
// Rows past the end are read as the last one and not written.
//
// kSelect: the block has all experts of its tokens and selects as well, a wave
// per token (lg: the caller's or null; the counts are cleared beforehand).
template <class T16, int MT, int NT, int NW, bool kSelect>
__global__ __launch_bounds__(NW * 64, 8 / NW) void router_logits_kernel(RouterParams p, int T,
                                                                const T16* __restrict__ x,
                                                                float* __restrict__ lg,
                                                                RouterOut o) {
  typedef typename Vec<T16>::x8 x8;
  constexpr int BM = MT * 16, BN = NT * 16, LD = BN + 4;
  constexpr int LA = 2 * MT, LB = 2 * NT;           // loads of a piece: 8 rows each
  constexpr int kPiece = (LA + LB) * 64;            // 16-byte slots of a piece
  constexpr int kRed = NW * BM * LD / 4;            // ... of the waves' sums
  __shared__ u32x4 lds[kRed > NW * kPiece ? kRed : NW * kPiece];
  __shared__ float sq[NW][BM + BN];
  __shared__ uint32_t nz[NW][BM + BN];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = blockIdx.z * gridDim.x + blockIdx.x;
  const int t0 = tile * BM, e0 = blockIdx.y * BN;
  if (t0 >= T) return;
  const bool norm_x = blockIdx.y == 0, norm_w = kSelect || tile == 0;
  if (!kSelect && tile == 0 && blockIdx.y == 0) {  // what the selection adds to
    if (threadIdx.x == 0) p.open[0] = 0;
    if (o.count)
      for (int e = threadIdx.x; e < p.E; e += NW * 64) o.count[e] = 0;
  }
  // this lane's chunks as offsets in bytes from the block's first row (a tile
  // has at most 128 rows of 32 KiB), so that loads take one uniform address
  Global<char> xb = global<char>(x + (int64_t)t0 * p.d);
  Global<char> wb = global<char>(static_cast<const T16*>(p.wg) + (int64_t)e0 * p.d);
  uint32_t xo[LA], wo[LB];
  const int r8 = lane >> 3, chunk = ((lane & 7) ^ r8) * 16;
#pragma unroll
  for (int j = 0; j < LA; ++j) xo[j] = (uint32_t)min(j * 8 + r8, T - 1 - t0) * (uint32_t)(p.d * 2) + chunk;
#pragma unroll
  for (int j = 0; j < LB; ++j) wo[j] = (uint32_t)min(j * 8 + r8, p.E - 1 - e0) * (uint32_t)(p.d * 2) + chunk;
  f32x4 acc[MT][NT];
  float sx[LA], sw[LB], px[LA], pw[LB];   // squares so far, and their sum over the steps
  uint32_t some = 0;   // a bit for each of this lane's rows that is not all zeros
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < LA; ++j) {
    sx[j] = px[j] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j < LB; ++j) {
    sw[j] = pw[j] = 0.0f;
  }
  const int n = (p.d / 64 - wave + NW - 1) / NW;  // this wave's pieces
  u32x4 a[LA], b[LB];
  auto load = [&](int i) {
    const int c = (wave + min(i, n - 1) * NW) * 128;  // (past the last: the last again)
#pragma unroll
    for (int j = 0; j < LA; ++j) a[j] = *(Global<u32x4>)(xb + c + xo[j]);
#pragma unroll
    for (int j = 0; j < LB; ++j) b[j] = *(Global<u32x4>)(wb + c + wo[j]);
  };
  u32x4* own = lds + wave * kPiece;
  const int row = lane & 15, at0 = row * 8 + ((lane >> 4) ^ (row & 7)), at1 = at0 ^ 4;
  if (n > 0) load(0);
  for (int i = 0; i < n; ++i) {
#pragma unroll
    for (int j = 0; j < LA; ++j) own[j * 64 + lane] = a[j];
#pragma unroll
    for (int j = 0; j < LB; ++j) own[(LA + j) * 64 + lane] = b[j];
    if (norm_x) {
#pragma unroll
      for (int j = 0; j < LA; ++j) {
        // (a row's squares lie in eight lanes: the sums of both are joined below)
        sx[j] = squares(__builtin_bit_cast(x8, a[j]), sx[j]);
        px[j] += sx[j];
        some |= any_bits(a[j]) ? 1u << j : 0u;
      }
    }
    if (norm_w) {
#pragma unroll
      for (int j = 0; j < LB; ++j) {
        sw[j] = squares(__builtin_bit_cast(x8, b[j]), sw[j]);
        pw[j] += sw[j];
        some |= any_bits(b[j]) ? 1u << (LA + j) : 0u;
      }
    }
    load(i + 1);
    wave_lds_order();
    __builtin_amdgcn_sched_barrier(0);
    // the piece's sums from zero (see the error of a logit), a row of tiles at
    // a time: registers
    x8 bf[2][NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      bf[0][j] = __builtin_bit_cast(x8, own[(MT + j) * 128 + at0]);
      bf[1][j] = __builtin_bit_cast(x8, own[(MT + j) * 128 + at1]);
    }
#pragma unroll
    for (int k = 0; k < MT; ++k) {
      const x8 a0 = __builtin_bit_cast(x8, own[k * 128 + at0]), a1 = __builtin_bit_cast(x8, own[k * 128 + at1]);
      f32x4 sum[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) sum[j] = mfma(a0, bf[0][j], f32x4{0, 0, 0, 0});
#pragma unroll
      for (int j = 0; j < NT; ++j) sum[j] = mfma(a1, bf[1][j], sum[j]);
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[k][j] += sum[j];
    }
    wave_lds_order();   // (the next piece is written over this one)
  }
  __syncthreads();
  float* red = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        red[(wave * BM + i * 16 + (lane >> 4) * 4 + r) * LD + j * 16 + row] = acc[i][j][r];
  // q^2 of the columns of this lane, the group k of every piece: a piece's
  // squares count in its groups from the k-th on, in it and in all later pieces
  const float k8 = (float)((lane & 7) ^ r8);
  auto squares_up_to = [&](float p, float s) { return 1.01f * (p + (8.0f - k8) * s) + (NW + 7) * s; };
  // a row's squares lie in eight neighbouring lanes
  auto put = [&](float s, uint32_t z, int at) {
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) {
      s += __shfl_xor(s, m, 64);
      z |= __shfl_xor(z, m, 64);
    }
    if ((lane & 7) == 0) {
      sq[wave][at + r8] = s;
      nz[wave][at + r8] = z;
    }
  };
  if (norm_x) {
#pragma unroll
    for (int j = 0; j < LA; ++j) put(squares_up_to(px[j], sx[j]), some >> j & 1, j * 8);
  }
  if (norm_w) {
#pragma unroll
    for (int j = 0; j < LB; ++j) put(squares_up_to(pw[j], sw[j]), some >> (LA + j) & 1, BM + j * 8);
  }
  __syncthreads();
  for (int v = threadIdx.x; v < BM * BN; v += NW * 64) {
    const int m = v / BN, c = v % BN;
    float s = red[m * LD + c];
#pragma unroll
    for (int w = 1; w < NW; ++w) s += red[(w * BM + m) * LD + c];
    const bool in = t0 + m < T && e0 + c < p.E;
    if (in && lg) lg[(int64_t)(t0 + m) * p.E + e0 + c] = s;
    if (kSelect) red[m * LD + c] = s;   // (over the first wave's sum, which only this thread reads)
  }
  __shared__ float bounds[BM + BN];
  for (int v = threadIdx.x; v < BM + BN; v += NW * 64) {
    if (v < BM ? !norm_x : !norm_w) continue;
    float s = 0.0f;
    uint32_t z = 0;
    for (int w = 0; w < NW; ++w) {
      s += sq[w][v];
      z |= nz[w][v];
    }
    const float bound = error_norm<T16>(s, z != 0, p.d);
    if (kSelect) bounds[v] = bound;
    else if (v < BM && t0 + v < T) p.x_norm[t0 + v] = bound;
    else if (v >= BM && e0 + v - BM < p.E) p.w_norm[e0 + v - BM] = bound;
  }
  if constexpr (kSelect) {
    static_assert(BN <= 64, "a lane per expert");
    __shared__ float rows[NW][64];
    __shared__ OpenLds<1> open[NW];
    __shared__ int32_t counts[64];
    if (o.count && threadIdx.x < 64) counts[threadIdx.x] = 0;
    __syncthreads();
    for (int m = wave; m < BM && t0 + m < T; m += NW) {
      Token<1> tk;
      const bool in = lane < p.E;
      tk.l[0] = in ? red[m * LD + lane] : -__builtin_inff();
      tk.b[0] = in && p.bias ? global<float>(p.bias)[lane] : 0.0f;
      tk.err[0] = in ? logit_error(bounds[m], bounds[BM + lane]) : 0.0f;
      select_token<T16, 1, 1>(p, x + (int64_t)(t0 + m) * p.d, rows[wave], tk, open[wave]);
      finish(p, t0 + m, tk, o, counts);
    }
    add_counts(p, o, counts);
  }
}

// Counts of a call whose first kernel already adds to them.
__global__ void router_clear_kernel(int32_t* count, int E) {
  for (int e = threadIdx.x; e < E; e += blockDim.x) count[e] = 0;
}

template <class T16, int MT, int NT, int NW>
hipError_t logits(const RouterParams& p, int T, const T16* x, float* lg, const RouterOut& o, hipStream_t s) {
  // blocks go to the eight dies in turn: those of one tile of tokens to the same
  // die, one right after another, which then finds the tokens in its L2 (us at
  // d 4096, against all tiles of tokens for one of experts after another: 16000
  // x 256 69 86, 3000 x 256 21.3 25.0, 8192 x 512 63 67, 8192 x 256 35.0 35.2)
  const int tiles = (T + MT * 16 - 1) / (MT * 16), dies = tiles < 8 ? tiles : 8;
  const dim3 grid(dies, (p.E + NT * 16 - 1) / (NT * 16), (tiles + dies - 1) / dies);
  router_logits_kernel<T16, MT, NT, NW, false><<<grid, NW * 64, 0, s>>>(p, T, x, lg, o);
  return hipGetLastError();
}

template <class T16, int C>
hipError_t select(const RouterParams& p, int T, const T16* x, const float* lg, const RouterOut& o,
                  hipStream_t s) {
  // Up to 2048 tokens a wave each, which sums again what is open in its own;
  // more by the kernel that leaves open tokens to a list, with a block of four
  // waves each.  us at d 4096 with the experts' counts, 60 experts / 256 in 8
  // groups / 512 in 8 groups, a wave each against the list: 256 tokens 5.5 8.2 /
  // 17.1 30.8 / 24.7 47.9, 1024 9.8 16.4 / 18.2 32.5 / 25.0 48.5, 2048 16.3 18.2
  // / 24.5 32.2 / 28.1 48.2, 4096 27.8 20.4 / 35.3 35.0 / 48.5 49.0, 8192 45.2
  // 23.1 / 52.2 47.6 / 74.6 64.0.  Without the counts, to which many blocks add,
  // a wave each is up to a tenth faster still at 8192 tokens x 256 (36.8 40.5).
  // A softmax beside a bias may need all of a token's logits in 64 bits, for
  // its denominator (45 us of one block at 256 experts): a block of eight
  // waves each, for all tokens or those on the list: 64 tokens 17.6 29.5, 256
  // 18.0 29.8, 512 30.2 30.2, 1024 45.0 30.8, 2048 75.1 31.5 (where none needs
  // all; with one that does 98 and 85), 8192 282 131.
  const bool wide = p.bias && p.score == SCORE_SOFTMAX;
  constexpr int kWideEach = 512, kWaveEach = 2048, kListBlocks = 768;
  // (one expert per lane leaves those kernels with scratch memory that they
  // never touch)
  constexpr int W = C < 2 ? 2 : C;
  if (wide && T <= kWideEach) {
    router_select_kernel<T16, W, 8><<<T, team_threads(8), 0, s>>>(p, T, 0, x, lg, o);
  } else if (!wide && T <= kWaveEach) {
    router_select_kernel<T16, C, 1><<<(T + 3) / 4, team_threads(1), 0, s>>>(p, T, 0, x, lg, o);
  } else {
    const int blocks = (T + kManyWaves - 1) / kManyWaves;
    router_select_many_kernel<C><<<blocks < kManyBlocks ? blocks : kManyBlocks, kManyThreads, 0, s>>>(p, T, lg, o);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (wide) router_select_kernel<T16, W, 8><<<kListBlocks, team_threads(8), 0, s>>>(p, T, 1, x, lg, o);
    else router_select_kernel<T16, W, 4><<<kListBlocks, team_threads(4), 0, s>>>(p, T, 1, x, lg, o);
  }
  return hipGetLastError();
}

template <class T16>
hipError_t run(const RouterParams& p, int T, const T16* x, const RouterOut& o, hipStream_t s) {
  if (p.E <= 16) {
    // all experts in one tile: one kernel
    if (o.count) {
      router_clear_kernel<<<1, 64, 0, s>>>(o.count, p.E);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    router_logits_kernel<T16, 1, 1, 8, true><<<(T + 15) / 16, 512, 0, s>>>(p, T, x, o.logits, o);
    return hipGetLastError();
  }
  float* lg = o.logits ? o.logits : p.logits;
  // The tile of which the busiest compute unit loads the fewest rows: a block
  // loads tokens + experts of them, and there are 256 units.  us at d 4096, 256
  // experts, tiles of 64x64 / 64x32 / 32x32 / 16x32 / 16x16 on eight waves:
  // 4096 tokens 23.4 27.8 29.8 37.4 45.6, 2048 21.4 16.0 17.6 22.3 26.7, 1024
  // 21.1 15.4 11.6 13.6 16.2, 512 21.0 14.8 10.5 8.4 10.1, 64 20.7 14.2 10.0 7.6
  // 6.0.  Two blocks of 64x64 fit a unit on four waves each, which is faster
  // where there are so many: 8192 tokens 34.8, on eight waves 40.3.
  constexpr int kTiles[5][2] = {{16, 16}, {16, 32}, {32, 32}, {64, 32}, {64, 64}};
  int tile = 0;
  int64_t least = 0, blocks = 0;
  for (int i = 0; i < 5; ++i) {
    const int m = kTiles[i][0], n = kTiles[i][1];
    const int64_t all = (int64_t)((T + m - 1) / m) * ((p.E + n - 1) / n), rows = (all + 255) / 256 * (m + n);
    if (i == 0 || rows < least) {
      tile = i;
      least = rows;
      blocks = all;
    }
  }
  hipError_t e;
  if (tile == 0) e = logits<T16, 1, 1, 8>(p, T, x, lg, o, s);
  else if (tile == 1) e = logits<T16, 1, 2, 8>(p, T, x, lg, o, s);
  else if (tile == 2) e = logits<T16, 2, 2, 8>(p, T, x, lg, o, s);
  else if (tile == 3) e = logits<T16, 4, 2, 8>(p, T, x, lg, o, s);
  else if (blocks <= 256) e = logits<T16, 4, 4, 8>(p, T, x, lg, o, s);
  else e = logits<T16, 4, 4, 4>(p, T, x, lg, o, s);
  if (e != hipSuccess) return e;
  if (p.E <= 64) return select<T16, 1>(p, T, x, lg, o, s);
  if (p.E <= 128) return select<T16, 2>(p, T, x, lg, o, s);
  if (p.E <= 256) return select<T16, 4>(p, T, x, lg, o, s);
  return select<T16, 8>(p, T, x, lg, o, s);
}

}  // namespace

hipError_t launch_router(const RouterParams& p, int T, const void* x, const RouterOut& o,
                         hipStream_t s) {
  return p.type == TYPE_F16 ? run(p, T, static_cast<const f16*>(x), o, s)
                            : run(p, T, static_cast<const bf16*>(x), o, s);
}

}  // namespace moe
