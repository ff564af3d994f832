// Routing rules: scores of the gate's logits, a bias that steers the balance,
// groups of experts, top-k and the weights.
//
//   l = x Wg^T;  s = sigmoid(l) or softmax(l);  key = s + b, or l without a b
//   group score = sum of the group's one or two best keys (scores without b)
//   top-k of the keys in the groups that count most, ties to the lower index
//   w = scale s, or scale s / sum of the selected s
//
// Which of two near keys is larger decides what is selected, so logits, keys
// and group scores are held in 64 bits.
#include "moe_internal.h"

namespace moe {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ inline double shfl_xor(double v, int m) { return __shfl_xor(v, m, 64); }
__device__ inline double wave_sum(double v) {
  for (int m = 1; m < 64; m <<= 1) v += shfl_xor(v, m);
  return v;
}
__device__ inline double wave_max(double v) {
  for (int m = 1; m < 64; m <<= 1) v = fmax(v, shfl_xor(v, m));
  return v;
}
__device__ inline bool finite(double v) { return fabs(v) <= 1.7976931348623157e308; }

// x . w over d columns by one wave, in 64 bits (a product of two 16-bit
// numbers is exact there).  Every lane gets the sum.
template <class T16>
__device__ inline double exact_dot(const T16* x, const T16* w, int d) {
  typedef T16 x8 __attribute__((ext_vector_type(8)));
  double s = 0.0;
  for (int c = (threadIdx.x & 63) * 8; c < d; c += 512) {
    const x8 a = *reinterpret_cast<const x8*>(x + c), b = *reinterpret_cast<const x8*>(w + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fma((double)(float)a[j], (double)(float)b[j], s);
  }
  return wave_sum(s);
}

// One wave per (token, expert).
template <class T16>
__global__ __launch_bounds__(kThreads) void router_logits_kernel(RouterParams p, int T,
                                                                 const T16* __restrict__ x,
                                                                 RouterOut o) {
  const int64_t i = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (o.count && blockIdx.x == 0)
    for (int e = threadIdx.x; e < p.E; e += kThreads) o.count[e] = 0;
  if (i >= (int64_t)T * p.E) return;
  const int t = (int)(i / p.E), e = (int)(i - (int64_t)t * p.E);
  const double l = exact_dot(x + (int64_t)t * p.d, static_cast<const T16*>(p.wg) + (int64_t)e * p.d, p.d);
  if ((threadIdx.x & 63) == 0) {
    p.logits[i] = l;
    if (o.logits) o.logits[i] = (float)l;
  }
}

// log sigmoid(l) without overflow or loss far from 0
__device__ inline double log_sigmoid(double l) { return fmin(l, 0.0) - log1p(exp(-fabs(l))); }

// Selection and weights of one token by one wave; lane i holds the experts
// i, i + 64, ... (C of them).
template <int C>
__global__ __launch_bounds__(kThreads) void router_select_kernel(RouterParams p, int T, RouterOut o) {
  __shared__ double rows[kWaves][C * 64];
  __shared__ double groups[kWaves][kRouterMaxGroups];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * kWaves + wave;
  const bool on = t < T;
  const double none = -__builtin_inf();
  double l[C], key[C];
  bool fit[C];   // can be selected
  double top = none;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int e = c * 64 + lane;
    l[c] = on && e < p.E ? p.logits[(int64_t)t * p.E + e] : none;
    fit[c] = finite(l[c]);
    if (fit[c]) top = fmax(top, l[c]);
  }
  double score[C];
  if (p.score == SCORE_SIGMOID) {
#pragma unroll
    for (int c = 0; c < C; ++c) score[c] = fit[c] ? 1.0 / (1.0 + exp(-l[c])) : 0.0;
  } else {
    top = wave_max(top);
    double z = 0.0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      score[c] = fit[c] ? exp(l[c] - top) : 0.0;
      z += score[c];
    }
    z = wave_sum(z);
#pragma unroll
    for (int c = 0; c < C; ++c) score[c] = fit[c] ? score[c] / z : 0.0;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int e = c * 64 + lane;
    key[c] = l[c];
    if (p.bias && e < p.E) {
      const float b = p.bias[e];
      fit[c] = fit[c] && finite(b);
      key[c] = score[c] + b;
    }
  }
  if (p.n_groups > 1) {
    // lane g scans the members of group g
    const int size = p.E / p.n_groups;
#pragma unroll
    for (int c = 0; c < C; ++c) rows[wave][c * 64 + lane] = fit[c] ? (p.bias ? key[c] : score[c]) : none;
    __syncthreads();
    double best = none, second = none;
    if (lane < p.n_groups)
      for (int i = 0; i < size; ++i) {
        const double v = rows[wave][lane * size + i];
        if (v > best) {
          second = best;
          best = v;
        } else {
          second = fmax(second, v);
        }
      }
    const double sum = p.group_best == 2 && second > none ? best + second : best;
    groups[wave][lane] = sum;
    __syncthreads();
    int rank = 0;
    for (int g = 0; g < p.n_groups; ++g) {
      const double v = groups[wave][g];
      rank += v > sum || (v == sum && g < lane);
    }
    const uint64_t kept = __ballot(lane < p.n_groups && rank < p.top_groups);
#pragma unroll
    for (int c = 0; c < C; ++c) fit[c] = fit[c] && (kept >> ((c * 64 + lane) / size) & 1);
  }
  // top-k: lane k keeps slot k
  int sel = -1;
  double sl = 0.0;
  for (int k = 0; k < p.K; ++k) {
    double bk = none;
    int be = 1 << 30;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (fit[c] && (be == 1 << 30 || key[c] > bk)) {
        bk = key[c];
        be = c * 64 + lane;
      }
    for (int m = 1; m < 64; m <<= 1) {
      const double ok = shfl_xor(bk, m);
      const int oe = __shfl_xor(be, m, 64);
      if (ok > bk || (ok == bk && oe < be)) {
        bk = ok;
        be = oe;
      }
    }
    if (be == 1 << 30) break;  // nobody left (uniform)
    double mine = 0.0;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (c * 64 + lane == be) {
        fit[c] = false;
        mine = l[c];
      }
    mine = __shfl(mine, be & 63, 64);
    if (lane == k) {
      sel = be;
      sl = mine;
    }
  }
  // weights: the share of the selected scores by their logarithms, so that
  // scores that underflow still have their ratios
  const bool have = sel >= 0;
  const double ls = !have ? none : p.score == SCORE_SIGMOID ? log_sigmoid(sl) : sl;
  const double lm = wave_max(ls);
  const double ex = have ? exp(ls - lm) : 0.0;
  const double sum = wave_sum(ex);
  const float share = have ? (float)(ex / sum) : 0.0f;
  float w = share;
  if (!p.renorm) {
    if (p.score == SCORE_SIGMOID) {
      w = have ? (float)exp(ls) : 0.0f;
    } else {
      double z = 0.0;
#pragma unroll
      for (int c = 0; c < C; ++c) z += finite(l[c]) ? exp(l[c] - top) : 0.0;
      z = wave_sum(z);
      w = have ? (float)(exp(sl - top) / z) : 0.0f;
    }
  }
  w *= p.scale;
  // Eq. 2 over the shares: the score of a slot is the sum of those above it
  int prec = PREC_SKIP;
  if (o.table) {
    float above = 0.0f;
    bool first = true;
    for (int j = 0; j < p.K; ++j) {
      const float sj = __shfl(share, j, 64);
      if (sj > share || (sj == share && j < lane)) {
        above += sj;
        first = false;
      }
    }
    if (have && on && lane < p.K) {
      const int tag = o.table[sel].tag;
      if (tag == TAG_FP16 || tag == TAG_INT8) prec = PREC_HIGH;
      else if (tag == TAG_INT4 || tag == TAG_INT2) prec = PREC_LOW;
      else prec = first || above <= o.t1 ? PREC_HIGH : above <= o.t2 ? PREC_LOW : PREC_SKIP;
    }
  }
  if (on && lane < p.K) {
    const int64_t i = (int64_t)t * p.K + lane;
    if (o.idx) o.idx[i] = sel;
    if (o.w) o.w[i] = w;
    if (o.prec) o.prec[i] = (int8_t)prec;
    if (o.user_idx) o.user_idx[i] = sel;
    if (o.user_w) o.user_w[i] = w;
    if (o.user_prec) o.user_prec[i] = (int8_t)prec;
    if (o.count && have) atomicAdd(o.count + sel, 1);
  }
}

template <class T16>
hipError_t run(const RouterParams& p, int T, const T16* x, const RouterOut& o, hipStream_t s) {
  const int64_t items = (int64_t)T * p.E;
  router_logits_kernel<T16><<<(unsigned)((items + kWaves - 1) / kWaves), kThreads, 0, s>>>(p, T, x, o);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int grid = (T + kWaves - 1) / kWaves;
  if (p.E <= 64) router_select_kernel<1><<<grid, kThreads, 0, s>>>(p, T, o);
  else if (p.E <= 128) router_select_kernel<2><<<grid, kThreads, 0, s>>>(p, T, o);
  else if (p.E <= 256) router_select_kernel<4><<<grid, kThreads, 0, s>>>(p, T, o);
  else router_select_kernel<8><<<grid, kThreads, 0, s>>>(p, T, o);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_router(const RouterParams& p, int T, const void* x, const RouterOut& o,
                         hipStream_t s) {
  return p.type == TYPE_F16 ? run(p, T, static_cast<const f16*>(x), o, s)
                            : run(p, T, static_cast<const bf16*>(x), o, s);
}

}  // namespace moe
