// Layer norm of the residual stream and its backward pass.
//
//   n = (h - mean h) r,  r = 1 / sqrt(mean (h - mean h)^2 + eps)
//   x = n gain + bias
//   a = d_x gain;  d_h = r (a - mean a - n mean(a n))
//   d_gain = sum_t d_x n;  d_bias = sum_t d_x
//
// One block per row, which it holds in registers: h is read once.  The
// variance is the mean square of the centred values (no difference of large
// sums).  The first mean is off by some roundings of its size, which is more
// than the spread of a row that lies far from zero; so the mean of the centred
// values is summed beside their squares and taken out of both, and where it is
// not small against the spread the squares are summed again.  All of it in
// fp32; x and d_x are of 16 bits.
//
// Both passes are bound by memory: 8192 rows of 4096 take 37.5 us (5.4 TB/s of
// h read and x written, a 1 GiB copy 5.1) and 60 + 4.7 us backward (5.6 TB/s
// of h, d_x and d_h).  One row is two dependent trips to memory and a launch,
// 3.3 us.
#include "moe_internal.h"

namespace moe {

namespace {

constexpr int kPieces = 4;  // float4 pieces of a row per thread

// Threads of a row's block: the fewest with at most 16 columns each.  us for
// 8192 rows against the next larger block: d 320 5.7 11.2, 1024 10.2 13.1, 2048
// 20.5 24.8, 4096 37.2 39.6, 8192 73.3 82.9; backward d 320 14.3 26.8, 1024
// 19.4 31.1, 2048 37.6 64.7, 4096 61.5 77.0, 8192 109 160.
inline int row_threads(int d) { return d <= 1024 ? 64 : d <= 4096 ? 256 : d <= 8192 ? 512 : 1024; }

template <class T16>
__device__ inline u32x2 pack4(f32x4 v) {
  typedef T16 x2 __attribute__((ext_vector_type(2)));
  const x2 lo = {(T16)v.x, (T16)v.y}, hi = {(T16)v.z, (T16)v.w};
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

template <class T16>
__device__ inline f32x4 unpack4(u32x2 u) {
  typedef T16 x2 __attribute__((ext_vector_type(2)));
  const uint32_t a = u.x, b = u.y;
  const x2 lo = __builtin_bit_cast(x2, a), hi = __builtin_bit_cast(x2, b);
  return f32x4{(float)lo.x, (float)lo.y, (float)hi.x, (float)hi.y};
}

// Sums of N values over the block's NT threads, in every thread, in a fixed
// order.  `red`: N * NT / 64 floats; the caller alternates two of them.
template <int NT, int N>
__device__ inline void block_sums(float (&v)[N], float* red) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum_dpp(v[i]);
  if constexpr (NT > 64) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) red[i * (NT / 64) + wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < NT / 64; ++w) v[i] += red[i * (NT / 64) + w];
    }
  }
}

// Rows are read and written once: they pass the caches by.
template <class V>
__device__ inline V stream_in(const V* p) { return __builtin_nontemporal_load(p); }
template <class V>
__device__ inline void stream_out(V* p, V v) { __builtin_nontemporal_store(v, p); }

__device__ inline float sum4(f32x4 v) { return (v.x + v.y) + (v.z + v.w); }

// Whether a mean `rest` of centred values is too large beside their mean square
// for the variance to be the difference of the two (a NaN is not).
__device__ inline bool centre_again(float rest, float square) { return rest * rest > 0.01f * square; }

template <class T16, int NT>
__global__ __launch_bounds__(NT) void layernorm_kernel(const float* __restrict__ h,
                                                       const float* __restrict__ gain,
                                                       const float* __restrict__ bias,
                                                       T16* __restrict__ x, int d, float eps) {
  __shared__ float red[2][2 * NT / 64];
  const int n4 = d >> 2;
  const f32x4* hr = reinterpret_cast<const f32x4*>(h + (int64_t)blockIdx.x * d);
  f32x4 v[kPieces];
  float s[1] = {0.0f};
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int q = threadIdx.x + i * NT;
    v[i] = q < n4 ? stream_in(hr + q) : f32x4{0, 0, 0, 0};
    s[0] += sum4(v[i]);
  }
  block_sums<NT, 1>(s, red[0]);
  float mean = s[0] / (float)d, var;
  for (bool again = false;; again = true) {
    float m[2] = {0.0f, 0.0f};  // centred values, their squares
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (threadIdx.x + i * NT < n4) {
        v[i] -= mean;
        m[0] += sum4(v[i]);
        m[1] += sum4(v[i] * v[i]);
      }
    block_sums<NT, 2>(m, red[1]);
    mean = m[0] / (float)d;
    var = m[1] / (float)d;
    if (again || !centre_again(mean, var)) break;
    if constexpr (NT > 64) __syncthreads();
  }
  const float r = 1.0f / sqrtf(fmaxf(var - mean * mean, 0.0f) + eps);
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int q = threadIdx.x + i * NT;
    if (q < n4) {
      f32x4 o = (v[i] - mean) * r;
      if (gain) o *= reinterpret_cast<const f32x4*>(gain)[q];
      if (bias) o += reinterpret_cast<const f32x4*>(bias)[q];
      stream_out(reinterpret_cast<u32x2*>(x + (int64_t)blockIdx.x * d + 4 * q), pack4<T16>(o));
    }
  }
}

// Rows blockIdx.x, blockIdx.x + gridDim.x, ...; the block's column sums of
// d_x n and d_x go to part[block][2][d].
template <class T16, int NT>
__global__ __launch_bounds__(NT) void layernorm_backward_kernel(
    const T16* __restrict__ dx, const float* __restrict__ h, const float* __restrict__ gain,
    float* __restrict__ dh, float* __restrict__ part, int T, int d, float eps, int accumulate) {
  __shared__ float red[2][4 * NT / 64];
  const int n4 = d >> 2;
  f32x4 dg[kPieces], db[kPieces], gn[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int q = threadIdx.x + i * NT;
    dg[i] = db[i] = f32x4{0, 0, 0, 0};
    gn[i] = gain && q < n4 ? reinterpret_cast<const f32x4*>(gain)[q] : f32x4{1, 1, 1, 1};
  }
  // a row's loads are on their way during the row before
  f32x4 vn[kPieces];
  u32x2 an[kPieces];
  const auto load = [&](int t) {
    const f32x4* hr = reinterpret_cast<const f32x4*>(h + (int64_t)t * d);
    const u32x2* xr = reinterpret_cast<const u32x2*>(dx + (int64_t)t * d);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int q = threadIdx.x + i * NT;
      vn[i] = q < n4 ? stream_in(hr + q) : f32x4{0, 0, 0, 0};
      an[i] = q < n4 ? stream_in(xr + q) : u32x2{0, 0};
    }
  };
  constexpr bool kAhead = NT < 1024;   // (where registers allow)
  if (kAhead) load(blockIdx.x);
  for (int t = blockIdx.x; t < T; t += gridDim.x) {
    if (!kAhead) load(t);
    f32x4 v[kPieces];
    // d_x, unpacked where it is used.  1024 threads have no registers to keep the
    // numbers in from one use to the next, which `forget` ends.
    u32x2 a[kPieces];
    const auto forget = [&]() {
      if constexpr (NT == 1024) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) asm("" : "+v"(a[i].x), "+v"(a[i].y));
      }
    };
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      v[i] = vn[i];
      a[i] = an[i];
      s[0] += sum4(v[i]);
    }
    if (kAhead && t + (int)gridDim.x < T) load(t + gridDim.x);
    block_sums<NT, 1>(s, red[0]);
    float mean = s[0] / (float)d;
    float m[4];  // squares, a, a n (before the scale r), centred values
    for (bool again = false;; again = true) {
      m[0] = m[1] = m[2] = m[3] = 0.0f;
      forget();
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        if (threadIdx.x + i * NT < n4) {
          v[i] -= mean;
          const f32x4 g = unpack4<T16>(a[i]) * gn[i];
          m[0] += sum4(v[i] * v[i]);
          m[1] += sum4(g);
          m[2] += sum4(g * v[i]);
          m[3] += sum4(v[i]);
        }
      block_sums<NT, 4>(m, red[1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = m[i] / (float)d;
      mean = m[3];
      if (again || !centre_again(mean, m[0])) break;
      if constexpr (NT > 64) __syncthreads();
    }
    const float r = 1.0f / sqrtf(fmaxf(m[0] - mean * mean, 0.0f) + eps);
    const float ma = m[1], mn = (m[2] - mean * m[1]) * r;
    forget();
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int q = threadIdx.x + i * NT;
      if (q < n4) {
        const f32x4 n = (v[i] - mean) * r, u = unpack4<T16>(a[i]);
        db[i] += u;
        dg[i] += u * n;
        f32x4 o = r * (u * gn[i] - ma - n * mn);
        f32x4* to = reinterpret_cast<f32x4*>(dh + (int64_t)t * d) + q;
        if (accumulate) o += *to;
        stream_out(to, o);
      }
    }
    if constexpr (NT > 64) __syncthreads();
  }
  if (part) {
    f32x4* pr = reinterpret_cast<f32x4*>(part + (int64_t)blockIdx.x * 2 * d);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int q = threadIdx.x + i * NT;
      if (q < n4) {
        pr[q] = dg[i];
        pr[n4 + q] = db[i];
      }
    }
  }
}

// Column sums of part[n][2 d] into d_gain and d_bias: a block takes 16 pieces
// of four columns, 16 threads of it every 64th row; the 64 sums
// are added in a fixed order.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void column_sums_kernel(const float* __restrict__ part,
                                                                  int n, int d,
                                                                  float* __restrict__ dg,
                                                                  float* __restrict__ db) {
  __shared__ f32x4 red[64][17];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int q = blockIdx.x * 16 + c, n4 = d >> 2;
  f32x4 s = {0, 0, 0, 0};
#pragma unroll 8
  for (int b = g; b < n; b += 64) s += reinterpret_cast<const f32x4*>(part + (int64_t)b * 2 * d)[q];
  red[g][c] = s;
  __syncthreads();
  // 64 sums in two steps of eight
  if (g < 8) {
    s = red[g * 8][c];
#pragma unroll
    for (int i = 1; i < 8; ++i) s += red[g * 8 + i][c];
    red[g * 8][c] = s;
  }
  __syncthreads();
  if (g == 0) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += red[i * 8][c];
    float* to = q < n4 ? dg : db;
    if (to) reinterpret_cast<f32x4*>(to)[q < n4 ? q : q - n4] = s;
  }
}

// Blocks of the backward pass, as many as are at work at once: each has a row
// of column sums that the second kernel reads.  us of both kernels for 8192 rows
// with half / these / twice as many: d 320 26.6 18.2 19.7, 1024 33.9 24.3 30.0,
// 2048 54.8 41.9 45.4, 4096 66.6 65.7 72.3, 8192 190 115 124.  A call of few rows
// writes a row of sums for each of them: 512 rows with half / these, d 2048 10.7
// 12.6, 4096 14.9 17.8, 8192 21.5 19.5; the rule does not go by that.
int backward_blocks(int T, int d) {
  const int most = d <= 1024 ? 1024 : d <= 4096 ? 512 : 256;
  return T < most ? T : most;
}

template <class T16>
hipError_t norm_forward(const float* h, const float* gain, const float* bias, T16* x, int T, int d,
                        float eps, hipStream_t s) {
  switch (row_threads(d)) {
    case 64: layernorm_kernel<T16, 64><<<T, 64, 0, s>>>(h, gain, bias, x, d, eps); break;
    case 256: layernorm_kernel<T16, 256><<<T, 256, 0, s>>>(h, gain, bias, x, d, eps); break;
    case 512: layernorm_kernel<T16, 512><<<T, 512, 0, s>>>(h, gain, bias, x, d, eps); break;
    default: layernorm_kernel<T16, 1024><<<T, 1024, 0, s>>>(h, gain, bias, x, d, eps);
  }
  return hipGetLastError();
}

template <class T16>
hipError_t norm_backward(const T16* dx, const float* h, const float* gain, float eps, int T, int d,
                         float* dh, int acc, float* part, hipStream_t s) {
  const int nb = backward_blocks(T, d);
  switch (row_threads(d)) {
    case 64:
      layernorm_backward_kernel<T16, 64><<<nb, 64, 0, s>>>(dx, h, gain, dh, part, T, d, eps, acc);
      break;
    case 256:
      layernorm_backward_kernel<T16, 256><<<nb, 256, 0, s>>>(dx, h, gain, dh, part, T, d, eps, acc);
      break;
    case 512:
      layernorm_backward_kernel<T16, 512><<<nb, 512, 0, s>>>(dx, h, gain, dh, part, T, d, eps, acc);
      break;
    default:
      layernorm_backward_kernel<T16, 1024><<<nb, 1024, 0, s>>>(dx, h, gain, dh, part, T, d, eps, acc);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_layernorm(const float* h, const float* gain, const float* bias, void* x,
                            int type, int T, int d, float eps, hipStream_t s) {
  return type == TYPE_F16 ? norm_forward(h, gain, bias, static_cast<f16*>(x), T, d, eps, s)
                          : norm_forward(h, gain, bias, static_cast<bf16*>(x), T, d, eps, s);
}

size_t layernorm_workspace(int T, int d) {
  return ((size_t)backward_blocks(T, d) * 2 * d * sizeof(float) + 255) & ~(size_t)255;
}

hipError_t launch_layernorm_backward(const void* dx, int type, const float* h, const float* gain,
                                     float eps, int T, int d, float* dh, bool accumulate,
                                     float* d_gain, float* d_bias, void* ws, hipStream_t s) {
  float* part = d_gain || d_bias ? static_cast<float*>(ws) : nullptr;
  hipError_t e = type == TYPE_F16
                     ? norm_backward(static_cast<const f16*>(dx), h, gain, eps, T, d, dh, accumulate, part, s)
                     : norm_backward(static_cast<const bf16*>(dx), h, gain, eps, T, d, dh, accumulate, part, s);
  if (e != hipSuccess || !part) return e;
  column_sums_kernel<<<d / 32, kSumThreads, 0, s>>>(part, backward_blocks(T, d), d, d_gain, d_bias);
  return hipGetLastError();
}

}  // namespace moe
