// MXFP4 quantiser: 32 columns share the scale 2^e, e = floor(log2 max|v|) - 2
// (at least -127), and hold the code of e2m1 nearest to v / 2^e.
//
// The codes come from the conversion instruction, which divides by the scale,
// rounds ties to the even code and saturates.  The largest magnitude is kept
// as the bits of its fp32 form, whose order is that of the numbers and ends in
// infinity and NaN; its exponent field less 2 is the scale byte (a number
// below 2^-126 has the field 0, and the byte 0 is the least).
//
// Bound by memory.  Four lanes share a block of columns: every load and store is
// then contiguous over the wave (a thread per block took 57 us where this takes
// 41, of 14336 x 4096: 267 MB with the values, 6.6 TB/s).  Four chunks per thread
// cover the way to memory; with 1, 2 or 8 it took 43, 43 or 45.
#include "moe_internal.h"

namespace moe {

namespace {

constexpr int kThreads = 256, kChunks = 4;
constexpr int kPerBlock = kThreads / 4 * kChunks;  // blocks of 32 columns

template <class T> struct Pair;
template <> struct Pair<f16> {
  typedef f16 x2 __attribute__((ext_vector_type(2)));
  template <int SEL> static __device__ uint32_t code(uint32_t old, uint32_t v, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(x2, v), s, SEL);
  }
  template <int SEL> static __device__ uint32_t value(uint32_t c, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, SEL));
  }
};
template <> struct Pair<bf16> {
  typedef bf16 x2 __attribute__((ext_vector_type(2)));
  template <int SEL> static __device__ uint32_t code(uint32_t old, uint32_t v, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(x2, v), s, SEL);
  }
  template <int SEL> static __device__ uint32_t value(uint32_t c, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, SEL));
  }
};

// 2^(byte - 127); the byte 255: NaN.
__device__ inline float scale_of(uint32_t byte) {
  return __builtin_bit_cast(float, byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

}  // namespace

// Four lanes share a block, 8 columns each, so that loads and stores are
// contiguous over a wave; chunk c of lane l is columns 8 (l % 4) .. + 7 of block
// 16 c + l / 4 of the wave's 64.
template <class T>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const T* v, int64_t n_blocks,
                                                               uint8_t* codes, uint8_t* scales,
                                                               T* values) {
  typedef typename Pair<T>::x2 x2;
  const int lane = threadIdx.x & 63;
  const int64_t b0 = (int64_t)blockIdx.x * kPerBlock + (threadIdx.x >> 6) * (16 * kChunks) + (lane >> 2);
  u32x4 in[kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int64_t b = b0 + 16 * c;
    in[c] = b < n_blocks ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(v) + 4 * b + (lane & 3))
                         : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int64_t b = b0 + 16 * c;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u = in[c][j];
      const x2 p = __builtin_bit_cast(x2, u);
      const uint32_t lo = __builtin_bit_cast(uint32_t, (float)p.x) & 0x7FFFFFFFu;
      const uint32_t hi = __builtin_bit_cast(uint32_t, (float)p.y) & 0x7FFFFFFFu;
      top = max(top, max(lo, hi));
    }
    top = dpp_max<0xB1>(top);  // quad_perm [1,0,3,2]
    top = dpp_max<0x4E>(top);  // quad_perm [2,3,0,1]
    const uint32_t field = top >> 23;
    const uint32_t byte = field == 255 ? 255 : field < 2 ? 0 : field - 2;
    const float s = scale_of(byte);
    uint32_t k = 0;
    k = Pair<T>::template code<0>(k, in[c][0], s);
    k = Pair<T>::template code<1>(k, in[c][1], s);
    k = Pair<T>::template code<2>(k, in[c][2], s);
    k = Pair<T>::template code<3>(k, in[c][3], s);
    if (b < n_blocks) {
      reinterpret_cast<uint32_t*>(codes)[4 * b + (lane & 3)] = k;
      if ((lane & 3) == 0) scales[b] = (uint8_t)byte;
      if (values)
        __builtin_nontemporal_store(
            u32x4{Pair<T>::template value<0>(k, s), Pair<T>::template value<1>(k, s),
                  Pair<T>::template value<2>(k, s), Pair<T>::template value<3>(k, s)},
            reinterpret_cast<u32x4*>(values) + 4 * b + (lane & 3));
    }
  }
}

hipError_t launch_mx_quantize(const void* v, int type, int64_t rows, int64_t cols, uint8_t* codes,
                              uint8_t* scales, void* values, hipStream_t s) {
  const int64_t n = rows * (cols / kMxBlock);
  if (n == 0) return hipSuccess;
  // (a launch has less than 2^32 threads)
  const unsigned blocks = (unsigned)((n + kPerBlock - 1) / kPerBlock);
  if (type == TYPE_F16)
    mx_quantize_kernel<<<blocks, kThreads, 0, s>>>((const f16*)v, n, codes, scales, (f16*)values);
  else
    mx_quantize_kernel<<<blocks, kThreads, 0, s>>>((const bf16*)v, n, codes, scales, (bf16*)values);
  return hipGetLastError();
}

}  // namespace moe
