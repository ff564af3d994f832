// MXFP4 quantiser: 32 columns share the scale 2^e, e = floor(log2 max|v|) - 2
// (at least -127), and hold the code of e2m1 nearest to v / 2^e.
//
// The codes come from the conversion instruction, which divides by the scale,
// rounds ties to the even code and saturates.  The largest magnitude is kept
// as the bits of its fp32 form, whose order is that of the numbers and ends in
// infinity and NaN; its exponent field less 2 is the scale byte (a number
// below 2^-126 has the field 0, and the byte 0 is the least).
#include "moe_internal.h"

namespace moe {

namespace {

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

// One thread per block of 32 columns.
template <class T>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T* v, int64_t n_blocks,
                                                          uint8_t* codes, uint8_t* scales,
                                                          T* values) {
  typedef typename Pair<T>::x2 x2;
  const int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (b >= n_blocks) return;
  u32x4 in[4];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    in[i] = reinterpret_cast<const u32x4*>(v)[4 * b + i];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t u = in[i][j];
      const x2 p = __builtin_bit_cast(x2, u);
      top = max(top, __builtin_bit_cast(uint32_t, (float)p.x) & 0x7FFFFFFFu);
      top = max(top, __builtin_bit_cast(uint32_t, (float)p.y) & 0x7FFFFFFFu);
    }
  }
  const uint32_t field = top >> 23;
  const uint32_t byte = field == 255 ? 255 : field < 2 ? 0 : field - 2;
  const float s = scale_of(byte);
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t c = 0;
    c = Pair<T>::template code<0>(c, in[i][0], s);
    c = Pair<T>::template code<1>(c, in[i][1], s);
    c = Pair<T>::template code<2>(c, in[i][2], s);
    c = Pair<T>::template code<3>(c, in[i][3], s);
    out[i] = c;
  }
  reinterpret_cast<u32x4*>(codes)[b] = out;
  scales[b] = (uint8_t)byte;
  if (values) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t c = out[i];
      reinterpret_cast<u32x4*>(values)[4 * b + i] =
          u32x4{Pair<T>::template value<0>(c, s), Pair<T>::template value<1>(c, s),
                Pair<T>::template value<2>(c, s), Pair<T>::template value<3>(c, s)};
    }
  }
}

hipError_t launch_mx_quantize(const void* v, int type, int64_t rows, int64_t cols, uint8_t* codes,
                              uint8_t* scales, void* values, hipStream_t s) {
  const int64_t n = rows * (cols / kMxBlock);
  if (n == 0) return hipSuccess;
  // (a launch has less than 2^32 threads)
  const unsigned blocks = (unsigned)((n + 255) / 256);
  if (type == TYPE_F16)
    mx_quantize_kernel<<<blocks, 256, 0, s>>>((const f16*)v, n, codes, scales, (f16*)values);
  else
    mx_quantize_kernel<<<blocks, 256, 0, s>>>((const bf16*)v, n, codes, scales, (bf16*)values);
  return hipGetLastError();
}

}  // namespace moe
