// Device helpers of the 8-bit matrix kernels.
#pragma once
#include "product_device.h"

namespace ss {

// ---- values in 8 bits (fp8_quant.hip has the format)
// Scale byte of a block of activations whose largest magnitude has the fp16 bits m:
// the least power of two 2^(s - 127) that brings it to 448 = 1.75 * 2^8 or less.
__device__ __forceinline__ uint32_t fp8_scale_of(uint32_t m) {
  const uint32_t b = bitcast<uint32_t>(h2f((uint16_t)m));  // every fp16 value is a normal fp32
  // past 1.75 the sum carries into the exponent
  return m >= 0x7C00u ? 255u : m == 0 ? 127u : ((b + 0x1FFFFFu) >> 23) - 8;
}
__device__ __forceinline__ uint32_t fp8_magnitude(const u32x4& v) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, bitcast<u16x2>(v[i] & 0x7FFF7FFFu));
  return max((uint32_t)m[0], (uint32_t)m[1]);
}
// codes of 8 values; a block without a scale (255) has codes 0
__device__ __forceinline__ u32x2 fp8_codes(const u32x4& v, uint32_t scale) {
  typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
  const float unit = bitcast<float>(scale << 23);
  i16x2 lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, bitcast<half2v>(v[0]), unit, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, bitcast<half2v>(v[1]), unit, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(hi, bitcast<half2v>(v[2]), unit, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(hi, bitcast<half2v>(v[3]), unit, true);
  return scale == 255u ? u32x2{0u, 0u} : u32x2{bitcast<uint32_t>(lo), bitcast<uint32_t>(hi)};
}

}  // namespace ss
