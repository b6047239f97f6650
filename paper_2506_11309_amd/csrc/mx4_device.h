// Device helpers of the 4-bit matrix kernels.
#pragma once
#include "product_device.h"

namespace ss {

// ---- microscaled 4-bit values (mx4_quant.hip has the format)
// Scale byte of a block whose largest magnitude has the fp16 bits m, and the
// float that the conversion divides by.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t m) {
  const uint32_t e = bitcast<uint32_t>(h2f((uint16_t)m)) >> 23;  // every fp16 value is a normal fp32
  return m >= 0x7C00u ? 255u : m == 0 ? 127u : e - 2;
}
__device__ __forceinline__ uint32_t mx4_magnitude(const u32x4& v) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, bitcast<u16x2>(v[i] & 0x7FFF7FFFu));
  return max((uint32_t)m[0], (uint32_t)m[1]);
}
// codes of 8 values; a block without a scale (255) has codes 0
__device__ __forceinline__ uint32_t mx4_codes(const u32x4& v, uint32_t scale) {
  const float unit = bitcast<float>(scale << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, bitcast<half2v>(v[0]), unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, bitcast<half2v>(v[1]), unit, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, bitcast<half2v>(v[2]), unit, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, bitcast<half2v>(v[3]), unit, 3);
  return scale == 255u ? 0u : c;
}

}  // namespace ss
