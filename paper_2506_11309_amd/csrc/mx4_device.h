// Device helpers of the 4-bit matrix and mixture kernels.
#pragma once
#include "ss_device.h"

namespace ss {

// Sum over the lanes up to this one, on the ALU's own lane shifts.
template <int kCtrl, int kRows>
__device__ __forceinline__ int dpp_or_zero(int v) {
  return __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xF, false);
}
__device__ __forceinline__ int wave_scan_add(int v) {
  v += dpp_or_zero<0x111, 0xF>(v);  // from 1, 2, 4, 8 lanes before, within rows of 16
  v += dpp_or_zero<0x112, 0xF>(v);
  v += dpp_or_zero<0x114, 0xF>(v);
  v += dpp_or_zero<0x118, 0xF>(v);
  v += dpp_or_zero<0x142, 0xA>(v);  // the last lane of a row to rows 1 and 3
  v += dpp_or_zero<0x143, 0xC>(v);  // lane 31 to rows 2 and 3
  return v;
}

// buffer_load_lds16 with 4 bytes a lane, landing at lds_addr + 4 l
__device__ __forceinline__ void buffer_load_lds4(i32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds_addr) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\t"
      "buffer_load_dword %1, %2, %3 offen lds\n\ts_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(voff), "s"(rsrc), "s"(soff), "s"(lds_addr)
      : "memory");
}

// Workgroup barrier after this wave's LDS traffic and all but N of its vector-
// memory operations.  The compiler sees the wait, so that values read from LDS
// before it need no other.
template <int N>
__device__ __forceinline__ void vm_lds_barrier() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

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
