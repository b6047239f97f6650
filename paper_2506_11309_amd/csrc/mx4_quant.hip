// Microscaled 4-bit matrices (MXFP4): quantisation, its inverse, and the
// operand forms that the matrix instructions read.
//
// A block is 32 consecutive k of one row: a scale byte s standing for
// 2^(s - 127) (255: NaN) and 32 e2m1 codes (0 .5 1 1.5 2 3 4 6, sign in bit
// 3).  Quantising a block with largest magnitude a: s - 127 = floor(log2 a) - 2,
// so that a lands in [4, 8), and each value goes to the nearest code, ties to
// the even one, saturating at 6.  a = 0: s = 127.  A block holding an infinity
// or a NaN has no scale: s = 255, codes 0, and whatever it enters is NaN.
// a is found on the fp16 bits (an unsigned maximum of magnitudes), its
// exponent is exact in fp32, and the conversion instruction rounds as above
// for every fp16 value, subnormals included.
#include "mx4_device.h"
#include "mx4_internal.h"

namespace ss {

namespace {

constexpr int kUnits = 2;  // pieces of a thread: 28672 x 8192 in 101 us; with 1 106, with 4 107, with 8 109

// 8 fp16 values of one lane, the block's magnitude maximum over its 4 lanes ->
// 8 codes and the scale byte
__device__ __forceinline__ uint32_t quantize8(const u32x4& v, uint32_t& scale) {
  uint32_t m = mx4_magnitude(v);
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));  // lane ^ 1
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));  // lane ^ 2
  scale = mx4_scale_of(m);
  return mx4_codes(v, scale);
}

// One workgroup writes the row blocks of a product (Mx4Map).
__device__ void write_map(const Mx4Map& m) {
  constexpr int kPer = SWIFTSPEC_MAX_EXPERTS / 256;
  __shared__ int first[SWIFTSPEC_MAX_EXPERTS + 1];  // blocks before expert e
  __shared__ int begin[SWIFTSPEC_MAX_EXPERTS], end[SWIFTSPEC_MAX_EXPERTS];
  __shared__ int wave_sum[4];
  __shared__ int bad;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  if (tid == 0) bad = 0;
  __syncthreads();
  int n[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = tid * kPer + i;
    n[i] = 0;
    if (e < m.E) {
      const int lo = m.offsets[e], hi = m.offsets[e + 1];
      begin[e] = lo;
      end[e] = hi;
      if (lo < 0 || hi < lo || hi > m.M || (e == 0 && lo != 0)) bad = 1;
      else n[i] = (hi - lo + m.tm - 1) / m.tm;
    }
    sum += n[i];
  }
  const int s = wave_scan_add(sum);
  if (lane == 63) wave_sum[wave] = s;
  __syncthreads();
  int at = s - sum;
  for (int w = 0; w < wave; ++w) at += wave_sum[w];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = tid * kPer + i;
    if (e < m.E) first[e] = at;
    at += n[i];
    if (e == m.E - 1) first[m.E] = at;
  }
  __syncthreads();
  if (tid == 0) {
    if (bad) report_error(m.ws, SWIFTSPEC_DEVERR_BAD_GROUPS);
    m.map[0] = !bad;
    m.map[1] = bad ? 0 : end[m.E - 1];
  }
  const int used = bad ? 0 : first[m.E];
  for (int i = tid; i < m.blocks; i += 256) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (i < used) {
      int lo = 0, hi = m.E - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (first[mid] <= i) lo = mid;
        else hi = mid - 1;
      }
      const int m0 = begin[lo] + (i - first[lo]) * m.tm;
      v = u32x4{(uint32_t)lo, (uint32_t)m0, (uint32_t)min(m.tm, end[lo] - m0), 0u};
    }
    *reinterpret_cast<u32x4*>(m.map + 4 * ((int64_t)i + 1)) = v;
  }
}

// One thread per 8 values, kUnits of them 256 apart; 4 neighbouring lanes hold a
// block (whole rows are multiples of 4 pieces, so a block never spans waves).
// OPERAND: rows padded to whole groups of 128, scales in the operand order; for
// experts the first workgroup writes the row blocks instead.
// Bound by its bytes: 28672 x 8192 (595 MB) 100 us, 5.9 TB/s.
template <bool OPERAND>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const uint16_t* __restrict__ x, int64_t M, int K, int64_t ldx,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                           const int32_t* last, Mx4Map map) {
  if constexpr (OPERAND) {
    if (map.offsets && blockIdx.x == 0) return write_map(map);
    if (last) M = min(M, (int64_t)max(last[map.E], 0));
  }
  const int kp = OPERAND ? (K + 127) / 128 * 16 : K / 8;  // pieces of a row
  const int sb = OPERAND ? (kp / 16 + 3) / 4 * 16 : K / 32;  // scale bytes of a row
  const int64_t first = (int64_t)(blockIdx.x - (OPERAND && map.offsets ? 1 : 0)) * (256 * kUnits);
  const int64_t row0 = first / kp;
  if (OPERAND && row0 >= M) return;
  const uint32_t c0 = (uint32_t)(first - row0 * kp) + threadIdx.x, d0 = c0 / (uint32_t)kp;
  const int over = 256 / kp, step = 256 - over * kp;  // 256 pieces on: `over` rows, or one more, and `step` pieces
  u32x4 v[kUnits];
  int64_t row[kUnits];
  int col[kUnits];
  row[0] = row0 + d0;
  col[0] = (int)(c0 - d0 * (uint32_t)kp);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (u) {
      const bool wrap = col[u - 1] + step >= kp;
      col[u] = col[u - 1] + step - (wrap ? kp : 0);
      row[u] = row[u - 1] + over + (wrap ? 1 : 0);
    }
    v[u] = u32x4{0, 0, 0, 0};
    if (row[u] < M && (!OPERAND || col[u] < K / 8)) v[u] = *reinterpret_cast<const u32x4*>(x + row[u] * ldx + 8 * col[u]);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    uint32_t s;
    const uint32_t q = quantize8(v[u], s);
    if (row[u] >= M) continue;
    *reinterpret_cast<uint32_t*>(codes + (row[u] * kp + col[u]) * 4) = q;
    if ((col[u] & 3) == 0) {
      const int b = col[u] >> 2;  // block of 32
      if (OPERAND) {
        const int g = b >> 2, kq = b & 3;
        uint8_t* p = scales + row[u] * sb + (g >> 2) * 16 + kq * 4;
        p[g & 3] = (uint8_t)s;
        // the last group also fills the bytes of the groups that are not there
        if (g == kp / 16 - 1)
          for (int j = (g & 3) + 1; j < 4; ++j) p[j] = 127;
      } else {
        scales[row[u] * sb + b] = (uint8_t)s;
      }
    }
  }
}

// 8 codes of one row to fp16, rounded to nearest even, overflowing to infinity.
// Bound by its bytes: 28672 x 8192 (595 MB) 104 us, 5.7 TB/s.
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                             int64_t M, int K, uint16_t* __restrict__ y, int64_t ldy) {
  const int kp = K / 8;
  const int64_t first = (int64_t)blockIdx.x * (256 * kUnits);
  const int64_t row0 = first / kp;
  const uint32_t c0 = (uint32_t)(first - row0 * kp) + threadIdx.x, d0 = c0 / (uint32_t)kp;
  const int over = 256 / kp, step = 256 - over * kp;
  uint32_t q[kUnits], s[kUnits];
  int64_t row[kUnits];
  int col[kUnits];
  row[0] = row0 + d0;
  col[0] = (int)(c0 - d0 * (uint32_t)kp);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (u) {
      const bool wrap = col[u - 1] + step >= kp;
      col[u] = col[u - 1] + step - (wrap ? kp : 0);
      row[u] = row[u - 1] + over + (wrap ? 1 : 0);
    }
    if (row[u] < M) {
      q[u] = *reinterpret_cast<const uint32_t*>(codes + (row[u] * kp + col[u]) * 4);
      s[u] = scales[row[u] * (K / 32) + (col[u] >> 2)];
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (row[u] >= M) continue;
    const float unit = s[u] == 255u ? __builtin_nanf("") : s[u] ? bitcast<float>(s[u] << 23) : 0x1p-127f;
    u32x4 o;
    auto two = [&](f32x2 f) {
      const uint32_t lo = f2h(f[0] * unit), hi = f2h(f[1] * unit);
      return lo | hi << 16;
    };
    o[0] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], 1.f, 0));
    o[1] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], 1.f, 1));
    o[2] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], 1.f, 2));
    o[3] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], 1.f, 3));
    // past the caches: the codes that are still to be read stay in them (28672 x
    // 8192 after its quantisation: 123 -> 100 us)
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(y + row[u] * ldy + 8 * col[u]));
  }
}

// A wave writes one kilobyte block (tile, group); its first group of four also
// the scale words of the four.  Bound by its bytes, once per matrix: 8 experts of
// 14336 x 4096 (499 MB read and written) 97 us.
__global__ __launch_bounds__(256) void mx4_prepack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                          int K, int64_t tiles, uint8_t* __restrict__ packed) {
  const int G = (K + 127) / 128, G4 = (G + 3) / 4, B = K / 32;
  const int lane = lane_id(), r = lane & 15, kq = lane >> 4;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = w / G;
  const int g = (int)(w - t * G);
  if (t >= tiles) return;
  const int64_t row = t * 16 + r;
  const int b = 4 * g + kq;
  u32x4 v = {0, 0, 0, 0};
  if (b < B) v = *reinterpret_cast<const u32x4*>(codes + (row * B + b) * 16);
  *reinterpret_cast<u32x4*>(packed + (w * 64 + lane) * 16) = v;
  if ((g & 3) == 0) {
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int bj = b + 4 * j;
      word |= (uint32_t)(bj < B ? scales[row * B + bj] : 127) << (8 * j);
    }
    uint8_t* sw = packed + tiles * G * 1024;
    *reinterpret_cast<uint32_t*>(sw + ((t * G4 + (g >> 2)) * 64 + lane) * 4) = word;
  }
}

unsigned blocks_for(int64_t pieces) { return (unsigned)((pieces + 256 * kUnits - 1) / (256 * kUnits)); }

}  // namespace

void launch_mx4_prepack(const uint8_t* codes, const uint8_t* scales, int K, int64_t rows, void* packed, hipStream_t st) {
  const int64_t tiles = rows / 16;
  hipLaunchKernelGGL(mx4_prepack_kernel, dim3((unsigned)((tiles * mx4_groups(K) + 3) / 4)), dim3(256), 0, st, codes, scales, K,
                     tiles, static_cast<uint8_t*>(packed));
}

void launch_mx4_quantize(const uint16_t* x, int64_t M, int K, int64_t ldx, uint8_t* codes, uint8_t* scales, hipStream_t st) {
  hipLaunchKernelGGL((mx4_quantize_kernel<false>), dim3(blocks_for(M * (K / 8))), dim3(256), 0, st, x, M, K, ldx, codes, scales,
                     (const int32_t*)nullptr, Mx4Map{});
}

void launch_mx4_prepare(const uint16_t* x, int64_t M, int K, int64_t ldx, uint8_t* codes, uint8_t* scales,
                        const int32_t* last, const Mx4Map& map, hipStream_t st) {
  hipLaunchKernelGGL((mx4_quantize_kernel<true>), dim3(blocks_for(M * mx4_groups(K) * 16) + (map.offsets ? 1 : 0)), dim3(256), 0,
                     st, x, M, K, ldx, codes, scales, last, map);
}

void launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t M, int K, uint16_t* y, int64_t ldy,
                           hipStream_t st) {
  hipLaunchKernelGGL(mx4_dequantize_kernel, dim3(blocks_for(M * (K / 8))), dim3(256), 0, st, codes, scales, M, K, y, ldy);
}

}  // namespace ss
