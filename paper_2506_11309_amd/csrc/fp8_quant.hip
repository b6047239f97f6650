// Block-scaled 8-bit matrices: quantisation, its inverse, and the operand forms that
// the matrix instructions read.
//
// A value is an e4m3 code (sign, four exponent and three mantissa bits, bias 7, largest
// 448, no infinities, 0x7F and 0xFF NaN) times the scale of its block.  A matrix has a
// float for each block of 128 rows and 128 columns; the scales of a published one are
// any floats.  Quantising a block with largest magnitude a takes the least power of two
// s with a <= 448 s, and the nearest code of each value / s, ties to the even one:
// codes that float keep their relative step under any scale, and with a power of two
// the division is exact and the matrix instruction multiplies by it as it reads its
// operand.  a = 0: s = 1.  A block that holds an infinity or a NaN has no scale: s is
// NaN, codes 0, and whatever it enters is NaN.
// a is found on the fp16 bits (an unsigned maximum of magnitudes), and the conversion
// instruction rounds as above for every fp16 value, subnormals included.
#include "fp8_device.h"
#include "fp8_internal.h"

namespace ss {

namespace {

constexpr int kUnits = 2;  // pieces of a thread

__device__ __forceinline__ float scale_value(uint32_t s) { return s == 255u ? __builtin_nanf("") : bitcast<float>(s << 23); }

// the largest of 16 neighbouring lanes
__device__ __forceinline__ uint32_t max16(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x128, 0xF, 0xF, true));  // rotations within rows of 16
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x124, 0xF, 0xF, true));
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x122, 0xF, 0xF, true));
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x121, 0xF, 0xF, true));
}

// One thread per 8 values, kUnits of them 256 apart; 16 neighbouring lanes hold a
// block (rows are padded to whole ones).  OPERAND: the activations of a product; for
// experts the first workgroup writes the row blocks instead.  Bound by its bytes: 40000
// rows of 1072 columns (129 MB) 21.6 us, 6.0 TB/s; few rows by its launch, 2.4 us.
template <bool OPERAND>
__global__ __launch_bounds__(256) void fp8_quantize_kernel(const uint16_t* __restrict__ x, int64_t M, int K, int64_t ldx,
                                                           uint8_t* __restrict__ codes, void* __restrict__ scales,
                                                           const int32_t* last, RowMap map) {
  if constexpr (OPERAND) {
    if (map.offsets && blockIdx.x == 0) return write_map(map);
    if (last) M = min(M, (int64_t)max(last[map.E], 0));
  }
  const int G = (K + 127) / 128, kp = G * 16;  // pieces of a row
  const int64_t first = (int64_t)(blockIdx.x - (OPERAND && map.offsets ? 1 : 0)) * (256 * kUnits);
  const int64_t row0 = first / kp;
  if (row0 >= M) return;
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
    if (row[u] < M && col[u] < K / 8) v[u] = *reinterpret_cast<const u32x4*>(x + row[u] * ldx + 8 * col[u]);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const uint32_t s = fp8_scale_of(max16(fp8_magnitude(v[u])));
    if (row[u] >= M || (!OPERAND && col[u] >= K / 8)) continue;
    *reinterpret_cast<u32x2*>(codes + row[u] * (OPERAND ? kp * 8 : K) + 8 * col[u]) = fp8_codes(v[u], s);
    if (col[u] & 15) continue;
    const int g = col[u] >> 4;
    if constexpr (OPERAND) {
      uint8_t* p = static_cast<uint8_t*>(scales) + row[u] * ((G + 3) / 4 * 4) + g;
      p[0] = (uint8_t)s;
      // the last group also fills the bytes of the groups that are not there
      if (g == G - 1)
        for (int j = 1; j < 4 - (g & 3); ++j) p[j] = 127;
    } else {
      static_cast<float*>(scales)[row[u] * G + g] = scale_value(s);
    }
  }
}

// A workgroup takes a block of 128 rows and columns, 8 pieces a thread, all loaded
// before the first is needed.  Bound by its bytes: 28672 x 8192 (705 MB) 122 us, 5.8 TB/s,
// more than a copy's 4.9.
__global__ __launch_bounds__(256) void fp8_quantize_blocks_kernel(const uint16_t* __restrict__ x, int64_t M, int K, int64_t ldx,
                                                                  uint8_t* __restrict__ codes, float* __restrict__ scales) {
  __shared__ uint32_t most[4];
  const int G = (K + 127) / 128;
  const int64_t rb = blockIdx.x / (uint32_t)G;
  const int g = (int)(blockIdx.x - rb * G), col = 16 * g + (threadIdx.x & 15);  // in pieces of 8
  const int64_t row0 = rb * 128 + (threadIdx.x >> 4);
  u32x4 v[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = u32x4{0, 0, 0, 0};
    if (row0 + 16 * i < M && col < K / 8) v[i] = *reinterpret_cast<const u32x4*>(x + (row0 + 16 * i) * ldx + 8 * col);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, fp8_magnitude(v[i]));
  m = max16(m);
  m = max(max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16)),
          max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48)));
  if (lane_id() == 0) most[threadIdx.x >> 6] = m;
  __syncthreads();
  const uint32_t s = fp8_scale_of(max(max(most[0], most[1]), max(most[2], most[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (row0 + 16 * i < M && col < K / 8) *reinterpret_cast<u32x2*>(codes + (row0 + 16 * i) * K + 8 * col) = fp8_codes(v[i], s);
  if (threadIdx.x == 0) scales[rb * G + g] = scale_value(s);
}

// 8 codes of one row to fp16, rounded to nearest even, overflowing to infinity.  Product
// and conversion are one instruction (v_fma_mix), which rounds once.  Bound by its
// bytes: 28672 x 8192 (705 MB) 117 us, 6.0 TB/s.
__global__ __launch_bounds__(256) void fp8_dequantize_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales,
                                                             int64_t M, int K, int rows, uint16_t* __restrict__ y, int64_t ldy) {
  const int kp = K / 8, G = (K + 127) / 128;
  const int64_t first = (int64_t)blockIdx.x * (256 * kUnits);
  const int64_t row0 = first / kp;
  const uint32_t c0 = (uint32_t)(first - row0 * kp) + threadIdx.x, d0 = c0 / (uint32_t)kp;
  const int over = 256 / kp, step = 256 - over * kp;
  u32x2 q[kUnits];
  float s[kUnits];
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
      q[u] = *reinterpret_cast<const u32x2*>(codes + row[u] * K + 8 * col[u]);
      s[u] = scales[(rows == 1 ? row[u] : row[u] >> 7) * G + (col[u] >> 4)];
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (row[u] >= M) continue;
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u][i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u][i], true);
      o[2 * i] = f2h(a[0] * s[u]) | (uint32_t)f2h(a[1] * s[u]) << 16;
      o[2 * i + 1] = f2h(b[0] * s[u]) | (uint32_t)f2h(b[1] * s[u]) << 16;
    }
    // past the caches: the codes that are still to be read stay in them
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(y + row[u] * ldy + 8 * col[u]));
  }
}

// Two waves write the 2 KB block of a (tile, group); behind the codes the scales as
// they are.  Bound by its bytes, once per matrix: 8 experts of 14336 x 4096 (940 MB read
// and written) 160 us.
__global__ __launch_bounds__(256) void fp8_prepack_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales, int K,
                                                          int64_t tiles, int64_t n_scales, uint8_t* __restrict__ packed) {
  const int G = (K + 127) / 128;
  const int64_t w = (int64_t)blockIdx.x * 2 + (threadIdx.x >> 7);
  const int p = (threadIdx.x >> 4) & 7, r = threadIdx.x & 15;
  const int64_t t = w / G;
  if (t < tiles) {
    const int piece = 8 * (int)(w - t * G) + p;
    u32x4 v = {0, 0, 0, 0};
    if (piece < K / 16) v = *reinterpret_cast<const u32x4*>(codes + (t * 16 + r) * K + 16 * piece);
    *reinterpret_cast<u32x4*>(packed + w * 2048 + 256 * p + 16 * r) = v;
  }
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;  // fewer than blocks: one for 128 x 128 values
  if (i < n_scales) reinterpret_cast<float*>(packed + tiles * G * 2048)[i] = scales[i];
}

unsigned blocks_for(int64_t pieces) { return (unsigned)((pieces + 256 * kUnits - 1) / (256 * kUnits)); }

}  // namespace

void launch_fp8_prepack(const uint8_t* codes, const float* scales, int K, int N, int E, void* packed, hipStream_t st) {
  const int64_t tiles = (int64_t)E * (N / 16);
  hipLaunchKernelGGL(fp8_prepack_kernel, dim3((unsigned)((tiles * fp8_blocks(K) + 1) / 2)), dim3(256), 0, st, codes, scales, K, tiles,
                     (int64_t)E * fp8_blocks(N) * fp8_blocks(K), static_cast<uint8_t*>(packed));
}

void launch_fp8_quantize(const uint16_t* x, int64_t M, int K, int64_t ldx, int rows, uint8_t* codes, float* scales, hipStream_t st) {
  if (rows == 128)
    hipLaunchKernelGGL(fp8_quantize_blocks_kernel, dim3((unsigned)((M + 127) / 128 * fp8_blocks(K))), dim3(256), 0, st, x, M, K, ldx,
                       codes, scales);
  else
    hipLaunchKernelGGL((fp8_quantize_kernel<false>), dim3(blocks_for(M * fp8_blocks(K) * 16)), dim3(256), 0, st, x, M, K, ldx, codes,
                       (void*)scales, (const int32_t*)nullptr, RowMap{});
}

void launch_fp8_prepare(const uint16_t* x, int64_t M, int K, int64_t ldx, uint8_t* codes, uint8_t* scales, const int32_t* last,
                        const RowMap& map, hipStream_t st) {
  hipLaunchKernelGGL((fp8_quantize_kernel<true>), dim3(blocks_for(M * fp8_blocks(K) * 16) + (map.offsets ? 1 : 0)), dim3(256), 0, st,
                     x, M, K, ldx, codes, (void*)scales, last, map);
}

void launch_fp8_dequantize(const uint8_t* codes, const float* scales, int64_t M, int K, int rows, uint16_t* y, int64_t ldy,
                           hipStream_t st) {
  hipLaunchKernelGGL(fp8_dequantize_kernel, dim3(blocks_for(M * (K / 8))), dim3(256), 0, st, codes, scales, M, K, rows, y, ldy);
}

}  // namespace ss
