// The last step of products whose results are summed by a kernel of their own: the
// experts' rows of a token, or the parts of a K that several workgroups share.
#include "product_device.h"

namespace ss {

namespace {

// One thread per 4 columns of a token; the addends in slot order, KU of them
// loaded at a time, each the sum of `split` parts in order.  Nothing is written where the offsets were invalid (map[0]).
// Bound by the fp32 rows that it reads: 5000 tokens of 8 slots (10 % of them masked)
// x 2048 columns, 295 MB, 50 us (5.9 TB/s).
template <int KU>
__global__ __launch_bounds__(256) void moe_combine_kernel(const float* __restrict__ part, int split, int T, int k, int N,
                                                          const int32_t* __restrict__ pos,
                                                          const int32_t* __restrict__ map,
                                                          const float* __restrict__ weights, uint16_t* y, int64_t ldy,
                                                          const uint16_t* res, int64_t ldr, void* ws) {
  const int per = N / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t t = i / per;
  if (t >= T) return;
  const int n = (int)(i - t * per) * 4;
  // the lists and the residual are read side by side
  const int valid = map[0], used = map[1];
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (res) add_residual(v, *reinterpret_cast<const u32x2*>(res + t * ldr + n));
  for (int j0 = 0; j0 < k; j0 += KU) {
    int p[KU];
    float w[KU];
    f32x4 o[KU];
#pragma unroll
    for (int j = 0; j < KU; ++j) {
      const int64_t at = t * k + min(j0 + j, k - 1);
      p[j] = pos[at];
      w[j] = weights[at];
    }
    if (!valid) return;
#pragma unroll
    for (int j = 0; j < KU; ++j) {
      if (j0 + j >= k) p[j] = -1;
      if (p[j] >= used) {
        report_error(ws, SWIFTSPEC_DEVERR_BAD_GROUPS);
        p[j] = -1;
      }
    }
#pragma unroll
    for (int j = 0; j < KU; ++j)
      if (p[j] >= 0) o[j] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(part + (int64_t)p[j] * N + n));
#pragma unroll
    for (int j = 0; j < KU; ++j)
      if (p[j] >= 0) {
        for (int s = 1; s < split; ++s) o[j] += *reinterpret_cast<const f32x4*>(part + ((int64_t)s * T * k + p[j]) * N + n);
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = __builtin_fmaf(w[j], o[j][c], v[c]);
      }
  }
  *reinterpret_cast<u32x2*>(y + t * ldy + n) = pack4(v);
}

// y = fp16(the sum of `split` parts [M][N] in order + residual); 4 columns a thread.
// The parts were just written: bound by its launch and one round of reads.
__global__ __launch_bounds__(256) void product_sum_kernel(const float* __restrict__ part, int split, int M, int N, uint16_t* y, int64_t ldy,
                                                      const uint16_t* res, int64_t ldr) {
  const int per = N / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = i / per;
  if (m >= M) return;
  const int n = (int)(i - m * per) * 4;
  const float* p = part + m * N + n;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  u32x2 r = {0u, 0u};
  if (res) r = *reinterpret_cast<const u32x2*>(res + m * ldr + n);
#pragma unroll 8
  for (int s = 0; s < split; ++s) v += *reinterpret_cast<const f32x4*>(p + (int64_t)s * M * N);
  add_residual(v, r);
  *reinterpret_cast<u32x2*>(y + m * ldy + n) = pack4(v);
}

}  // namespace

void launch_moe_combine(const float* part, int split, int T, int k, int N, const int32_t* pos, const int32_t* map,
                        const float* weights, uint16_t* y, int64_t ldy, const uint16_t* res, int64_t ldr, void* ws,
                        hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)T * (N / 4) + 255) / 256));
  if (k <= 2) hipLaunchKernelGGL(moe_combine_kernel<2>, grid, dim3(256), 0, st, part, split, T, k, N, pos, map, weights, y, ldy, res, ldr, ws);
  else if (k <= 4) hipLaunchKernelGGL(moe_combine_kernel<4>, grid, dim3(256), 0, st, part, split, T, k, N, pos, map, weights, y, ldy, res, ldr, ws);
  else hipLaunchKernelGGL(moe_combine_kernel<8>, grid, dim3(256), 0, st, part, split, T, k, N, pos, map, weights, y, ldy, res, ldr, ws);
}

void launch_product_sum(const float* part, int split, int M, int N, uint16_t* y, int64_t ldy, const uint16_t* res, int64_t ldr,
                        hipStream_t st) {
  hipLaunchKernelGGL(product_sum_kernel, dim3((unsigned)(((int64_t)M * (N / 4) + 255) / 256)), dim3(256), 0, st, part, split, M, N, y,
                     ldy, res, ldr);
}

}  // namespace ss
