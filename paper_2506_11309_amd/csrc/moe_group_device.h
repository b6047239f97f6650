// Device code that the routers share: reductions over a token's 16 lanes and the
// stable grouping of the (token, slot) pairs by expert.
#pragma once
#include "moe_internal.h"
#include "product_device.h"

namespace ss {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxE = SWIFTSPEC_MAX_EXPERTS;

// Over the 16 lanes of a row (rotations within it): every lane gets the result.
template <int kRotate>
__device__ __forceinline__ uint32_t rotated(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x120 + kRotate, 0xF, 0xF, true);  // row_ror
}
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, rotated<8>(v));
  v = max(v, rotated<4>(v));
  v = max(v, rotated<2>(v));
  return max(v, rotated<1>(v));
}
__device__ __forceinline__ float row_sum(float v) {
  v += bitcast<float>(rotated<8>(bitcast<uint32_t>(v)));
  v += bitcast<float>(rotated<4>(bitcast<uint32_t>(v)));
  v += bitcast<float>(rotated<2>(bitcast<uint32_t>(v)));
  return v + bitcast<float>(rotated<1>(bitcast<uint32_t>(v)));
}

struct GroupLds {
  int base[kMaxE];           // next place of each expert's pairs
  int count[kWaves][kMaxE];  // pairs of each wave
  int wave_total[kWaves];
};

// The places of the pairs of tokens t0 .. t1.  Thread e brings the number of expert
// e's pairs, of all tokens and of those before t0.
__device__ __forceinline__ void group_tokens(const GroupArgs& a, int t0, int t1, int all, int before, bool writes_offsets,
                                             const int16_t* chosen, int e_first, GroupLds& s) {
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int scan = wave_scan_add(all);
  if (lane == 63) s.wave_total[wave] = scan;
  __syncthreads();
  int lead = 0, used = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int n = s.wave_total[w];
    lead += w < wave ? n : 0;
    used += n;
  }
  if (tid < a.E) {
    const int off = lead + scan - all;
    s.base[tid] = off + before;
    if (writes_offsets) {
      a.offsets[tid] = off;
      if (tid == a.E - 1) a.offsets[a.E] = off + all;
    }
  }
  const int n0 = t0 * a.k, n1 = t1 * a.k;
  // places past the last pair
  for (int i = n0 + tid; i < n1; i += kThreads)
    if (i >= used) a.rows[i] = -1;
  for (int i0 = n0; i0 < n1; i0 += kThreads) {
    if (tid < a.E)
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s.count[w][tid] = 0;
    __syncthreads();
    const int i = i0 + tid;
    int e = i >= n1 ? -1 : chosen ? chosen[i] : i0 == n0 ? e_first : a.experts[i];
    if (e >= a.E) e = -1;
    const bool has = e >= 0;
    // lanes of this wave with the same expert
    uint64_t same = __ballot(has);
#pragma unroll
    for (int bit = 0; (1 << bit) < kMaxE; ++bit) {
      const uint64_t m = __ballot((e >> bit) & 1);
      same &= (e >> bit) & 1 ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (has && rank == 0) s.count[wave][e] = __popcll(same);
    __syncthreads();
    int place = -1;
    if (has) {
      place = s.base[e] + rank;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) place += w < wave ? s.count[w][e] : 0;
      a.rows[place] = i;
    }
    if (i < n1) a.pos[i] = place;
    if (i0 + kThreads >= n1) break;
    __syncthreads();
    if (tid < a.E) {
      int c = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) c += s.count[w][tid];
      s.base[tid] += c;
    }
    __syncthreads();
  }
}

}  // namespace ss
