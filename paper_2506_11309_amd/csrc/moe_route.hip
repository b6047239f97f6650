// Router of a mixture of experts: softmax and top-k of each token's scores, and
// the stable grouping of the (token, slot) pairs by expert.
//
// Scores are compared as 16-bit keys that ascend with the value (-0 as +0)
// above the complement of the index, so that one unsigned maximum gives the
// largest score and, among equals, the lowest index.  -inf and NaN are masked:
// their key is 0 and they have no share of the softmax.
// The grouping is a counting sort: each workgroup counts its stretch of pairs
// per expert; a second launch adds the counts of the stretches before it and
// ranks its own pairs in order (up to 1024 pairs: one workgroup, one launch).  Counts are integers, so the order of the LDS
// atomics that add them does not show.
#include "ss_device.h"
#include "ss_internal.h"

namespace ss {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxE = SWIFTSPEC_MAX_EXPERTS;
constexpr int kMaxStretches = 128;

// tokens of a stretch: whole tokens, at most kMaxStretches stretches
__host__ __device__ inline int stretch_tokens(int T, int k) {
  const int least = kThreads / k;  // about one pair a thread
  const int need = (T + kMaxStretches - 1) / kMaxStretches;
  return need > least ? need : least;
}

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

// ascending 16-bit key of an fp16 score, 0 where masked (-inf, NaN); +inf counts as 65504
__device__ __forceinline__ uint32_t score_key(uint32_t h) {
  if ((h & 0x7FFFu) > 0x7C00u || h == 0xFC00u) return 0;
  if (h == 0x8000u) h = 0;
  if (h == 0x7C00u) h = 0x7BFFu;
  return h & 0x8000u ? 0xFFFFu - h : h + 0x8000u;
}
__device__ __forceinline__ float key_score(uint32_t key) {
  return h2f((uint16_t)(key & 0x8000u ? key - 0x8000u : 0xFFFFu - key));
}

struct RouteArgs {
  const uint16_t* logits;
  int64_t ldl;
  int T, E, k, renormalize, tokens;
  bool lines;  // rows can be read 16 bytes at a time
  int32_t* experts;
  float* weights;
  int32_t *offsets, *rows, *pos, *hist;
};

// 16 lanes take the top k of a token's row, V scores each (from 8 on in whole
// 16-byte pieces, 8 (16 q + lane) .. + 7), so that a wave routes four tokens and
// its reductions stay within the rows of 16 lanes that the ALU shifts in.  Lane
// j < k keeps the j-th expert; every lane follows the sums.  Where t >= T nothing
// is written.
template <int V>
__device__ __forceinline__ void route_token(const RouteArgs& a, int t, int* counts) {
  const int l = lane_id() & 15;
  const bool there = t < a.T;
  const uint16_t* row = a.logits + (int64_t)(there ? t : 0) * a.ldl;
  uint32_t key[V];
  if constexpr (V < 8) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = l + 16 * i;
      key[i] = e < a.E ? row[e] : 0xFC00u;
    }
  } else {
#pragma unroll
    for (int q = 0; q < V / 8; ++q) {
      const int e = 8 * (16 * q + l);
      u32x4 v = {0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u};
      if (a.lines && e + 8 <= a.E) {
        v = *reinterpret_cast<const u32x4*>(row + e);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (e + i < a.E) v[i >> 1] = i & 1 ? (v[i >> 1] & 0xFFFFu) | (uint32_t)row[e + i] << 16 : (v[i >> 1] & 0xFFFF0000u) | row[e + i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) key[8 * q + i] = i & 1 ? v[i >> 1] >> 16 : v[i >> 1] & 0xFFFFu;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = V < 8 ? l + 16 * i : 8 * (16 * (i >> 3) + l) + (i & 7);
    const uint32_t s = score_key(key[i]);
    key[i] = s ? s << 16 | (0xFFFFu - (uint32_t)e) : 0u;
  }
  uint32_t best = 0;
  float top = 0.f, mine = 0.f, chosen = 0.f, all = 0.f;
  for (int j = 0; j < a.k; ++j) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) m = max(m, key[i]);
    m = row_max(m);
    if (j == 0) {
      top = m ? key_score(m >> 16) : 0.f;
      if (!a.renormalize) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (key[i]) all += expf(key_score(key[i] >> 16) - top);
        all = row_sum(all);
      }
    }
    const float p = m ? expf(key_score(m >> 16) - top) : 0.f;
    chosen += p;
    if (l == j) {
      best = m;
      mine = p;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (key[i] == m) key[i] = 0;
  }
  if (l < a.k && there) {
    const int e = best ? (int)(0xFFFFu - (best & 0xFFFFu)) : -1;
    const float total = a.renormalize ? chosen : all;
    a.experts[(int64_t)t * a.k + l] = e;
    a.weights[(int64_t)t * a.k + l] = best ? mine / total : 0.f;
    if (e >= 0) atomicAdd(counts + e, 1);
  }
}

// Choose (or read) the experts of tokens t0 .. t1 and count them.
template <int V>
__device__ __forceinline__ void route_stretch(const RouteArgs& a, int t0, int t1, int* counts) {
  for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
  __syncthreads();
  if (a.logits) {
    for (int t = t0 + 4 * (int)(threadIdx.x >> 6); t < t1; t += 4 * kWaves) {
      const int mine = t + (lane_id() >> 4);
      route_token<V>(a, mine < t1 ? mine : a.T, counts);
    }
  } else {
    for (int i = t0 * a.k + (int)threadIdx.x; i < t1 * a.k; i += kThreads) {
      const int e = a.experts[i];
      if (e >= 0 && e < a.E) atomicAdd(counts + e, 1);
    }
  }
  __syncthreads();
}

struct GroupLds {
  int base[kMaxE];           // next place of each expert's pairs in this stretch
  int count[kWaves][kMaxE];  // pairs of each wave
  int wave_total[kWaves];
};

// The places of the pairs of tokens t0 .. t1.  Thread e brings expert e's pairs
// in all stretches and in those before this one.
__device__ __forceinline__ void group_stretch(const RouteArgs& a, int t0, int t1, int all, int before, bool writes_offsets,
                                              GroupLds& s) {
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  int scan = all;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(scan, d, kWave);
    if (lane >= d) scan += o;
  }
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
    int e = i < n1 ? a.experts[i] : -1;
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

// One stretch: everything in one workgroup.
template <int V>
__global__ __launch_bounds__(kThreads) void route_one_kernel(RouteArgs a) {
  __shared__ int counts[kMaxE];
  __shared__ GroupLds s;
  route_stretch<V>(a, 0, a.T, counts);
  group_stretch(a, 0, a.T, (int)threadIdx.x < a.E ? counts[threadIdx.x] : 0, 0, true, s);
}

// Several: count, then place.
template <int V>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  __shared__ int counts[kMaxE];
  const int t0 = blockIdx.x * a.tokens;
  route_stretch<V>(a, t0, min(a.T, t0 + a.tokens), counts);
  for (int e = threadIdx.x; e < a.E; e += kThreads) a.hist[(int64_t)blockIdx.x * a.E + e] = counts[e];
}

__global__ __launch_bounds__(kThreads) void group_kernel(RouteArgs a, int stretches) {
  __shared__ int part_all[kThreads], part_before[kThreads];
  __shared__ GroupLds s;
  // a power of two of experts side by side, the stretches shared out between
  // the parts of the workgroup that this leaves
  const int tid = threadIdx.x, wide = 1 << (32 - __builtin_clz(max(a.E, 2) - 1));
  const int part = tid / wide, parts = kThreads / wide, e = tid - part * wide;
  int all = 0, before = 0;
  if (e < a.E) {
#pragma unroll 8
    for (int i = part; i < stretches; i += parts) {
      const int c = a.hist[(int64_t)i * a.E + e];
      all += c;
      before += i < (int)blockIdx.x ? c : 0;
    }
  }
  part_all[tid] = all;
  part_before[tid] = before;
  __syncthreads();
  all = before = 0;
  if (tid < a.E)
    for (int p = 0; p < parts; ++p) {
      all += part_all[p * wide + tid];
      before += part_before[p * wide + tid];
    }
  const int t0 = blockIdx.x * a.tokens;
  group_stretch(a, t0, min(a.T, t0 + a.tokens), all, before, blockIdx.x == 0, s);
}

template <int V>
void launch_route(const RouteArgs& a, int stretches, hipStream_t st) {
  if (stretches <= 1) {
    hipLaunchKernelGGL(route_one_kernel<V>, dim3(1), dim3(kThreads), 0, st, a);
  } else {
    hipLaunchKernelGGL(route_kernel<V>, dim3((unsigned)stretches), dim3(kThreads), 0, st, a);
    hipLaunchKernelGGL(group_kernel, dim3((unsigned)stretches), dim3(kThreads), 0, st, a, stretches);
  }
}

}  // namespace

size_t route_hist_bytes(int T, int E, int k) {
  const int tokens = stretch_tokens(T, k);
  return (size_t)((T + tokens - 1) / tokens) * E * sizeof(int32_t);
}

void launch_moe_route(const RouteLaunch& L, hipStream_t st) {
  RouteArgs a;
  a.logits = L.logits;
  a.ldl = L.ldl;
  a.T = L.T;
  a.E = L.E;
  a.k = L.k;
  a.renormalize = L.renormalize;
  a.tokens = stretch_tokens(L.T, L.k);
  a.experts = L.experts;
  a.weights = L.weights;
  a.offsets = L.offsets;
  a.rows = L.rows;
  a.pos = L.pos;
  a.hist = L.hist;
  a.lines = (reinterpret_cast<uintptr_t>(L.logits) & 15) == 0 && L.ldl % 8 == 0;
  const int stretches = (L.T + a.tokens - 1) / a.tokens;
  const int v = L.logits ? (L.E + 15) / 16 : 1;  // scores of a lane
  if (v <= 1) launch_route<1>(a, stretches, st);
  else if (v <= 2) launch_route<2>(a, stretches, st);
  else if (v <= 4) launch_route<4>(a, stretches, st);
  else if (v <= 8) launch_route<8>(a, stretches, st);
  else if (v <= 16) launch_route<16>(a, stretches, st);
  else launch_route<32>(a, stretches, st);
}

}  // namespace ss
