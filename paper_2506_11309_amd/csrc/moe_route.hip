// Router of a mixture of experts: softmax and top-k of each token's scores, and
// the stable grouping of the (token, slot) pairs by expert.
//
// Scores are compared as 16-bit keys that ascend with the value (-0 as +0)
// above the complement of the index, so that one unsigned maximum gives the
// largest score and, among equals, the lowest index.  -inf and NaN are masked:
// their key is 0 and they have no share of the softmax.
// The grouping is a counting sort: each workgroup counts its stretch of pairs
// per expert; a second launch adds the counts of the stretches before it and
// ranks its own pairs in order.  Counts are integers, so the order of the LDS
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

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d, kWave));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
  return v;
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

// One wave: top k of the token's row.  Lane j < k gets the j-th expert and weight.
template <int V>
__device__ __forceinline__ void route_token(const uint16_t* row, int E, int k, bool renormalize, int32_t* experts, float* weights,
                                            int* counts) {
  const int lane = lane_id();
  uint32_t key[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane + 64 * i;
    const uint32_t s = e < E ? score_key(row[e]) : 0u;
    key[i] = s ? s << 16 | (0xFFFFu - (uint32_t)e) : 0u;
  }
  uint32_t best = 0;
  float top = 0.f, mine = 0.f, chosen = 0.f, all = 0.f;
  for (int j = 0; j < k; ++j) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) m = max(m, key[i]);
    m = wave_max(m);
    if (j == 0) {
      top = m ? key_score(m >> 16) : 0.f;
      if (!renormalize) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (key[i]) all += expf(key_score(key[i] >> 16) - top);
        all = wave_sum(all);
      }
    }
    const float p = m ? expf(key_score(m >> 16) - top) : 0.f;
    chosen += p;
    if (lane == j) {
      best = m;
      mine = p;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (key[i] == m) key[i] = 0;
  }
  if (lane < k) {
    const int e = best ? (int)(0xFFFFu - (best & 0xFFFFu)) : -1;
    const float total = renormalize ? chosen : all;
    experts[lane] = e;
    weights[lane] = best ? mine / total : 0.f;
    if (e >= 0) atomicAdd(counts + e, 1);
  }
}

struct RouteArgs {
  const uint16_t* logits;
  int64_t ldl;
  int T, E, k, renormalize, tokens;
  int32_t* experts;
  float* weights;
  int32_t *offsets, *rows, *pos, *hist;
};

// Choose (or read) a stretch's experts and count them.
template <int V>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  __shared__ int counts[kMaxE];
  const int wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
  __syncthreads();
  const int t0 = blockIdx.x * a.tokens, t1 = min(a.T, t0 + a.tokens);
  if (a.logits) {
    for (int t = t0 + wave; t < t1; t += kWaves)
      route_token<V>(a.logits + t * a.ldl, a.E, a.k, a.renormalize != 0, a.experts + (int64_t)t * a.k,
                     a.weights + (int64_t)t * a.k, counts);
  } else {
    for (int i = t0 * a.k + (int)threadIdx.x; i < t1 * a.k; i += kThreads) {
      const int e = a.experts[i];
      if (e >= 0 && e < a.E) atomicAdd(counts + e, 1);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kThreads) a.hist[(int64_t)blockIdx.x * a.E + e] = counts[e];
}

// Offsets, and the places of this stretch's pairs.
__global__ __launch_bounds__(kThreads) void group_kernel(RouteArgs a, int stretches) {
  __shared__ int base[kMaxE];           // next place of each expert's pairs in this stretch
  __shared__ int count[kWaves][kMaxE];  // pairs of each wave
  __shared__ int wave_total[kWaves];
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  // totals of all stretches, and of those before this one
  int all = 0, before = 0;
  if (tid < a.E)
    for (int s = 0; s < stretches; ++s) {
      const int c = a.hist[(int64_t)s * a.E + tid];
      all += c;
      before += s < (int)blockIdx.x ? c : 0;
    }
  int scan = all;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(scan, d, kWave);
    if (lane >= d) scan += o;
  }
  if (lane == 63) wave_total[wave] = scan;
  __syncthreads();
  int lead = 0, used = 0;
  for (int w = 0; w < kWaves; ++w) {
    lead += w < wave ? wave_total[w] : 0;
    used += wave_total[w];
  }
  if (tid < a.E) {
    const int off = lead + scan - all;
    base[tid] = off + before;
    if (blockIdx.x == 0) {
      a.offsets[tid] = off;
      if (tid == a.E - 1) a.offsets[a.E] = off + all;
    }
  }
  const int n0 = blockIdx.x * a.tokens * a.k, n1 = min(a.T, (int)(blockIdx.x + 1) * a.tokens) * a.k;
  // places past the last pair
  for (int i = n0 + tid; i < n1; i += kThreads)
    if (i >= used) a.rows[i] = -1;
  for (int i0 = n0; i0 < n1; i0 += kThreads) {
    __syncthreads();
    for (int i = tid; i < kWaves * a.E; i += kThreads) count[i / a.E][i % a.E] = 0;
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
    if (has && rank == 0) count[wave][e] = __popcll(same);
    __syncthreads();
    int place = -1;
    if (has) {
      place = base[e] + rank;
      for (int w = 0; w < wave; ++w) place += count[w][e];
    }
    if (i < n1) a.pos[i] = place;
    if (has) a.rows[place] = i;
    __syncthreads();
    for (int x = tid; x < a.E; x += kThreads) {
      int c = 0;
      for (int w = 0; w < kWaves; ++w) c += count[w][x];
      base[x] += c;
    }
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
  const int stretches = (L.T + a.tokens - 1) / a.tokens;
  const int v = L.logits ? (L.E + 63) / 64 : 1;
  const dim3 grid((unsigned)stretches), block(kThreads);
  if (stretches > 0) {
    if (v <= 1) hipLaunchKernelGGL(route_kernel<1>, grid, block, 0, st, a);
    else if (v <= 2) hipLaunchKernelGGL(route_kernel<2>, grid, block, 0, st, a);
    else if (v <= 4) hipLaunchKernelGGL(route_kernel<4>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(route_kernel<8>, grid, block, 0, st, a);
  }
  hipLaunchKernelGGL(group_kernel, dim3((unsigned)(stretches > 0 ? stretches : 1)), block, 0, st, a, stretches);
}

}  // namespace ss
