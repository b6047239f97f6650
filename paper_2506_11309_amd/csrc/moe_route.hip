// Router of a mixture of experts: softmax and top-k of each token's scores, and
// the stable grouping of the (token, slot) pairs by expert.
//
// Scores are compared as 16-bit keys that ascend with the value (-0 as +0)
// above the complement of the index, so that one unsigned maximum gives the
// largest score and, among equals, the lowest index.  -inf and NaN are masked:
// their key is 0 and they have no share of the softmax.
// The grouping is a counting sort: each workgroup counts its unit of tokens'
// pairs per expert; a second launch adds the counts of the units before its own
// and ranks its pairs in order (few tokens: one workgroup, one launch).  Counts are
// integers, so the order of the LDS atomics that add them does not show.
// Bound by latency: launches, dependent reads, k rounds of row maxima.  64 tokens,
// 8 of 64 experts: 4.6 to 5 us in one launch; 16000 tokens, 8 of 256 (8 MB of
// scores): 7.7 us to choose and count, 7.3 us to place; 8 of 512 18.8 and 9.6 us (a
// lane's 32 scores and both ways of reading them spill to scratch); of given experts
// 1.9 us to count for 256, 3.1 us for 64 tokens in one launch.
#include "mx4_device.h"
#include "mx4_internal.h"

namespace ss {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxE = SWIFTSPEC_MAX_EXPERTS;
constexpr int kUnits = 2;          // units that a workgroup groups

// Tokens of a unit: as many as its waves take at one time, so that a prompt fills
// the chip, but at most 256 units (each grouping workgroup reads all their
// counts) as long as a unit's counts fit 16 bits.
constexpr int kLeast = 4 * kWaves;
inline int unit_tokens(int T, int k) {
  const int most = 65535 / k, need = (T + 255) / 256;
  return need < kLeast ? kLeast : need > most ? most : need;
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
  int32_t *offsets, *rows, *pos;
  uint16_t* hist;  // [units][E rounded up to 4]
};

// 16 lanes take the top k of a token's row, V scores each (in whole 16-byte pieces,
// 8 (16 q + lane) .. + 7, where rows are aligned and wide enough), so that a wave
// routes four tokens and its reductions stay within the rows of 16 lanes that the
// ALU shifts in.  Lane j < k keeps the j-th expert.  Where t >= T nothing is written.
template <int V>
__device__ __forceinline__ void route_token(const RouteArgs& a, int t, int* counts, int16_t* chosen) {
  const int l = lane_id() & 15;
  const bool there = t < a.T;
  const uint16_t* row = a.logits + (int64_t)(there ? t : 0) * a.ldl;
  uint32_t key[V];
  const bool lines = V >= 8 && a.lines;
  if (!lines) {
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
      if (e + 8 <= a.E) {
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
    const int e = lines ? 8 * (16 * (i >> 3) + l) + (i & 7) : l + 16 * i;
    const uint32_t s = score_key(key[i]);
    key[i] = s ? s << 16 | (0xFFFFu - (uint32_t)e) : 0u;
  }
  // the j-th largest key, all keys that are there being different: the largest
  // difference, modulo 2^32, to the one before it is that of the next below
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) m = max(m, key[i]);
  m = row_max(m);
  const float top = m ? key_score(m >> 16) : 0.f;
  uint32_t best = l == 0 ? m : 0u;
  for (int j = 1; j < a.k; ++j) {
    uint32_t d = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) d = max(d, key[i] - m);
    d = row_max(d);
    m = m ? m + d : 0u;
    if (l == j) best = m;
  }
  const float mine = best ? expf(key_score(best >> 16) - top) : 0.f;
  float total = mine;
  if (!a.renormalize) {
    total = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (key[i]) total += expf(key_score(key[i] >> 16) - top);
  }
  total = row_sum(total);
  if (l < a.k && there) {
    const int e = best ? (int)(0xFFFFu - (best & 0xFFFFu)) : -1;
    a.experts[(int64_t)t * a.k + l] = e;
    a.weights[(int64_t)t * a.k + l] = best ? mine / total : 0.f;
    if (chosen) chosen[t * a.k + l] = (int16_t)e;
    if (e >= 0) atomicAdd(counts + e, 1);
  }
}

// Choose (or read) the experts of tokens t0 .. t1 and count them; `chosen` (LDS,
// nullable) receives them too, -1 for none.
template <int V>
__device__ __forceinline__ void route_tokens(const RouteArgs& a, int t0, int t1, int* counts, int16_t* chosen) {
  const int threads = blockDim.x;
  for (int e = threadIdx.x; e < a.E; e += threads) counts[e] = 0;
  __syncthreads();
  if (a.logits) {
    for (int t = t0 + 4 * (int)(threadIdx.x >> 6); t < t1; t += threads / 16) {
      const int mine = t + (lane_id() >> 4);
      route_token<V>(a, mine < t1 ? mine : a.T, counts, chosen);
    }
  } else {
    for (int i = t0 * a.k + (int)threadIdx.x; i < t1 * a.k; i += threads) {
      const int e = a.experts[i];
      const bool has = e >= 0 && e < a.E;
      if (chosen) chosen[i] = (int16_t)(has ? e : -1);
      if (has) atomicAdd(counts + e, 1);
    }
  }
  __syncthreads();
}

struct GroupLds {
  int base[kMaxE];           // next place of each expert's pairs
  int count[kWaves][kMaxE];  // pairs of each wave
  int wave_total[kWaves];
};

// The places of the pairs of tokens t0 .. t1.  Thread e brings the number of expert
// e's pairs, of all tokens and of those before t0.
__device__ __forceinline__ void group_tokens(const RouteArgs& a, int t0, int t1, int all, int before, bool writes_offsets,
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

// Few tokens (up to 1024 pairs): everything in one workgroup.
template <int V>
__global__ __launch_bounds__(kThreads) void route_one_kernel(RouteArgs a) {
  __shared__ int counts[kMaxE];
  __shared__ int16_t chosen[kThreads];
  __shared__ GroupLds s;
  route_tokens<V>(a, 0, a.T, counts, chosen);
  group_tokens(a, 0, a.T, (int)threadIdx.x < a.E ? counts[threadIdx.x] : 0, 0, true, chosen, -1, s);
}

// More: count, then place.
template <int V>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  __shared__ int counts[kMaxE];
  const int t0 = blockIdx.x * a.tokens;
  route_tokens<V>(a, t0, min(a.T, t0 + a.tokens), counts, nullptr);
  const int Ep = (a.E + 3) & ~3;
  for (int e = threadIdx.x; e < Ep; e += kThreads) a.hist[(int64_t)blockIdx.x * Ep + e] = e < a.E ? (uint16_t)counts[e] : 0;
}

__global__ __launch_bounds__(kThreads) void group_kernel(RouteArgs a, int units) {
  __shared__ int part_all[kThreads][4], part_before[kThreads][4];
  __shared__ GroupLds s;
  // four experts a thread, a power of two of threads side by side, the units
  // shared out between up to 32 parts of the workgroup
  const int tid = threadIdx.x, E4 = (a.E + 3) >> 2, wide = 1 << (32 - __builtin_clz(max(E4, 2) - 1));
  const int part = tid / wide, parts = min(kThreads / wide, 32), e4 = tid - part * wide;
  const int u0 = kUnits * blockIdx.x;
  const int64_t t0 = (int64_t)u0 * a.tokens, t1 = t0 + (int64_t)kUnits * a.tokens;
  const int64_t mine = t0 * a.k + tid;  // this thread's first pair: read beside the counts
  const int e_first = mine < (int64_t)a.T * a.k ? a.experts[mine] : -1;
  int n[4] = {}, b[4] = {};
  if (part < parts && e4 < E4) {
#pragma unroll 8
    for (int i = part; i < units; i += parts) {
      const u32x2 c = *reinterpret_cast<const u32x2*>(a.hist + ((int64_t)i * E4 + e4) * 4);
      const int v[4] = {(int)(c[0] & 0xFFFFu), (int)(c[0] >> 16), (int)(c[1] & 0xFFFFu), (int)(c[1] >> 16)};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        n[q] += v[q];
        b[q] += i < u0 ? v[q] : 0;
      }
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    part_all[tid][q] = n[q];
    part_before[tid][q] = b[q];
  }
  __syncthreads();
  int all = 0, before = 0;
  if (tid < a.E)
    for (int p = 0; p < parts; ++p) {
      all += part_all[p * wide + (tid >> 2)][tid & 3];
      before += part_before[p * wide + (tid >> 2)][tid & 3];
    }
  group_tokens(a, (int)t0, (int)(t1 < a.T ? t1 : a.T), all, before, blockIdx.x == 0, nullptr, e_first, s);
}

template <int V>
void launch_route(const RouteArgs& a, hipStream_t st) {
  // One launch takes 64 tokens at a time on one compute unit: 256 tokens of 64
  // experts (k = 2) 7.8 against 8.3 us with two launches, 371 10.2 against 8.3; of
  // 256 experts 96 tokens 7.6 against 8.7, 128 9.4 against 9.0.
  const int most = !a.logits ? kThreads : V <= 4 ? 4 * kLeast : kLeast + kLeast / 2;
  if ((int64_t)a.T * a.k <= kThreads && a.T <= most) {
    hipLaunchKernelGGL(route_one_kernel<V>, dim3(1), dim3(kThreads), 0, st, a);
    return;
  }
  const int units = (a.T + a.tokens - 1) / a.tokens;
  hipLaunchKernelGGL(route_kernel<V>, dim3((unsigned)units), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(group_kernel, dim3((unsigned)((units + kUnits - 1) / kUnits)), dim3(kThreads), 0, st, a, units);
}

}  // namespace

size_t route_hist_bytes(int T, int E, int k) {
  // what any smaller number of tokens may need too: up to 256 units of the least
  // size, more only of the largest
  const int64_t most = 65535 / k;
  const int64_t small = (T + kLeast - 1) / kLeast, large = (T + most - 1) / most;
  const int64_t units = small < 256 ? small : large > 256 ? large : 256;
  return (size_t)units * ((E + 3) / 4 * 4) * sizeof(uint16_t);
}

void launch_moe_route(const RouteLaunch& L, hipStream_t st) {
  RouteArgs a;
  a.logits = L.logits;
  a.ldl = L.ldl;
  a.T = L.T;
  a.E = L.E;
  a.k = L.k;
  a.renormalize = L.renormalize;
  a.tokens = unit_tokens(L.T, L.k);
  a.experts = L.experts;
  a.weights = L.weights;
  a.offsets = L.offsets;
  a.rows = L.rows;
  a.pos = L.pos;
  a.hist = L.hist;
  a.lines = (reinterpret_cast<uintptr_t>(L.logits) & 15) == 0 && L.ldl % 8 == 0;
  const int v = L.logits ? (L.E + 15) / 16 : 1;  // scores of a lane
  if (v <= 1) launch_route<1>(a, st);
  else if (v <= 2) launch_route<2>(a, st);
  else if (v <= 4) launch_route<4>(a, st);
  else if (v <= 8) launch_route<8>(a, st);
  else if (v <= 16) launch_route<16>(a, st);
  else launch_route<32>(a, st);
}

}  // namespace ss
