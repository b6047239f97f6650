// Router of a mixture of experts by probabilities or gates: scores, a bias for
// balance, groups of experts, top-k, renormalised weights; then the grouping of
// moe_route.hip.
//
// s_e is the softmax or the sigmoid of a score, computed in 64 bits and rounded to 32;
// c_e = s_e + b_e in 32 bits decides.  64 bits, because experts whose c differ by a
// step of 2^-24 must come out in the same order whatever computes them.  A group's
// value is its largest c, or the sum of its two largest; the best groups' experts are
// compared.  c is compared as a 32-bit key that ascends with the value, 0 where the
// expert is masked; equal keys go to the lower index.
// 16 lanes take a token, so that a wave routes four and its reductions stay within the
// rows of lanes that the ALU shifts in.  Each lane holds neighbouring experts: where
// whole lanes make up a group its value is found among them, otherwise through LDS.
// Bound by latency and the ALU: 64 tokens, 6 of 64 experts, 8.1 us in one launch; 16000
// tokens, 8 of 256 (16 MB of scores) 18.9 us to choose and count, 7.4 us to place.  Of
// the former the 64-bit gates are 3 us, the eight rounds of maxima 6, the groups 1; with
// the compiler's exponential and divisions, whose constants spilled, it was 170.
#include "moe_group_device.h"

namespace ss {

namespace {

struct ScoredArgs : GroupArgs {
  const void* logits;
  int64_t ldl;
  const float* bias;
  int groups, size, top_groups, best;  // size: experts of a group
  uint32_t per;                        // ceil(2^18 / size): e * per >> 18 is e's group
  int block;                           // experts of a lane: e = lane * block + i
  int lanes;                           // lanes of a group if that is 1, 2, 4 or 8, otherwise 0
  bool lines;                          // scores and bias can be read four at a time
  bool renormalize;
  float scale;
};

__device__ __forceinline__ uint32_t row_min(uint32_t v) { return ~row_max(~v); }
__device__ __forceinline__ double row_sum(double v) {
  auto rotate = [](double d, auto by) {
    constexpr int kBy = decltype(by)::value;
    const uint64_t b = bitcast<uint64_t>(d);
    return bitcast<double>((uint64_t)rotated<kBy>((uint32_t)(b >> 32)) << 32 | rotated<kBy>((uint32_t)b));
  };
  v += rotate(v, std::integral_constant<int, 8>{});
  v += rotate(v, std::integral_constant<int, 4>{});
  v += rotate(v, std::integral_constant<int, 2>{});
  return v + rotate(v, std::integral_constant<int, 1>{});
}

// ascending key of a float, 0 for -inf and NaN
__device__ __forceinline__ uint32_t value_key(float c) {
  const uint32_t b = bitcast<uint32_t>(c);
  const uint32_t key = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);  // all bits of a negative value, the sign of others
  return c > -__builtin_inff() ? key : 0u;
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return bitcast<float>(key ^ (~(uint32_t)((int32_t)key >> 31) | 0x80000000u));
}

// e^x in 64 bits for -200 <= x <= 200: x = n log 2 + r with |r| <= 0.3466, e^r by its
// series up to r^12 (what is left out is below 2^-52).  The coefficients stay in scalar
// registers: the compiler would move each into a vector register at every use.
struct Exp64 {
  double c[11];
  __device__ __forceinline__ Exp64() {
    double f = 1.0;
#pragma unroll
    for (int i = 0; i < 11; ++i) {
      f /= i + 2;  // 1 / 2! ... 1 / 12!
      c[i] = f;
      asm volatile("" : "+s"(c[i]));
    }
  }
  __device__ __forceinline__ double operator()(double x) const {
    const float n = __builtin_rintf((float)x * 1.44269504f);
    double r = __builtin_fma((double)n, -0x1.62e42fefa39efp-1, x);
    r = __builtin_fma((double)n, -0x1.abc9e3b39803fp-56, r);
    double y = c[10];
#pragma unroll
    for (int i = 9; i >= 0; --i) y = __builtin_fma(y, r, c[i]);
    y = __builtin_fma(y, r, 1.0);
    y = __builtin_fma(y, r, 1.0);
    return __builtin_amdgcn_ldexp(y, (int)n);
  }
};
// 1 / x for x >= 1, two of Newton's steps behind the instruction's own 2^-14 or better
__device__ __forceinline__ double reciprocal64(double x) {
  double y = __builtin_amdgcn_rcp(x);
  y = __builtin_fma(__builtin_fma(-x, y, 1.0), y, y);
  return __builtin_fma(__builtin_fma(-x, y, 1.0), y, y);
}

__device__ __forceinline__ float finite(float x, float most) { return x == __builtin_inff() ? most : x; }
// score e of a row, +inf as the largest finite value
template <typename T>
__device__ __forceinline__ float score_at(const T* row, int e) {
  if constexpr (sizeof(T) == 2) return finite(h2f(row[e]), 65504.f);
  else return finite(row[e], 3.4028234663852886e38f);
}
// scores e .. e + 3
template <typename T>
__device__ __forceinline__ void scores_at(const T* row, int e, float* x) {
  if constexpr (sizeof(T) == 2) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(row + e);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = finite(h2f((uint16_t)(v[i >> 1] >> (16 * (i & 1)))), 65504.f);
  } else {
    const f32x4 v = *reinterpret_cast<const f32x4*>(row + e);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = finite(v[i], 3.4028234663852886e38f);
  }
}

// The two largest of a and of what another lane holds.
__device__ __forceinline__ void merge_two(uint32_t& first, uint32_t& second, uint32_t f, uint32_t s) {
  second = max(min(first, f), max(second, s));
  first = max(first, f);
}
template <int kCtrl>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xF, 0xF, true);
}
template <int kBy>
__device__ __forceinline__ void count_before(uint32_t v, uint32_t g, int& n) {
  // the lane kBy before, round the row, and its group
  const uint32_t w = rotated<kBy>(v), o = rotated<kBy>(g);
  n += w > v || (w == v && o < g);
  if constexpr (kBy < 15) count_before<kBy + 1>(v, g, n);
}

// Whether this lane's group of a.lanes neighbours is among the best: the lanes' two
// largest keys are merged, and the lanes of better groups counted.
template <int V>
__device__ __forceinline__ bool group_taken(const ScoredArgs& a, const uint32_t (&key)[V]) {
  uint32_t first = 0, second = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) merge_two(first, second, key[i], 0u);
  if (a.lanes >= 2) merge_two(first, second, from_lane<0xB1>(first), from_lane<0xB1>(second));    // lane ^ 1
  if (a.lanes >= 4) merge_two(first, second, from_lane<0x4E>(first), from_lane<0x4E>(second));    // lane ^ 2
  if (a.lanes >= 8) merge_two(first, second, from_lane<0x141>(first), from_lane<0x141>(second));  // the other four of eight
  if (a.best == 2 && second) first = value_key(key_value(first) + key_value(second));
  const uint32_t g = (uint32_t)(lane_id() & 15) / (uint32_t)a.lanes;
  int n = 0;
  count_before<1>(first, g, n);
  return n < a.top_groups * a.lanes;
}

// v[i] = v[i + N], round the array: a loop over N values at a time finds them in the same
// registers, where unrolled it would be a page of code that a short kernel waits for
template <int V, int N, typename T>
__device__ __forceinline__ void rotate(T (&v)[V]) {
  if constexpr (N < V) {
    T t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = v[(i + N) % V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = t[i];
  }
}

// 16 lanes take a token, up to V neighbouring scores each.  room: V * 16 words of LDS of
// this token.  Lane j < k keeps the j-th expert.  Where t >= T nothing is written.
template <int V, bool SIGMOID, typename T>
__device__ __forceinline__ void route_scored_token(const ScoredArgs& a, int t, int* counts, int16_t* chosen, uint32_t* room) {
  const int l = lane_id() & 15, e0 = l * a.block, n = max(0, min(a.block, a.E - e0));
  constexpr int kStep = V < 4 ? V : 4;
  const bool there = t < a.T;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)(there ? t : 0) * a.ldl;
  float x[V];
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
  const bool lines = V >= 4 && a.lines;
  if (lines) {
#pragma unroll
    for (int i = 0; i < V; i += 4)
      if (i < n) scores_at(row, e0 + i, x + i);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) x[i] = score_at(row, e0 + i);
  }
  const Exp64 exp64;
  float top = 0.f;
  // e^-v of a gate, e^(v - top) of a probability; beyond these limits it is 0 or 1 in 32
  // bits.  The difference has more than 24 bits.
  auto power = [&](float v) {
    return exp64(SIGMOID ? (double)__builtin_fminf(__builtin_fmaxf(-v, -100.f), 200.f) : __builtin_fmax((double)v - (double)top, -200.0));
  };
  double share = 1.0;  // of a softmax: 1 / the sum
  uint32_t key[V];
  if constexpr (!SIGMOID) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) m = max(m, value_key(x[i]));
    m = row_max(m);
    top = m ? key_value(m) : 0.f;
    double total = 0.0;
#pragma unroll 1
    for (int q = 0; q < V; q += kStep) {
#pragma unroll
      for (int i = 0; i < kStep; ++i) {
        double p = power(x[i]);
        asm volatile("" : "+v"(p));  // one after the other: side by side the 64-bit values would not fit the registers
        total += x[i] > -__builtin_inff() ? p : 0.0;
      }
      rotate<V, kStep>(x);
    }
    total = row_sum(total);
    share = total >= 1.0 ? reciprocal64(total) : 0.0;
  }
  auto score = [&](float v) { return (float)(SIGMOID ? reciprocal64(1.0 + power(v)) : power(v) * share); };
#pragma unroll 1
  for (int q = 0; q < V; q += kStep) {
    float b[kStep] = {};
    if (a.bias) {
      if (lines) {
        if (q < n) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(a.bias + e0 + q);
#pragma unroll
          for (int i = 0; i < kStep; ++i) b[i] = v[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < kStep; ++i) b[i] = q + i < n ? a.bias[e0 + q + i] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      float s = score(x[i]);
      asm volatile("" : "+v"(s));
      // a masked score makes the sum -inf
      key[i] = value_key(x[i] > -__builtin_inff() ? s + b[i] : -__builtin_inff());
    }
    rotate<V, kStep>(x);
    rotate<V, kStep>(key);
  }
  if (a.lanes) {
    if (!group_taken<V>(a, key)) {
#pragma unroll
      for (int i = 0; i < V; ++i) key[i] = 0;
    }
  } else if (a.top_groups < a.groups) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) room[e0 + i] = key[i];
    __builtin_amdgcn_wave_barrier();
    for (int g = l; g < a.groups; g += 16) {
      // its two largest; the lanes start at different members, so that they read
      // different banks
      uint32_t* mine = room + g * a.size;
      uint32_t first = 0, second = 0;
      int at = l % a.size;
      for (int i = 0; i < a.size; ++i) {
        const uint32_t v = mine[at];
        second = max(second, min(first, v));
        first = max(first, v);
        at = at + 1 == a.size ? 0 : at + 1;
      }
      if (a.best == 2 && second) first = value_key(key_value(first) + key_value(second));
      mine[0] = first;  // only this lane reads it as a member
    }
    __builtin_amdgcn_wave_barrier();
    uint32_t taken = 0;
    for (int g = l, i = 0; g < a.groups; g += 16, ++i) {
      const uint32_t v = room[g * a.size];
      int before = 0;
      for (int o = 0; o < a.groups; ++o) {
        const uint32_t w = room[o * a.size];
        before += w > v || (w == v && o < g);
      }
      taken |= (uint32_t)(before < a.top_groups) << i;
    }
    __builtin_amdgcn_wave_barrier();
    for (int g = l, i = 0; g < a.groups; g += 16, ++i) room[g * a.size] = taken >> i & 1;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = min(e0 + i, a.E - 1);
      if (!room[((uint32_t)e * a.per >> 18) * a.size]) key[i] = 0;
    }
    __builtin_amdgcn_wave_barrier();
  }
  int mine = -1;
  for (int j = 0; j < a.k; ++j) {
    uint32_t m = 0, e = ~0u;
#pragma unroll
    for (int i = 0; i < V; ++i) m = max(m, key[i]);
    m = row_max(m);
#pragma unroll
    for (int i = V - 1; i >= 0; --i) e = key[i] == m ? (uint32_t)(e0 + i) : e;
    e = row_min(e);
    if (!m) break;  // of this token: its lanes leave together
    if (l == j) mine = (int)e;
#pragma unroll
    for (int i = 0; i < V; ++i)
      key[i] = (uint32_t)i == e - (uint32_t)e0 ? 0u : key[i];
  }
  float s = 0.f;
  if (mine >= 0) s = score(score_at(row, mine));
  const double sum = a.renormalize ? row_sum((double)s) : 1.0;
  if (l < a.k && there) {
    a.experts[(int64_t)t * a.k + l] = mine;
    a.weights[(int64_t)t * a.k + l] = mine >= 0 && sum > 0.0 ? (float)((double)s / sum * (double)a.scale) : 0.f;
    if (chosen) chosen[t * a.k + l] = (int16_t)mine;
    if (mine >= 0) atomicAdd(counts + mine, 1);
  }
}

// Choose the experts of tokens t0 .. t1 and count them; `chosen` (LDS, nullable)
// receives them too, -1 for none.  room: V * 16 words for each of 64 tokens.
template <int V, bool SIGMOID, typename T>
__device__ __forceinline__ void route_scored_tokens(const ScoredArgs& a, int t0, int t1, int* counts, int16_t* chosen, uint32_t* room) {
  for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
  __syncthreads();
  for (int t = t0 + 4 * (int)(threadIdx.x >> 6); t < t1; t += kThreads / 16) {
    const int mine = t + (lane_id() >> 4);
    route_scored_token<V, SIGMOID, T>(a, mine < t1 ? mine : a.T, counts, chosen, room + (threadIdx.x >> 4) * (V * 16));
  }
  __syncthreads();
}

// Few tokens (up to 1024 pairs): everything in one workgroup.
template <int V, bool SIGMOID, typename T>
__global__ __launch_bounds__(kThreads) void route_scored_one_kernel(ScoredArgs a) {
  __shared__ int counts[kMaxE];
  __shared__ int16_t chosen[kThreads];
  __shared__ union {
    uint32_t room[kThreads / 16 * V * 16];
    GroupLds group;
  } s;
  route_scored_tokens<V, SIGMOID, T>(a, 0, a.T, counts, chosen, s.room);
  group_tokens(a, 0, a.T, (int)threadIdx.x < a.E ? counts[threadIdx.x] : 0, 0, true, chosen, -1, s.group);
}

// More: count, then place.
template <int V, bool SIGMOID, typename T>
__global__ __launch_bounds__(kThreads) void route_scored_kernel(ScoredArgs a) {
  __shared__ int counts[kMaxE];
  __shared__ uint32_t room[kThreads / 16 * V * 16];
  const int t0 = blockIdx.x * a.tokens;
  route_scored_tokens<V, SIGMOID, T>(a, t0, min(a.T, t0 + a.tokens), counts, nullptr, room);
  const int Ep = (a.E + 3) & ~3;
  for (int e = threadIdx.x; e < Ep; e += kThreads) a.hist[(int64_t)blockIdx.x * Ep + e] = e < a.E ? (uint16_t)counts[e] : 0;
}

template <int V, bool SIGMOID, typename T>
void launch_scored(const ScoredArgs& a, hipStream_t st) {
  if ((int64_t)a.T * a.k <= kThreads && a.T <= kLeast) {
    hipLaunchKernelGGL((route_scored_one_kernel<V, SIGMOID, T>), dim3(1), dim3(kThreads), 0, st, a);
    return;
  }
  const int units = (a.T + a.tokens - 1) / a.tokens;
  hipLaunchKernelGGL((route_scored_kernel<V, SIGMOID, T>), dim3((unsigned)units), dim3(kThreads), 0, st, a);
  launch_group_units(a, units, st);
}

template <bool SIGMOID, typename T>
void launch_width(const ScoredArgs& a, hipStream_t st) {
  const int v = (a.E + 15) / 16;  // scores of a lane
  if (v <= 1) launch_scored<1, SIGMOID, T>(a, st);
  else if (v <= 2) launch_scored<2, SIGMOID, T>(a, st);
  else if (v <= 4) launch_scored<4, SIGMOID, T>(a, st);
  else if (v <= 8) launch_scored<8, SIGMOID, T>(a, st);
  else if (v <= 16) launch_scored<16, SIGMOID, T>(a, st);
  else launch_scored<32, SIGMOID, T>(a, st);
}

}  // namespace

void launch_moe_route_scored(const ScoredLaunch& L, hipStream_t st) {
  ScoredArgs a;
  static_cast<GroupArgs&>(a) = L.group;
  a.tokens = unit_tokens(a.T, a.k);
  a.logits = L.logits;
  a.ldl = L.ldl;
  a.bias = L.bias;
  a.groups = L.groups;
  a.size = a.E / L.groups;
  a.top_groups = L.top_groups;
  a.best = L.best;
  a.per = ((1u << 18) + a.size - 1) / a.size;
  a.block = (a.E + 15) / 16;
  const int lanes = a.size % a.block ? 0 : a.size / a.block;
  a.lanes = a.top_groups < a.groups && (lanes == 1 || lanes == 2 || lanes == 4 || lanes == 8) && lanes * a.groups <= 16 ? lanes : 0;
  a.lines = a.block % 4 == 0 && a.E % 4 == 0 && a.ldl % 4 == 0 && reinterpret_cast<uintptr_t>(a.logits) % (L.wide ? 16 : 8) == 0 &&
            reinterpret_cast<uintptr_t>(a.bias) % 16 == 0;
  a.renormalize = L.renormalize;
  a.scale = L.scale;
  if (L.sigmoid) L.wide ? launch_width<true, float>(a, st) : launch_width<true, uint16_t>(a, st);
  else L.wide ? launch_width<false, float>(a, st) : launch_width<false, uint16_t>(a, st);
}

}  // namespace ss
