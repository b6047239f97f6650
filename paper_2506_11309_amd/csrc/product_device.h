// Device code that the products with 4-bit and 8-bit matrices share: which rows a
// workgroup owns, what they read, and how results are written.
#pragma once
#include "product_internal.h"
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

// A lane offset past the end of every buffer of activations (they stay below 2 GiB):
// such a load gives zeros.  The uniform offset beside it may not count in the range
// check: it stays inside the buffer, and is 0 where all lanes are outside.  (Of a
// matrix of more than 2 GiB the load reads other codes of it, which then meet rows
// of zeros or none.)
constexpr uint32_t kOutside = 0x80000000u;

// what a product's kernels know of its rows and results
struct ProductArgs {
  int M, N, Nt;         // Nt: column tiles (16)
  const int32_t* map;   // {expert, first row, rows, 0} per row block, or null
  const int32_t* rows;
  int div;
  uint16_t* y;
  int64_t ldy;
  const uint16_t* res;
  int64_t ldr;
  float* part;
  void* ws;
  int col_blocks;
  int split;  // shares of K, each with its own part [M][N]
  bool past;  // results go past the caches
  // rows quantised by the product itself
  const uint16_t* x;
  uint32_t x_row, x_bytes;  // bytes from row to row, of all rows
  const int32_t* offsets;
  int E;
};

__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __expf(-g)); }

// the row block of a workgroup: expert, first output row, number of rows
struct RowBlock {
  int e, m0, n;
};
__device__ __forceinline__ RowBlock row_block(const ProductArgs& a, int rb, int TM) {
  if (!a.map) return RowBlock{0, rb * TM, min(TM, a.M - rb * TM)};
  // written by an earlier launch: read through the scalar cache
  const auto* p = (const __attribute__((address_space(4))) int32_t*)(a.map + 4 * ((int64_t)rb + 1));
  return RowBlock{p[0], p[1], p[2]};
}

// The same from the offsets (as RowMap describes it), by each wave for itself.
__device__ __forceinline__ RowBlock find_block(const ProductArgs& a, int rb, int TM, bool first) {
  if (!a.offsets) return RowBlock{0, rb * TM, min(TM, a.M - rb * TM)};
  const int lane = lane_id();
  RowBlock r{0, 0, 0};
  bool bad = false;
  int base = 0;
  for (int e0 = 0; e0 < a.E; e0 += kWave) {
    const int e = e0 + lane;
    const int lo = e < a.E ? a.offsets[e] : 0, hi = e < a.E ? a.offsets[e + 1] : 0;
    bad = bad || __any(lo < 0 || hi < lo || hi > a.M || (e == 0 && lo != 0));
    const int n = bad ? 0 : (hi - lo + TM - 1) / TM;
    const int s = wave_scan_add(n);
    const uint64_t past = __ballot(base + s > rb);
    if (past && r.n == 0) {
      const int l = __builtin_ctzll(past);
      r.e = e0 + l;
      r.m0 = __builtin_amdgcn_readlane(lo + (rb - (base + s - n)) * TM, l);
      r.n = min(TM, __builtin_amdgcn_readlane(hi, l) - r.m0);
    }
    base += __builtin_amdgcn_readlane(s, 63);
  }
  if (first && lane == 0) {  // one wave of the launch
    if (bad) report_error(a.ws, SWIFTSPEC_DEVERR_BAD_GROUPS);
    int32_t* map = const_cast<int32_t*>(a.map);
    map[0] = !bad;
    map[1] = bad ? 0 : a.offsets[a.E];
  }
  if (bad) r.n = 0;
  return RowBlock{__builtin_amdgcn_readfirstlane(r.e), __builtin_amdgcn_readfirstlane(r.m0), __builtin_amdgcn_readfirstlane(r.n)};
}

// Workgroup -> row and column block of a tile.  Tiles are taken in bands of 4 row
// blocks, column by column, and stretches of 32 of them (what a chiplet's
// compute units run at one time) go to the 8 chiplets in turn, as workgroups do:
// what a chiplet reads is then a few row blocks and 8 column blocks, out of its
// own L2.  Of one matrix the last tiles, fewer than 256, go to the chiplets in 8
// stretches as well (128 rows of 8192 x 8192 in 8 bits 38.5 -> 32.0 us, 384 rows 55 ->
// 50; in 4 bits 25.2 -> 21.8 and 34.4 -> 32.0, 512 rows of 8192 x 28672 82 -> 73, 3000 of
// 4096 x 4096 and 8192 of 8192 x 8192 the same); of experts one by one, so that the empty
// row blocks at the end of their list are no chiplet's alone (down for 100 tokens of 4
// experts 4096 x 8192 43 against 58 us).
__device__ __forceinline__ void place_of(const ProductArgs& a, int& rb, int& cb) {
  const int all = gridDim.x, x = blockIdx.x & 7, s = blockIdx.x >> 3;
  const int whole = all & ~255, rest = all - whole;
  int id = blockIdx.x;
  if (id < whole) id = (((s >> 5) << 3) + x) * 32 + (s & 31);
  else if (!a.map && id - whole < (rest & ~7)) id = whole + x * (rest >> 3) + (s - (whole >> 3));
  const int band = id / (4 * a.col_blocks), in = id - band * 4 * a.col_blocks;
  const int high = min(4, all / a.col_blocks - 4 * band);
  rb = 4 * band + in % high;
  cb = in / high;
}

// activation row that output row m reads, or -1 where the caller's list is wrong
__device__ __forceinline__ int source_of(const ProductArgs& a, int listed) {
  const uint32_t r = (uint32_t)listed;
  if (r >= (uint32_t)a.M) {
    report_error(a.ws, SWIFTSPEC_DEVERR_BAD_GROUPS);
    return -1;
  }
  return (int)(r / (uint32_t)a.div);
}
__device__ __forceinline__ int source_row(const ProductArgs& a, int m) { return a.rows ? source_of(a, a.rows[m]) : m; }

// four columns n .. n + 3 of output row m
__device__ __forceinline__ u32x2 residual(const ProductArgs& a, int64_t m, int n) {
  return *reinterpret_cast<const u32x2*>(a.res + m * a.ldr + n);
}
__device__ __forceinline__ void add_residual(f32x4& v, u32x2 r) {
  v[0] += h2f((uint16_t)r[0]);
  v[1] += h2f((uint16_t)(r[0] >> 16));
  v[2] += h2f((uint16_t)r[1]);
  v[3] += h2f((uint16_t)(r[1] >> 16));
}
__device__ __forceinline__ u32x2 pack4(const f32x4& v) {
  return u32x2{f2h(v[0]) | (uint32_t)f2h(v[1]) << 16, f2h(v[2]) | (uint32_t)f2h(v[3]) << 16};
}
// 16 bytes to an address of 8-byte alignment
__device__ __forceinline__ void store_rows16(uint16_t* p, const u32x4& v, bool past) {
  typedef uint32_t Line __attribute__((ext_vector_type(4), aligned(8)));
  if (past) __builtin_nontemporal_store(v, reinterpret_cast<Line*>(p));
  else *reinterpret_cast<Line*>(p) = v;
}
template <Epilogue EPI>
__device__ __forceinline__ void write_out(const ProductArgs& a, int64_t m, int n, f32x4 v) {
  if constexpr (EPI == OUT_ROWS)
    *reinterpret_cast<f32x4*>(a.part + m * a.N + n) = v;
  else
    *reinterpret_cast<u32x2*>(a.y + m * a.ldy + n) = pack4(v);
}

// One workgroup writes the row blocks of a product (RowMap).
__device__ inline void write_map(const RowMap& m) {
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

}  // namespace ss
