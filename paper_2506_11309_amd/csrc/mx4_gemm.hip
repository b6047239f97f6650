// Products with microscaled 4-bit matrices (MXFP4 x MXFP4, fp32 sums), for one
// matrix or for the experts of a mixture with ragged groups of rows.
//
// y[m][n] = sum_k A[m][k] W[n][k]; both operands stay in 4 bits up to the
// block-scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4, whose lane
// kq*16 + i takes the 32 codes of row i in k block kq and that block's scale
// byte.  The weights are its first operand, so that a lane ends up with four
// consecutive columns of one output row.
#include "mx4_device.h"
#include "mx4_internal.h"

#include <algorithm>
#include <type_traits>

namespace ss {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// c += W (16 columns x 128) . A (16 rows x 128); byte J of the weights' scale word, JA of the rows'
template <int J, int JA = J>
__device__ __forceinline__ f32x4 mfma_mx4(const u32x4& w, uint32_t ws, const u32x4& a, uint32_t as, const f32x4& c) {
  const i32x8 w8 = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
  const i32x8 a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, a8, c, 4, 4, J, (int)ws, JA, (int)as);
}

// c += W (32 columns x 64) . A (32 rows x 64): lane h*32 + i holds block h of row i
template <int J>
__device__ __forceinline__ f32x16 mfma_mx4_32(const u32x4& w, uint32_t ws, const u32x4& a, uint32_t as, const f32x16& c) {
  const i32x8 w8 = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
  const i32x8 a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w8, a8, c, 4, 4, J, (int)ws, J, (int)as);
}

struct Mx4Args : ProductArgs {
  const uint8_t *w0, *w1;    // codes; the scales follow all codes
  const uint8_t *s0, *s1;
  int64_t w_stride, s_stride;  // bytes of one expert
  int G, G4;
  const uint8_t *a, *as;
  uint32_t a_bytes, as_bytes;
  int blocks;               // blocks of 32 columns of a row
};

// ------------------------------------------------------------ few rows
// W waves of a workgroup own NT column tiles (SwiGLU: NT/2 gate and NT/2 up
// tiles) over all of K and split K between them; sums meet in LDS and are
// added in wave order.  Nothing is staged: a weight block is one coalesced
// kilobyte, read once from memory by the wave that multiplies it, U groups of
// each tile at a time and the next U on their way.
// RAW: a single launch for very few rows, which each wave quantises itself as it
// reads them (66 vector instructions a group of 128 columns: 33 to each kilobyte of
// weights); the block's expert is found from the offsets.
// Bound by launch, first loads and drain for small matrices, by the weights' bytes
// for large ones: 32 rows of 8192 x 8192 (36 MB) 11.4 us, 3.1 TB/s; SwiGLU of a
// token through 8 experts 2048 x 1024 (18 MB) 8.0 us in one launch.
template <int W, int MT, int NT, int U, bool RAW, Epilogue EPI>
__global__ __launch_bounds__(64 * W) void mx4_stream_kernel(Mx4Args a) {
  constexpr bool SW = EPI == OUT_SWIGLU;
  constexpr int kC = SW ? NT / 2 : NT;
  __shared__ f32x4 red[W][MT * NT][kWave];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int rb = blockIdx.x / a.col_blocks, cb = blockIdx.x - rb * a.col_blocks;
  // RAW: at most 16 rows, whose list is read beside the offsets
  const int listed = RAW && a.rows && lane < a.M ? a.rows[lane] : 0;
  const RowBlock b = RAW ? find_block(a, rb, 16 * MT, blockIdx.x == 0 && wave == 0) : row_block(a, rb, 16 * MT);
  if (b.n <= 0) return;
  const int t0 = cb * kC;
  const int C = (a.G + U - 1) / U;  // chunks of U groups
  const int c0 = wave * C / W, c1 = (wave + 1) * C / W;
  const uint32_t wb = (uint32_t)a.w_stride, sb = (uint32_t)a.s_stride;
  const auto rw0 = buffer_rsrc(a.w0 + b.e * a.w_stride, wb), rs0 = buffer_rsrc(a.s0 + b.e * a.s_stride, sb);
  const auto rw1 = buffer_rsrc((SW ? a.w1 : a.w0) + b.e * a.w_stride, wb);
  const auto rs1 = buffer_rsrc((SW ? a.s1 : a.s0) + b.e * a.s_stride, sb);
  const auto ra = RAW ? buffer_rsrc(a.x, a.x_bytes) : buffer_rsrc(a.a, a.a_bytes);
  const auto ras = buffer_rsrc(a.as, RAW ? 0u : a.as_bytes);
  struct Stage {
    u32x4 w[U][NT], x[U][MT][RAW ? 4 : 1];
    uint32_t ws[NT], xs[MT];
  };
  auto load_weights = [&](Stage& s, int c) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // tiles past the last repeat it (their sums are not written)
      const uint32_t t = (uint32_t)min(t0 + nt % kC, a.Nt - 1);
      const bool up = SW && nt >= kC;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t g = (uint32_t)(c * U + u);
        const bool in = g < (uint32_t)a.G;
        s.w[u][nt] = buffer_load_x4(up ? rw1 : rw0, in ? (uint32_t)lane * 16u : kOutside, in ? (t * a.G + g) * 1024u : 0u);
      }
      s.ws[nt] = buffer_load_x1(up ? rs1 : rs0, (uint32_t)lane * 4u, (t * a.G4 + (uint32_t)(c * U / 4)) * 256u);
    }
  };
  // the first weights are on their way while the rows are looked up
  Stage s[2];
  if (c0 < c1) load_weights(s[0], c0);
  uint32_t va[MT], vs[MT];
  bool live[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int m = 16 * mt + r16;
    const int row = RAW && a.rows ? __shfl(listed, (b.m0 + m) & 63, kWave) : 0;
    const int src = m >= b.n ? -1 : RAW && a.rows ? source_of(a, row) : source_row(a, b.m0 + m);
    live[mt] = src >= 0;
    if constexpr (RAW) {
      va[mt] = live[mt] ? (uint32_t)src * a.x_row + (uint32_t)kq * 64u : kOutside;
    } else {
      va[mt] = live[mt] ? (uint32_t)src * (uint32_t)(a.G * 64) + (uint32_t)kq * 16u : kOutside;
      vs[mt] = live[mt] ? (uint32_t)src * (uint32_t)(a.G4 * 16) + (uint32_t)kq * 4u : kOutside;
    }
  }
  f32x4 acc[MT][NT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto load_rows = [&](Stage& s, int c) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t g = (uint32_t)(c * U + u), at = g < (uint32_t)a.G ? g : 0u;
        if constexpr (RAW) {
          const uint32_t v = (int)(4 * g) + kq < a.blocks ? va[mt] : kOutside;
#pragma unroll
          for (int q = 0; q < 4; ++q) s.x[u][mt][q] = buffer_load_x4(ra, v, at * 256u + 16u * q);
        } else {
          s.x[u][mt][0] = buffer_load_x4(ra, g < (uint32_t)a.G ? va[mt] : kOutside, at * 64u);
        }
      }
      if constexpr (!RAW) s.xs[mt] = buffer_load_x1(ras, vs[mt], (uint32_t)(c * U / 4) * 16u);
    }
  };
  auto load = [&](Stage& s, int c) {
    load_weights(s, c);
    load_rows(s, c);
  };
  // the rows' operand of group u and its scale (RAW: in byte 0)
  auto operand = [&](const Stage& s, int u, int mt, uint32_t& scale) {
    if constexpr (RAW) {
      const u32x4* v = s.x[u][mt];
      const uint32_t m = max(max(mx4_magnitude(v[0]), mx4_magnitude(v[1])), max(mx4_magnitude(v[2]), mx4_magnitude(v[3])));
      scale = mx4_scale_of(m);
      return u32x4{mx4_codes(v[0], scale), mx4_codes(v[1], scale), mx4_codes(v[2], scale), mx4_codes(v[3], scale)};
    } else {
      scale = s.xs[mt];
      return s.x[u][mt][0];
    }
  };
  auto multiply = [&](Stage& s, int c) {
    const int sh = 8 * ((c * U) & 3);  // this chunk's bytes of its scale words
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s.ws[nt] >>= sh;
    if constexpr (!RAW) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) s.xs[mt] >>= sh;
    }
    auto group = [&](auto uc) {
      constexpr int u = decltype(uc)::value;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t xs;
        const u32x4 x = operand(s, u, mt, xs);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          acc[mt][nt] = mfma_mx4<u, RAW ? 0 : u>(s.w[u][nt], s.ws[nt], x, xs, acc[mt][nt]);
      }
    };
    group(std::integral_constant<int, 0>{});
    group(std::integral_constant<int, 1>{});
    static_assert(U == 2, "groups of a chunk");
  };
  if (c0 < c1) load_rows(s[0], c0);
  // The first MT kC waves write a block of 16 x 16 results each; its residual comes
  // beside the operands.
  static_assert(MT * kC <= W, "one block a wave");
  const int mt = min(wave / kC, MT - 1), c = wave % kC;
  const int64_t m = b.m0 + 16 * mt + r16;
  const int n = 16 * (t0 + c) + 4 * kq;
  bool writes = wave < MT * kC && t0 + c < a.Nt;
#pragma unroll
  for (int j = 0; j < MT; ++j) writes = writes && (j != mt || live[j]);
  u32x2 add = {0u, 0u};
  if (EPI == OUT_RESIDUAL && writes) add = residual(a, m, n);
  for (int c = c0; c < c1; c += 2) {
    if (c + 1 < c1) load(s[1], c + 1);
    multiply(s[0], c);
    if (c + 1 >= c1) break;
    if (c + 2 < c1) load(s[0], c + 2);
    multiply(s[1], c + 1);
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) red[wave][mt * NT + nt][lane] = acc[mt][nt];
  __syncthreads();
  auto total = [&](int f) {
    f32x4 v = red[0][f][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) v += red[w][f][lane];
    return v;
  };
  if (!writes) return;
  f32x4 v = total(mt * NT + c);
  if constexpr (SW) {
    const f32x4 u = total(mt * NT + kC + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = silu(v[i]) * u[i];
  }
  if constexpr (EPI == OUT_RESIDUAL) add_residual(v, add);
  write_out<EPI>(a, m, n, v);
}

// ----------------------------------------------------------- many rows
// 4 waves (WM x WN) own a tile of 16 WM MTW rows and 16 WN NTW columns; each
// wave multiplies MTW x NTW blocks of 16, two by two through the 32 x 32 x 64
// form of the instruction (one wave a SIMD issues it at 9.0 PFLOP/s, the
// 16 x 16 x 128 form at 5.1; on random operands, at the clock that the power then
// leaves, 6.7 and 5.1).  Both operands pass through LDS, loaded there
// directly: the weights group by group as they are packed, four groups ahead;
// the activations two groups at a time, so that a row's piece is a whole
// 128-byte line however the rows are gathered.  The 16-byte pieces of a line
// stand in LDS at piece ^ (row / 2 % 8), so that a column of 16 rows covers the
// 64 banks once.  A step multiplies group g out of registers while it reads group
// g + 1 from LDS, so neither latency shows; one barrier a step.  Scale words
// cover four groups: they are loaded in the first of four steps, when every
// wave has the present ones in registers, and read in the last.
// Where the tiles are too few for the chip, K is split between workgroups whose
// parts another kernel adds in order.
// With few rows an expert it is bound by the weights: SwiGLU of 32 tokens through 8
// experts 4096 x 14336 (499 MB) 82-92 us, 5.4-6.1 TB/s.  With many no unit alone
// is the bound: with one wave a SIMD the times of a wave's matrix instructions,
// vector instructions and waits add up, and the first loads and last stores of a
// tile count where K is short.  8192 x 8192 x 8192 4.5 PFLOP/s (the instruction
// alone, on random operands: 6.7), 4001 rows of 4096 x 14336 3.7 (matrix
// instructions in 49 % of the cycles), SwiGLU of 8191 tokens through 8 of 64
// experts 2048 x 1024 in 37 %.  256 rows a tile halve the LDS reads of a product
// against 128, but one workgroup fills a compute unit's registers.
// The waits count this wave's loads in issue order.  Step g loads, in order,
// the scales of the next four groups (g % 4 == 0), the activations of groups
// g + 3 and g + 4 (g odd), the weights of group g + 4.
constexpr int kTurnRow = 144;  // bytes of a 128-byte line with its padding

template <int WM, int WN, int MTW, int NTW, Epilogue EPI>
__global__ __launch_bounds__(256, 1) void mx4_tile_kernel(Mx4Args a) {
  constexpr bool SW = EPI == OUT_SWIGLU;
  constexpr int AT = WM * MTW, WT = WN * NTW, TM = 16 * AT;
  constexpr int kA = 2 * AT / 4, kW = WT / 4, kS = (AT + WT) / 4;  // loads of a wave: two groups of rows, a group of weights, scales
  constexpr int kC = SW ? WT / 2 : WT;   // output column tiles of the workgroup
  constexpr int kCW = SW ? NTW / 2 : NTW;  // and of a wave
  static_assert(WM * WN == 4 && AT % 4 == 0 && WT % 4 == 0, "four waves load alike, rows in whole 16s");
  struct Operands {
    u32x4 ax[2][TM * 8];  // rows: two slots of two groups
    u32x4 wx[4][WT][kWave];
  };
  __shared__ Operands room;
  auto& ax = room.ax;
  auto& wx = room.wx;
  __shared__ uint32_t sc[AT + WT][kWave];
  __shared__ uint32_t row_list[4][kWave];
  __shared__ uint8_t live[TM];  // rows that are written
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave - wm * WN;
  const int r16 = lane & 15, kq = lane >> 4;
  int rb, cb;
  place_of(a, rb, cb);
  const RowBlock b = row_block(a, rb, TM);
  if (b.n <= 0) return;
  const int t0 = cb * kC;
  // this workgroup's share of K: whole scale words
  const int first = blockIdx.y * a.G4 / a.split, G4 = (blockIdx.y + 1) * a.G4 / a.split - first;
  const int G = min(a.G - 4 * first, 4 * G4);
  const uint32_t wb = (uint32_t)a.w_stride, sb = (uint32_t)a.s_stride;
  const i32x4 rw0 = raw_rsrc(a.w0 + b.e * a.w_stride, wb), rs0 = raw_rsrc(a.s0 + b.e * a.s_stride, sb);
  const i32x4 rw1 = raw_rsrc((SW ? a.w1 : a.w0) + b.e * a.w_stride, wb);
  const i32x4 rs1 = raw_rsrc((SW ? a.s1 : a.s0) + b.e * a.s_stride, sb);
  const i32x4 ra = raw_rsrc(a.a, a.a_bytes), ras = raw_rsrc(a.as, a.as_bytes);
  // This wave's loads: rows 8 i .. 8 i + 7 of its quarter of the rows, its quarter
  // of the weight tiles, the scales of its quarter of the row blocks.
  uint32_t va[kA], vs[AT / 4];
  uint32_t wt[kW];  // tile of the matrix; tile w of the workgroup: wave w / NTW, for SwiGLU a gate tile and its up tile in turn
#pragma unroll
  for (int i = 0; i < kW; ++i) {
    const int w = wave * kW + i, own = w / NTW, j = w - own * NTW;
    wt[i] = (uint32_t)min(t0 + own * kCW + (SW ? j / 2 : j), a.Nt - 1);
  }
  auto is_up = [&](int i) { return SW && ((wave * kW + i) & 1); };
  const uint32_t ax_lds = lds_address(&ax[0][0]), wx_lds = lds_address(&wx[0][0][0]), sc_lds = lds_address(&sc[0][0]);
  // load i of the rows' groups 2 p and 2 p + 1, of the weights' group g, of the
  // scales of groups 4 c .. 4 c + 3; nothing past the last group
  auto load_rows = [&](int i, int p) {
    const bool in = 2 * p < G;
    buffer_load_lds16(ra, in ? va[i] : kOutside, in ? (uint32_t)(p + 2 * first) * 128u : 0u,
                      ax_lds + (uint32_t)(p & 1) * (TM * 128u) + (uint32_t)(wave * kA + i) * 1024u);
  };
  auto load_weights = [&](int i, int g) {
    const bool in = g < G;
    buffer_load_lds16(is_up(i) ? rw1 : rw0, in ? (uint32_t)lane * 16u : kOutside, in ? (wt[i] * a.G + g + 4 * first) * 1024u : 0u,
                      wx_lds + (uint32_t)(g & 3) * (WT * 1024u) + (uint32_t)(wave * kW + i) * 1024u);
  };
  auto load_scale = [&](int i, int c) {
    const bool in = c < G4;
    if (i < AT / 4)
      buffer_load_lds4(ras, in ? vs[i] : kOutside, in ? (uint32_t)(c + first) * 16u : 0u, sc_lds + (uint32_t)(wave * (AT / 4) + i) * 256u);
    else
      buffer_load_lds4(is_up(i - AT / 4) ? rs1 : rs0, in ? (uint32_t)lane * 4u : kOutside,
                       in ? (wt[i - AT / 4] * a.G4 + c + first) * 256u : 0u, sc_lds + (uint32_t)(AT + wave * kW + i - AT / 4) * 256u);
  };
  // [2 p + h]: half h of the group (k blocks 2 h, 2 h + 1) of the blocks 2 p, 2 p + 1
  struct Ops {
    u32x4 x[MTW], w[NTW];
  };
  struct Scales {
    uint32_t x[MTW], w[NTW];
  };
  constexpr int kR = MTW + NTW;  // pieces that a wave reads
  const int r32 = lane & 31;
  const int piece = (lane >> 5) * 16 + r16, second = r32 >> 4;  // of which block of the pair
  const int row0 = 16 * wm * MTW + r32, twist = (r32 >> 1) & 7;
  auto read_op = [&](Ops& o, int i, int g) {  // g: the group modulo 4
    if (i < MTW) o.x[i] = ax[(g >> 1) & 1][(row0 + 16 * (i & ~1)) * 8 + (((g & 1) * 4 + (i & 1) * 2 + (lane >> 5)) ^ twist)];
    else o.w[i - MTW] = wx[g][wn * NTW + ((i - MTW) & ~1) + second][(i & 1) * 32 + piece];
  };
  auto read_scale = [&](Scales& s, int i) {
    if (i < MTW) s.x[i] = sc[wm * MTW + (i & ~1) + second][(i & 1) * 32 + piece];
    else s.w[i - MTW] = sc[AT + wn * NTW + ((i - MTW) & ~1) + second][(i & 1) * 32 + piece];
  };
  constexpr int kMP = MTW / 2, kNP = NTW / 2;
  static_assert(MTW % 2 == 0 && NTW % 2 == 0, "blocks go two by two");
  f32x16 acc[kMP][kNP];
  // First what needs no list of rows, behind the list itself (through LDS: the
  // wait for it then leaves the weights on their way).
  const int mine = wave * (TM / 4) + lane;
  if (a.rows)
    buffer_load_lds4(raw_rsrc(a.rows, (uint32_t)a.M * 4u), mine < b.n ? (uint32_t)(b.m0 + mine) * 4u : kOutside, 0u,
                     lds_address(&row_list[wave][0]));
#pragma unroll
  for (int i = 0; i < 2 * kW; ++i) load_weights(i % kW, i / kW);
  if (a.rows) {
    vm_wait<2 * kW>();
    asm volatile("" ::: "memory");
  }
  // lane m: the activation row of row m of this wave's quarter; -1: none, or the
  // caller's list is wrong
  int src = lane < TM / 4 && mine < b.n ? b.m0 + mine : -1;
  if (a.rows && src >= 0) {
    const uint32_t r = row_list[wave][lane];
    src = r < (uint32_t)a.M ? (int)(r / (uint32_t)a.div) : -1;
    if (src < 0) report_error(a.ws, SWIFTSPEC_DEVERR_BAD_GROUPS);
  }
  if (lane < TM / 4) live[mine] = src >= 0;
#pragma unroll
  for (int i = 0; i < kA; ++i) {
    const int from = __shfl(src, 8 * i + (lane >> 3), kWave);
    va[i] = from >= 0 ? (uint32_t)from * (uint32_t)(a.G * 64) + (uint32_t)((lane & 7) ^ (4 * (i & 1) + (lane >> 4))) * 16u : kOutside;
  }
#pragma unroll
  for (int i = 0; i < AT / 4; ++i) {
    const int from = __shfl(src, 16 * i + r16, kWave);
    vs[i] = from >= 0 ? (uint32_t)from * (uint32_t)(a.G4 * 16) + (uint32_t)kq * 4u : kOutside;
  }
#pragma unroll
  for (int i = 0; i < kS; ++i) load_scale(i, 0);
#pragma unroll
  for (int i = 0; i < 2 * kA; ++i) load_rows(i % kA, i / kA);
#pragma unroll
  for (int i = 0; i < 2 * kW; ++i) load_weights(i % kW, 2 + i / kW);
  // the sums are cleared while the loads run
#pragma unroll
  for (int i = 0; i < kMP; ++i)
#pragma unroll
    for (int j = 0; j < kNP; ++j) {
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
      asm volatile("" : "+a"(acc[i][j]));
    }
  vm_lds_barrier<kA + 2 * kW>();  // the weights of group 0, the scales, the rows of groups 0 and 1
  Ops ops[2];
  Scales s[2];
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    read_scale(s[0], i);
    read_op(ops[0], i, 0);
  }
  // Group 4 c + J.  The loads and LDS reads stand between the matrix
  // instructions, a few to each, where their issue costs nothing.
  auto step = [&](auto jc, int c, Scales& now, Scales& next) {
    constexpr int J = decltype(jc)::value;
    constexpr int kScale = J == 0 ? kS : 0, kRows = J & 1 ? kA : 0, kLoads = kScale + kRows + kW;
    constexpr int kReads = kR + (J == 3 ? kR : 0), kMfma = 2 * kMP * kNP;
    const int g = 4 * c + J;
    // what was loaded after the weights of g + 1 (J even) or the rows of g + 1 (J odd)
    vm_lds_barrier<(J & 1 ? 2 * kW : 2 * kW + kA) + (J == 1 || J == 2 ? kS : 0)>();
    const Ops& o = ops[J & 1];
    Ops& n = ops[(J & 1) ^ 1];
    auto load = [&](int q) {
      if (q < kScale) load_scale(q, c + 1);
      else if ((q -= kScale) < kRows) load_rows(q, (g + 3) / 2);
      else load_weights(q - kRows, g + 4);
    };
    auto read = [&](int q) {
      if (q < kR) read_op(n, q, (J + 1) & 3);
      else read_scale(next, q - kR);
    };
    // one LDS read to a matrix instruction, the loads spread evenly: a burst of
    // them would fill the address unit's queue and hold up the wave
#pragma unroll
    for (int k = 0; k < kMfma; ++k) {
      const int h = k / (kMP * kNP), j = k / kMP % kNP, i = k % kMP;
      acc[i][j] = mfma_mx4_32<J>(o.w[2 * j + h], now.w[2 * j + h], o.x[2 * i + h], now.x[2 * i + h], acc[i][j]);
#pragma unroll
      for (int q = k * kReads / kMfma; q < (k + 1) * kReads / kMfma; ++q) read(q);
#pragma unroll
      for (int q = k * kLoads / kMfma; q < (k + 1) * kLoads / kMfma; ++q) load(q);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int c = 0; c < G4; c += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (4 * (c + h) < G) step(std::integral_constant<int, 0>{}, c + h, s[h], s[h ^ 1]);
      if (4 * (c + h) + 1 < G) step(std::integral_constant<int, 1>{}, c + h, s[h], s[h ^ 1]);
      if (4 * (c + h) + 2 < G) step(std::integral_constant<int, 2>{}, c + h, s[h], s[h ^ 1]);
      if (4 * (c + h) + 3 < G) step(std::integral_constant<int, 3>{}, c + h, s[h], s[h ^ 1]);
    }
  }
  vm_lds_barrier<0>();  // loads past the last group still write LDS, other waves read theirs
  // Register 4 q + c of a pair of blocks holds column 8 q + 4 (lane / 32) + c of
  // row lane % 32 (SwiGLU: gate columns for q < 2, their up columns after them).
  // Through LDS the rows come out as whole 128-byte lines: 64 fp16 columns, or 32
  // fp32 ones (results that a residual or another sum awaits).
  constexpr bool wide = EPI == OUT_ROWS || EPI == OUT_RESIDUAL;
  constexpr int kPC = SW ? 16 : 32;             // columns of a pair
  constexpr int kPL = wide ? 1 : 64 / kPC;      // pairs of a line
  constexpr int kLines = (kNP + kPL - 1) / kPL;  // of 32 rows, all in LDS at one time
  constexpr int kLine = 32 * kTurnRow;
  uint8_t* my = reinterpret_cast<uint8_t*>(&room) + wave * (kLines * kLine);
  static_assert(sizeof(Operands) >= 4 * kLines * kLine, "the lines' room");
  const int tr = lane >> 3, tc = lane & 7;  // row (of 8) and 16-byte piece of a line
  // The residual is loaded at once, into the registers that the operands leave: eight
  // rows at a time cost 16 latencies (1946 rows of 2208 x 5296: 42 against 31 us,
  // 2048 of 8192 x 8192 90 against 84).
  u32x2 add[EPI == OUT_RESIDUAL ? kMP : 1][4][kLines];
  if constexpr (EPI == OUT_RESIDUAL) {
#pragma unroll
    for (int i = 0; i < kMP; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int l = 0; l < kLines; ++l) {
          const int r = 16 * (wm * MTW + 2 * i) + 8 * u + tr, col = 16 * (t0 + wn * kCW) + kPC * kPL * l + 4 * tc;
          add[i][u][l] = u32x2{0u, 0u};
          if (live[r] && col < a.N) add[i][u][l] = residual(a, b.m0 + r, col);
        }
  }
#pragma unroll
  for (int i = 0; i < kMP; ++i) {
    const int ml = 16 * (wm * MTW + 2 * i);
#pragma unroll
    for (int j = 0; j < kNP; ++j)
#pragma unroll
      for (int q = 0; q < kPC / 8; ++q) {
        f32x4 v;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          v[c] = acc[i][j][4 * q + c];
          if constexpr (SW) v[c] = silu(v[c]) * acc[i][j][4 * (q + 2) + c];
        }
        uint8_t* line = my + (j / kPL) * kLine + r32 * kTurnRow;
        const int col = kPC * (j % kPL) + 8 * q + 4 * (lane >> 5);
        if constexpr (wide) *reinterpret_cast<f32x4*>(line + 4 * col) = v;
        else *reinterpret_cast<u32x2*>(line + 2 * col) = pack4(v);
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = 8 * u + tr;
      const bool write = live[ml + r];
      const int64_t m = b.m0 + ml + r;
      u32x4 v[kLines];
#pragma unroll
      for (int l = 0; l < kLines; ++l) v[l] = *reinterpret_cast<const u32x4*>(my + l * kLine + r * kTurnRow + 16 * tc);
#pragma unroll
      for (int l = 0; l < kLines; ++l) {
        constexpr int kAll = kPC * kNP;  // columns of the wave
        const int in = kPC * kPL * l + (wide ? 4 : 8) * tc, col = 16 * (t0 + wn * kCW) + in;
        if (!write || in >= kAll || col >= a.N) continue;
        if constexpr (EPI == OUT_ROWS) {
          u32x4* p = reinterpret_cast<u32x4*>(a.part + ((int64_t)blockIdx.y * a.M + m) * a.N + col);
          if (a.past) __builtin_nontemporal_store(v[l], p);
          else *p = v[l];
        } else if constexpr (EPI == OUT_RESIDUAL) {
          f32x4 f = bitcast<f32x4>(v[l]);
          add_residual(f, add[i][u][l]);
          *reinterpret_cast<u32x2*>(a.y + m * a.ldy + col) = pack4(f);
        } else {
          store_rows16(a.y + m * a.ldy + col, v[l], SW && a.past);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int W, int MT, int NT, bool RAW, Epilogue EPI>
void launch_stream(Mx4Args a, int blocks, hipStream_t st) {
  constexpr int kC = EPI == OUT_SWIGLU ? NT / 2 : NT;
  a.col_blocks = (a.Nt + kC - 1) / kC;
  hipLaunchKernelGGL((mx4_stream_kernel<W, MT, NT, 2, RAW, EPI>), dim3((unsigned)blocks * a.col_blocks), dim3(64 * W), 0, st, a);
}

template <int WM, int WN, int MTW, int NTW, Epilogue EPI>
void launch_tile(Mx4Args a, int blocks, hipStream_t st) {
  constexpr int kC = EPI == OUT_SWIGLU ? WN * NTW / 2 : WN * NTW;
  a.col_blocks = (a.Nt + kC - 1) / kC;
  hipLaunchKernelGGL((mx4_tile_kernel<WM, WN, MTW, NTW, EPI>), dim3((unsigned)blocks * a.col_blocks, a.split), dim3(256), 0, st, a);
}

// of each Mx4Form
constexpr int kRowsOf[] = {16, 16, 32, 64, 128, 256};
constexpr int kColumnsOf[] = {32, 32, 32, 128, 128, 256};

}  // namespace

// Every line was drawn on products whose weights come from HBM (copies rotated
// through more than the Infinity Cache), preparation included; the figures are
// microseconds of the two sides.
Mx4Plan plan_mx4_gemm(int M, int E, int K, int N, bool swiglu, bool grouped, bool raw) {
  const int G4 = (mx4_groups(K) + 3) / 4;
  const int64_t weights = (int64_t)(E < M ? E : M) * K * N / 2 * (swiglu ? 2 : 1);  // bytes that are read, at most
  auto plan = [](Mx4Form f, int split = 1) { return Mx4Plan{f, kRowsOf[f], split}; };
  // shares of K that bring the tiles to one for each compute unit, each of at least
  // `least` scale words (four groups each)
  auto split_of = [&](int64_t tiles, int least) {
    const int64_t want = 256 / tiles, most = G4 / least;
    return (int)(want < 1 || most < 1 ? 1 : want < most ? want : most);
  };
  // One launch, but more registers and work in it: 8 rows of 8192 x 8192 12.4
  // against 13.1, 1 row 10.8 against 11.9; of 8192 x 28672 (112 MB) 37.0 against 26.9.
  // Up to a whole block of rows where there is little to read (16 of 4096 x 4096 8.3
  // against 9.6; 16 pairs of experts 1024 x 1024, 8 MB, with their combination 11.2
  // against 13.9; but SwiGLU of them, 16 MB, 13.2 against 10.1).
  if (raw && M <= (weights <= (12 << 20) ? 16 : 8) && weights <= (64 << 20)) return plan(STREAM_RAW);
  if (grouped) {
    const int64_t avg = M / E;
    // Rows per expert: at 2 the stream is faster (8 experts 4096 x 14336: 56.6
    // against 69.8), at 4 they meet, at 8 the tiles are (98.7 against 89.1); over a
    // short K, where its workgroups are brief, from 1 (128 experts 1024 x 512: 18.2
    // against 15.8).
    if (M < (K <= 1024 ? 1 : 4) * (int64_t)E) return plan(STREAM_1);
    // Larger tiles as long as there are enough of them for the chip (blocks of
    // rows: an expert's last is half full): down 5536 x 864, 10 experts of 899 rows,
    // 160 tiles of 256 rows 73.7 against 78.8 with 128; 8192 x 2048, 8 experts of 200
    // rows, 80 of them 63.1 against 56.1.  128 against 64 rows: 288 tiles (4096 x
    // 4096, 5 experts of 200 rows) 37.5 and 38.0; but 256 (8192 x 2048) 56.1 and 50.2,
    // 160 (8192 x 1280) 40.1 and 46.6: their number alone does not decide it.
    auto enough = [&](Mx4Form f) {
      return (M / kRowsOf[f] + (E < M ? E : M) / 2) * (int64_t)((N * (swiglu ? 2 : 1) + kColumnsOf[f] - 1) / kColumnsOf[f]) >= (f == TILE_256 ? 160 : 200);
    };
    // 64 rows: 64 against 128 rows a tile 43.9 and 47.3 (64 experts 2048 x 1024);
    // 128 rows: 60.0 and 57.5.  256 against 128 rows a tile (64 experts): SwiGLU
    // 2048 x 1024 of 384 rows 115 and 102, 768 rows 177 and 174, 1536 rows 306 and
    // 316; down 1024 x 2048 of 384 rows 132 and 128, 768 rows 234 and 241; over a
    // long K (8 experts, down 14336 x 4096) of 192 rows 111 and 133.
    if (avg >= (K >= 8192 ? 192 : 512) && enough(TILE_256)) return plan(TILE_256);
    const Mx4Form f = avg >= 96 && enough(TILE_128) ? TILE_128 : TILE_64;
    // K in shares where tiles are few, and the combination adds their sums: 28 rows
    // of 6 experts 4544 x 1120 16.6 against 14.3, 400 of 8 experts 14336 x 1024 41.8
    // against 36.0.
    return plan(f, swiglu ? 1 : split_of((int64_t)std::max(std::min(E, M), M / kRowsOf[f] + std::min(E, M) / 2) * ((N + 127) / 128), 2));
  }
  if (M <= 16) return plan(STREAM_1);
  auto tiles = [&](Mx4Form f) { return (int64_t)((M + kRowsOf[f] - 1) / kRowsOf[f]) * ((N + kColumnsOf[f] - 1) / kColumnsOf[f]); };
  // Few rows or little to read: 128 rows of 4096 x 4096 14.3 against 14.8, 32 of
  // 8192 x 8192 15.3 against 21; but 28672 x 8192 39.2 against 31.6, 8192 x 28672
  // 38.5 against 35.
  // 16 rows a workgroup, not 32, where those would leave compute units idle (32
  // rows of 11008 x 4096 13.7 against 16.9, of 4096 x 4096 10.0 against 11.8; but of
  // 8192 x 8192 16.3 against 15.1).
  if ((M <= 128 && (int64_t)K * N <= (1 << 24)) || (M <= 32 && K < 16384 && N < 24576))
    return plan(tiles(STREAM_2) < 256 ? STREAM_1 : STREAM_2);
  // 64-row tiles as long as they are at most one for each compute unit (256 rows of
  // 8192 x 8192 26.5 against 32.1; of 4096 x 4096 16.0 against 17.8), over a long K
  // only few of them (14336 x 4096: 128 rows 22.3 against 23.3, 256 rows 30.7
  // against 26.9).
  if (M <= 64 || (M <= 512 && tiles(TILE_64) <= (K <= 8192 ? 256 : 64))) return plan(TILE_64, split_of(tiles(TILE_64), 2));
  // 256-row tiles where they nearly fill the chip (384 rows of 8192 x 28672, 224
  // tiles: 66 against 75; 192 rows, 112 tiles: 55 against 51), over a long K with
  // two shares or more (28672 x 8192: 1024 rows 141 against 158).
  const int64_t big = tiles(TILE_256);
  if (M > 192 && (big >= 160 || (K >= 14336 && big >= 96) || (K >= 16384 && big >= 64)))
    return plan(TILE_256, K >= 14336 ? split_of(tiles(TILE_256), 14) : 1);
  return plan(TILE_128, split_of(tiles(TILE_128), 2));
}

namespace {

template <Epilogue EPI>
void launch_form(const Mx4Plan& p, const Mx4Args& a, int blocks, hipStream_t st) {
  switch (p.form) {
    case STREAM_RAW: return launch_stream<8, 1, 2, true, EPI>(a, blocks, st);
    case STREAM_1: return launch_stream<8, 1, 2, false, EPI>(a, blocks, st);
    case STREAM_2:
      if constexpr (EPI == OUT_PLAIN || EPI == OUT_RESIDUAL) launch_stream<8, 2, 2, false, EPI>(a, blocks, st);
      return;
    case TILE_64: return launch_tile<1, 4, 4, 2, EPI>(a, blocks, st);
    case TILE_128: return launch_tile<2, 2, 4, 4, EPI>(a, blocks, st);
    case TILE_256: return launch_tile<2, 2, 8, 8, EPI>(a, blocks, st);
  }
}

}  // namespace

int launch_mx4_gemm(const ProductLaunch& L, hipStream_t st) {
  // rows that the product may read itself: within a 2 GiB buffer, not overwritten
  const uint64_t x_bytes = ((uint64_t)(L.a_rows - 1) * L.ldx + L.K) * 2;
  const Mx4Plan p = plan_mx4_gemm(L.M, L.E, L.K, L.N, L.epi == OUT_SWIGLU, L.offsets, x_bytes < kOutside && !L.x_written);
  // 32 rows a workgroup: one matrix whose K is whole
  if (p.form == STREAM_2 && (L.offsets || p.split > 1)) return 0;
  RowMap map = {};
  map.offsets = L.offsets;
  map.E = L.E;
  map.M = L.M;
  map.tm = p.tm;
  map.blocks = L.offsets ? row_blocks(L.M, L.E, p.tm) : (L.M + p.tm - 1) / p.tm;
  map.map = L.map;
  map.ws = L.ws;
  if (p.form != STREAM_RAW) launch_mx4_prepare(L.x, L.a_rows, L.K, L.ldx, L.a, L.a_scales, L.rows ? nullptr : L.offsets, map, st);
  Mx4Args a = {};
  const size_t wq = mx4_code_bytes(L.N, L.K), wsb = mx4_scale_bytes(L.N, L.K);
  a.w0 = static_cast<const uint8_t*>(L.w0);
  a.s0 = a.w0 + L.E * wq;
  a.w1 = static_cast<const uint8_t*>(L.w1);
  a.s1 = a.w1 ? a.w1 + L.E * wq : nullptr;
  a.w_stride = (int64_t)wq;
  a.s_stride = (int64_t)wsb;
  a.G = mx4_groups(L.K);
  a.G4 = (a.G + 3) / 4;
  a.N = L.N;
  a.Nt = L.N / 16;
  a.a = L.a;
  a.as = L.a_scales;
  a.a_bytes = (uint32_t)mx4_code_bytes(L.a_rows, L.K);
  a.as_bytes = (uint32_t)mx4_scale_bytes(L.a_rows, L.K);
  a.M = L.M;
  a.map = L.offsets ? L.map : nullptr;
  a.rows = L.rows;
  a.div = L.div;
  a.y = L.y;
  a.ldy = L.ldy;
  a.res = L.res;
  a.ldr = L.ldr;
  a.part = L.part;
  a.ws = L.ws;
  a.x = L.x;
  a.x_row = (uint32_t)(L.ldx * 2);
  a.x_bytes = (uint32_t)x_bytes;
  a.split = p.split;
  // An expert product's results of more than the L2s hold go past them, so that
  // the weights stay (8191 tokens' SwiGLU 194 -> 186 us; 5000 tokens' down product
  // with its combination 203 -> 179 us); parts of a split K are read at once.
  a.past = L.offsets && (int64_t)L.M * L.N * (L.epi == OUT_ROWS ? 4 : 2) > (32 << 20);
  a.blocks = L.K / 32;
  a.offsets = L.offsets;
  a.E = L.E;
  if (L.epi == OUT_SWIGLU) {
    launch_form<OUT_SWIGLU>(p, a, map.blocks, st);
  } else if (L.epi == OUT_ROWS) {
    launch_form<OUT_ROWS>(p, a, map.blocks, st);
  } else if (p.split > 1) {
    launch_form<OUT_ROWS>(p, a, map.blocks, st);
    launch_product_sum(L.part, p.split, L.M, L.N, L.y, L.ldy, L.res, L.ldr, st);
  } else if (L.res) {
    launch_form<OUT_RESIDUAL>(p, a, map.blocks, st);
  } else {
    launch_form<OUT_PLAIN>(p, a, map.blocks, st);
  }
  return p.split;
}

bool mx4_grid_fits(int M, int E, int K, int N, bool swiglu, bool grouped) {
  if (M < 1) return true;
  for (bool raw : {false, true}) {
    const Mx4Plan p = plan_mx4_gemm(M, E, K, N, swiglu, grouped, raw);
    const int64_t blocks = grouped ? row_blocks(M, E, p.tm) : (M + p.tm - 1) / p.tm;
    const int64_t columns = ((int64_t)N * (swiglu ? 2 : 1) + kColumnsOf[p.form] - 1) / kColumnsOf[p.form];
    if (blocks * columns * (p.form <= STREAM_2 ? 512 : 256) >= 1ll << 32) return false;
  }
  return true;
}

size_t mx4_part_bytes(int M, int K, int N) {
  const Mx4Plan p = plan_mx4_gemm(M, 1, K, N, false, false, false);
  return p.split > 1 ? (size_t)p.split * M * N * sizeof(float) : 0;
}

size_t mx4_part_bytes_most(int M, int K, int N) {
  // at most 256 tiles' worth of parts, and no more shares than plan_mx4_gemm allows
  const int64_t G4 = (mx4_groups(K) + 3) / 4;
  auto most = [&](Mx4Form f, int64_t split) {
    const int64_t all = 256ll * kRowsOf[f] * kColumnsOf[f], mine = split * M * N;
    return split > 1 ? (size_t)(all < mine ? all : mine) * sizeof(float) : 0;
  };
  const size_t a = most(TILE_128, G4 / 2), b = K >= 14336 ? most(TILE_256, G4 / 14) : 0;
  return a > b ? a : b;
}

size_t mx4_rows_bytes(int M, int E, int K, int N) {
  return (size_t)plan_mx4_gemm(M, E, K, N, false, true, false).split * M * N * sizeof(float);
}

size_t mx4_rows_bytes_most(int64_t M, int K, int N) {
  // one part, or as many as plan_mx4_gemm allows of at most 256 tiles
  const size_t one = (size_t)M * N * sizeof(float), all = std::max<int64_t>((mx4_groups(K) + 3) / 4 / 2, 1) * one;
  return std::max(one, std::min(all, (size_t)256 * 128 * 128 * sizeof(float)));
}

}  // namespace ss
