// Launches of the 4-bit matrix and mixture kernels.
#pragma once
#include "ss_internal.h"

namespace ss {

// ---- microscaled 4-bit matrices (MXFP4) and the experts of a mixture ----
// Operand forms, both in groups of 128 k (the depth of one matrix
// instruction; K is padded to whole groups with codes 0 and scale byte 127):
//   weights: codes [E][N/16][G][64 lanes] x 16 bytes -- lane kq*16 + c holds
//            the 32 codes of k in [128 g + 32 kq, +32) of row 16 t + c -- then
//            scales [E][N/16][ceil(G/4)][64 lanes] u32, byte j = group 4 g4 + j;
//   activations: codes [M][G] x 64 bytes (row-major, so that an expert's rows
//            can be gathered), scales [M][ceil(G/4)][4 kq] u32, bytes as above.
inline int mx4_groups(int K) { return (int)(((int64_t)K + 127) / 128); }
inline size_t mx4_code_bytes(int64_t M, int K) { return (size_t)M * mx4_groups(K) * 64; }
inline size_t mx4_scale_bytes(int64_t M, int K) { return (size_t)M * ((mx4_groups(K) + 3) / 4) * 16; }
inline size_t mx4_packed_bytes(int K, int N, int E) {
  return (size_t)E * (mx4_code_bytes(N, K) + mx4_scale_bytes(N, K));
}

void launch_mx4_prepack(const uint8_t* codes, const uint8_t* scales, int K, int64_t rows, void* packed,
                        hipStream_t st);
// x [M][ldx] fp16 -> codes [M][K/2], scales [M][K/32]
void launch_mx4_quantize(const uint16_t* x, int64_t M, int K, int64_t ldx, uint8_t* codes, uint8_t* scales,
                         hipStream_t st);
void launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t M, int K, uint16_t* y, int64_t ldy,
                           hipStream_t st);
// The row blocks of a product, which the preparation of its activations writes
// for experts (offsets not null):  map[0] = {offsets are valid, rows of all
// experts}; map[1 + i] = {expert, first row, rows} of the i-th block of tm rows,
// experts in order; the blocks past the last have no rows.  Offsets that do not
// ascend from 0 to at most M set the error word and leave every block empty.
struct Mx4Map {
  const int32_t* offsets;
  int E, M, tm, blocks;
  int32_t* map;
  void* ws;
};
// the most blocks of tm rows that M rows of E experts can make
inline int mx4_row_blocks(int M, int E, int tm) { return M / tm + (E < M ? E : M); }  // M < 2^28
inline size_t mx4_map_bytes(int M, int E) { return ((size_t)mx4_row_blocks(M, E, 16) + 1) * 16; }
// x [M][ldx] fp16 -> the activations' operand form; with experts whose rows are
// in order (last not null) only the first last[E] rows
void launch_mx4_prepare(const uint16_t* x, int64_t M, int K, int64_t ldx, uint8_t* codes, uint8_t* scales,
                        const int32_t* last, const Mx4Map& map, hipStream_t st);

enum Mx4Epilogue { MX4_PLAIN, MX4_RESIDUAL, MX4_SWIGLU, MX4_ROWS };  // a launch asks for PLAIN, with res or without
struct Mx4Launch {
  Mx4Epilogue epi;
  const void* w0;  // packed matrices of E experts (E = 1: one matrix)
  const void* w1;  // up projections of the SwiGLU
  int K, N, E;
  const uint16_t* x;        // activations [a_rows][ldx] fp16
  int64_t ldx, a_rows;
  bool x_written;           // the output shares memory with x
  uint8_t* a;               // and room for their operand form
  uint8_t* a_scales;
  int M;                    // output rows: of the matrix, or the most that the experts share (T k)
  // experts: row i of the output belongs to the expert e with offsets[e] <= i < offsets[e + 1]
  const int32_t* offsets;   // null: one matrix, rows 0 .. M-1
  const int32_t* rows;      // row i reads activation row rows[i] / div (null: row i)
  int div;
  int32_t* map;             // mx4_map_bytes(M, E): written and read by the launch
  uint16_t* y;              // fp16 output (PLAIN, SWIGLU)
  int64_t ldy;
  const uint16_t* res;      // residual (PLAIN)
  int64_t ldr;
  float* part;              // fp32 output [M][N] (ROWS), or room for the parts of a split K
  void* ws;                 // error word
};
// bytes of the parts of one matrix's product whose K is split: of M rows, and the
// most of up to M rows
size_t mx4_part_bytes(int M, int K, int N);
size_t mx4_part_bytes_most(int M, int K, int N);
// whether a product's launch has fewer than 2^32 threads
bool mx4_grid_fits(int M, int E, int K, int N, bool swiglu, bool grouped);
// of the fp32 rows of an experts' product (ROWS), exactly, and the most of up to M rows
size_t mx4_rows_bytes(int M, int E, int K, int N);
size_t mx4_rows_bytes_most(int64_t M, int K, int N);
// The form of a product, the rows of its row blocks and the shares of K.  raw: the
// product may read the rows itself.
enum Mx4Form { STREAM_RAW, STREAM_1, STREAM_2, TILE_64, TILE_128, TILE_256 };
struct Mx4Plan {
  Mx4Form form;
  int tm, split;
};
Mx4Plan plan_mx4_gemm(int M, int E, int K, int N, bool swiglu, bool grouped, bool raw);
// quantises the activations, then multiplies; the parts [M][N] that ROWS left, or 0
// (and nothing launched) if the plan's form has no kernel for this product
int launch_mx4_gemm(const Mx4Launch& L, hipStream_t st);
// y[t] = fp16(res[t] + sum over j < k with pos[t][j] >= 0 of weights[t][j] part[pos[t][j]]),
// part the sum of `split` parts [T k][N] in order; map as the product's launch left it
void launch_moe_combine(const float* part, int split, int T, int k, int N, const int32_t* pos, const int32_t* map,
                        const float* weights, uint16_t* y, int64_t ldy, const uint16_t* res, int64_t ldr, void* ws,
                        hipStream_t st);

struct RouteLaunch {
  const uint16_t* logits;  // null: the experts are given
  int ldl, T, E, k, renormalize;
  int32_t* experts;
  float* weights;
  int32_t *offsets, *rows, *pos;
  uint16_t* hist;  // route_hist_bytes
};
size_t route_hist_bytes(int T, int E, int k);  // T k < 2^28
void launch_moe_route(const RouteLaunch& L, hipStream_t st);

}  // namespace ss
