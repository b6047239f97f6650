// Launches that the products with 4-bit and 8-bit matrices share.
#pragma once
#include "ss_internal.h"

namespace ss {

// The row blocks of a product, which the preparation of its activations writes
// for experts (offsets not null):  map[0] = {offsets are valid, rows of all
// experts}; map[1 + i] = {expert, first row, rows} of the i-th block of tm rows,
// experts in order; the blocks past the last have no rows.  Offsets that do not
// ascend from 0 to at most M set the error word and leave every block empty.
struct RowMap {
  const int32_t* offsets;
  int E, M, tm, blocks;
  int32_t* map;
  void* ws;
};
// the most blocks of tm rows that M rows of E experts can make
inline int row_blocks(int M, int E, int tm) { return M / tm + (E < M ? E : M); }  // M < 2^28
inline size_t row_map_bytes(int M, int E) { return ((size_t)row_blocks(M, E, 16) + 1) * 16; }

enum Epilogue { OUT_PLAIN, OUT_RESIDUAL, OUT_SWIGLU, OUT_ROWS };  // a launch asks for PLAIN, with res or without
struct ProductLaunch {
  Epilogue epi;
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
  int32_t* map;             // row_map_bytes(M, E): written and read by the launch
  uint16_t* y;              // fp16 output (PLAIN, SWIGLU)
  int64_t ldy;
  const uint16_t* res;      // residual (PLAIN)
  int64_t ldr;
  float* part;              // fp32 output [M][N] (ROWS), or room for the parts of a split K
  void* ws;                 // error word
};
// y[t] = fp16(res[t] + sum over j < k with pos[t][j] >= 0 of weights[t][j] part[pos[t][j]]),
// part the sum of `split` parts [T k][N] in order; map as the product's launch left it
void launch_moe_combine(const float* part, int split, int T, int k, int N, const int32_t* pos, const int32_t* map,
                        const float* weights, uint16_t* y, int64_t ldy, const uint16_t* res, int64_t ldr, void* ws,
                        hipStream_t st);
// y = fp16(the sum of `split` parts [M][N] in order + res)
void launch_product_sum(const float* part, int split, int M, int N, uint16_t* y, int64_t ldy, const uint16_t* res, int64_t ldr,
                        hipStream_t st);

}  // namespace ss
