// Launches of the 8-bit matrix kernels.
#pragma once
#include "product_internal.h"

namespace ss {

// ---- block-scaled 8-bit matrices (e4m3 codes) ----
// Operand forms, both in groups of 128 k (the depth of one matrix instruction and of
// a block; K is padded to whole groups with codes 0):
//   weights: codes [E][N/16][G][8 pieces][16 rows] x 16 bytes -- a piece is 16
//            consecutive k of row 16 t + r -- then scales [E][ceil(N/128)][G] float;
//   activations: codes [M][G] x 128 bytes (row-major, so that an expert's rows can be
//            gathered), scales [M][ceil(G/4)] u32, byte j = that of group 4 g4 + j:
//            s stands for 2^(s - 127), 255 for NaN.
inline int fp8_blocks(int n) { return (int)(((int64_t)n + 127) / 128); }
inline size_t fp8_code_bytes(int64_t M, int K) { return (size_t)M * fp8_blocks(K) * 128; }
inline size_t fp8_scale_bytes(int64_t M, int K) { return (size_t)M * ((fp8_blocks(K) + 3) / 4) * 4; }
inline size_t fp8_matrix_scale_bytes(int K, int N) { return (size_t)fp8_blocks(N) * fp8_blocks(K) * 4; }
inline size_t fp8_packed_bytes(int K, int N, int E) {
  return (size_t)E * (fp8_code_bytes(N, K) + fp8_matrix_scale_bytes(K, N));
}

void launch_fp8_prepack(const uint8_t* codes, const float* scales, int K, int N, int E, void* packed, hipStream_t st);
// x [M][ldx] fp16 -> codes [M][K], scales [M][G], or [ceil(M/128)][G] of blocks of 128 rows
void launch_fp8_quantize(const uint16_t* x, int64_t M, int K, int64_t ldx, int rows, uint8_t* codes, float* scales, hipStream_t st);
void launch_fp8_dequantize(const uint8_t* codes, const float* scales, int64_t M, int K, int rows, uint16_t* y, int64_t ldy,
                           hipStream_t st);
// x [M][ldx] fp16 -> the activations' operand form; with experts whose rows are in
// order (last not null) only the first last[E] rows
void launch_fp8_prepare(const uint16_t* x, int64_t M, int K, int64_t ldx, uint8_t* codes, uint8_t* scales, const int32_t* last,
                        const RowMap& map, hipStream_t st);

// bytes of the parts of one matrix's product whose K is split: of M rows, and the
// most of up to M rows
size_t fp8_part_bytes(int M, int K, int N);
size_t fp8_part_bytes_most(int M, int K, int N);
// whether a product's launch has fewer than 2^32 threads
bool fp8_grid_fits(int M, int E, int K, int N, bool swiglu, bool grouped);
// of the fp32 rows of an experts' product (ROWS), exactly, and the most of up to M rows
size_t fp8_rows_bytes(int M, int E, int K, int N);
size_t fp8_rows_bytes_most(int64_t M, int K, int N);
// The form of a product, the rows of its row blocks and the shares of K.  raw: the
// product may read the rows itself.
enum class Fp8Form { STREAM_RAW, STREAM_1, STREAM_2, TILE_64, TILE_128_DEEP, TILE_128, TILE_256 };
struct Fp8Plan {
  Fp8Form form;
  int tm, split;
};
Fp8Plan plan_fp8_gemm(int M, int E, int K, int N, bool swiglu, bool grouped, bool raw);
// quantises the activations, then multiplies; the parts [M][N] that ROWS left, or 0
// (and nothing launched) if the plan's form has no kernel for this product
int launch_fp8_gemm(const ProductLaunch& L, hipStream_t st);

}  // namespace ss
