// Launches of the 4-bit matrix kernels.
#pragma once
#include "product_internal.h"

namespace ss {

// ---- microscaled 4-bit matrices (MXFP4) ----
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
// x [M][ldx] fp16 -> the activations' operand form; with experts whose rows are
// in order (last not null) only the first last[E] rows
void launch_mx4_prepare(const uint16_t* x, int64_t M, int K, int64_t ldx, uint8_t* codes, uint8_t* scales,
                        const int32_t* last, const RowMap& map, hipStream_t st);

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
int launch_mx4_gemm(const ProductLaunch& L, hipStream_t st);

}  // namespace ss
