// mx4.hpp -- layout of matrices in microscaled 4-bit floating point and the
// launchers of their kernels (quantisation, reading back, product).
//
// The format.  Blocks of 32 consecutive elements of a row share a scale
// 2^(byte - 127), byte = max(e - 2, 0) with e the float32 exponent field of
// the block's largest magnitude (floor(log2) + 127); an element is its value
// over the scale, rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties
// to the even code, saturating at 6), with a sign bit.  A block that holds an
// infinity or a NaN has byte 255 and reads back as NaN.
//
// The layout is that of the matrix instruction's operands, so that every
// kernel moves whole fragments and none rearranges one: a matrix of R rows
// and K columns lies in tiles of 64 rows x 128 columns, tile (r, k) at index
// r * ceil(K / 128) + k, batch after batch.  A tile's codes are four
// fragments of 32 rows x 64 columns, 1 KB each, fragment 2 p + h holding row
// half p and column half h: lane l = (row % 32) + 32 * (block % 2) holds the
// 16 bytes of one block of its row, low nibble first.  A tile's scales are
// 64 dwords, one per lane, whose byte f belongs to fragment f.  Rows and
// columns past the matrix are zero.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fgd {

constexpr int kMx4TileRows = 64, kMx4TileCols = 128;
constexpr int kMx4CodeBytes = 4096, kMx4ScaleBytes = 256;  // of one tile

inline int64_t mx4_row_tiles(int64_t rows) { return (rows + kMx4TileRows - 1) / kMx4TileRows; }
inline int64_t mx4_col_tiles(int64_t cols) { return (cols + kMx4TileCols - 1) / kMx4TileCols; }
inline int64_t mx4_tiles(int64_t batch, int64_t rows, int64_t cols) {
    return batch * mx4_row_tiles(rows) * mx4_col_tiles(cols);
}

// x[b][r][k] at b * batch_stride + r * row_stride + k * col_stride, one of
// the last two strides 1.  False if a launch failed.
bool mx4_quantize_launch(const void *x, bool bf16, int64_t batch, int64_t rows, int64_t cols, int64_t batch_stride,
                         int64_t row_stride, int64_t col_stride, void *codes, void *scales, hipStream_t stream);

// The same of x[b][r][k] at b * batch_stride + r * row_stride + k and of its
// transpose.
bool mx4_quantize_both_launch(const void *x, bool bf16, int64_t batch, int64_t rows, int64_t cols,
                              int64_t batch_stride, int64_t row_stride, void *codes, void *scales, void *t_codes,
                              void *t_scales, hipStream_t stream);

bool mx4_dequantize_launch(const void *codes, const void *scales, int64_t batch, int64_t rows, int64_t cols,
                           void *out, bool bf16, int64_t batch_stride, int64_t row_stride, hipStream_t stream);

// out[b][i][j] = sum_k a[b][i][k] w[b][j][k]: i < m, j < n.
bool mx4_matmul_launch(const void *a_codes, const void *a_scales, const void *w_codes, const void *w_scales,
                       int64_t batch, int64_t m, int64_t n, int64_t k, void *out, bool bf16, int64_t batch_stride,
                       int64_t row_stride, hipStream_t stream);

// The same product of x[b][i][k] at b * x_batch_stride + i * x_row_stride + k,
// quantised on the way: for the few rows for which mx4_linear_fuses.
bool mx4_linear_fuses(int64_t batch, int64_t m, int64_t n, int64_t k);
bool mx4_linear_launch(const void *x, bool x_bf16, int64_t x_batch_stride, int64_t x_row_stride, const void *w_codes,
                       const void *w_scales, int64_t batch, int64_t m, int64_t n, int64_t k, void *out, bool bf16,
                       int64_t batch_stride, int64_t row_stride, hipStream_t stream);

}  // namespace fgd
