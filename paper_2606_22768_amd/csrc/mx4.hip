// mx4.hip -- matrices to and from microscaled 4-bit floating point (the
// format and its layout: mx4.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx4.hpp"
#include "mx4_block.hpp"

namespace fgd {
namespace {

// f(tile, batch entry, row tile, column tile) for a block's tiles: blocks of
// one row of tiles are neighbours (those of one column: 143 us for 127 at
// 128256 x 2048 bf16), and no index is divided.  (A loop over the columns as
// well takes reading back from 119 to 177 us right after the quantisation.)
template <typename F>
__device__ inline void for_tiles(int64_t row_tiles, int64_t col_tiles, int64_t batch, int64_t first_col, F f) {
    const int64_t k = first_col + blockIdx.x;
    for (int64_t b = blockIdx.z; b < batch; b += gridDim.z)
        for (int64_t r = blockIdx.y; r < row_tiles; r += gridDim.y)
            f((b * row_tiles + r) * col_tiles + k, b, r, k);
}

// Rows contiguous: a 64 x 128 tile per block of 256 threads, a thread per
// block of 32: no sum or maximum crosses lanes, and a wave stores a whole
// fragment.  Bound by memory: 128256 x 2048 bf16 in 128 us, 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *__restrict__ x, int64_t batch, int64_t rows,
                                                            int64_t cols, int64_t row_tiles, int64_t col_tiles,
                                                            int64_t first_col,
                                                            int64_t batch_stride, int64_t row_stride,
                                                            uint8_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales) {
    const int lane = threadIdx.x & 63, frag = threadIdx.x >> 6;
    for_tiles(row_tiles, col_tiles, batch, first_col, [&](int64_t tile, int64_t b, int64_t rt, int64_t kt) {
        const int64_t r = rt * kMx4TileRows + (frag >> 1) * 32 + (lane & 31),
                      k0 = kt * kMx4TileCols + (frag & 1) * 64 + (lane >> 5) * 32;
        float v[32];
        load_block(x + b * batch_stride + r * row_stride + k0, r < rows ? cols - k0 : 0, v);
        uint4 c;
        const uint32_t byte = encode_block(v, c);
        *reinterpret_cast<uint4 *>(codes + tile * kMx4CodeBytes + frag * 1024 + lane * 16) = c;
        scales[tile * kMx4ScaleBytes + lane * 4 + frag] = static_cast<uint8_t>(byte);
    });
}

// Columns contiguous: blocks along the columns of the stored matrix.  A
// thread takes two neighbouring rows' blocks, so that a wave reads 128 (bf16)
// or 256 bytes of each stored row: one row each read 2-byte elements, at 1.7
// TB/s.  128256 x 2048 bf16 along the columns: 153 us, 4.3 TB/s.
template <typename T>
__global__ __launch_bounds__(128) void quantize_columns_kernel(const T *__restrict__ x, int64_t batch, int64_t rows,
                                                               int64_t cols, int64_t row_tiles, int64_t col_tiles,
                                                            int64_t first_col,
                                                               int64_t batch_stride, int64_t col_stride,
                                                               uint8_t *__restrict__ codes,
                                                               uint8_t *__restrict__ scales) {
    struct __attribute__((packed, aligned(sizeof(T)))) Pair {
        T v[2];
    };
    const int pair = threadIdx.x & 31, block = threadIdx.x >> 5;
    const int row = 2 * pair, lane = (row & 31) + 32 * (block & 1), frag = 2 * (row >> 5) + (block >> 1);
    for_tiles(row_tiles, col_tiles, batch, first_col, [&](int64_t tile, int64_t b, int64_t rt, int64_t kt) {
        const int64_t r = rt * kMx4TileRows + row, k0 = kt * kMx4TileCols + block * 32;
        const T *src = x + b * batch_stride + r + k0 * col_stride;
        float v[2][32];
        if (r + 1 < rows && k0 + 32 <= cols) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const Pair p = *reinterpret_cast<const Pair *>(src + i * col_stride);
                v[0][i] = widen(p.v[0]);
                v[1][i] = widen(p.v[1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                v[0][i] = r < rows && k0 + i < cols ? widen(src[i * col_stride]) : 0.0f;
                v[1][i] = r + 1 < rows && k0 + i < cols ? widen(src[i * col_stride + 1]) : 0.0f;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint4 c;
            const uint32_t byte = encode_block(v[h], c);
            *reinterpret_cast<uint4 *>(codes + tile * kMx4CodeBytes + frag * 1024 + (lane + h) * 16) = c;
            scales[tile * kMx4ScaleBytes + (lane + h) * 4 + frag] = static_cast<uint8_t>(byte);
        }
    });
}

// Rows contiguous, along both axes in one reading: 128 x 128 elements per
// block of 256 threads, quantised along the rows on their way to LDS and along
// the columns from there.  An LDS row's odd stride in dwords keeps the lanes of
// both passes, rows of one column and columns of one row, on banks of their own.
// Bound by memory: 4096 x 8192 bf16 in 27 us, 3.8 TB/s (20.7 with x in the
// last-level cache, for 14.6 and 16.3 one by one).
template <typename T>
__global__ __launch_bounds__(256) void quantize_both_kernel(const T *__restrict__ x, int64_t batch, int64_t rows,
                                                            int64_t cols, int64_t row_tiles, int64_t col_tiles,
                                                            int64_t first_col, int64_t t_row_tiles,
                                                            int64_t t_col_tiles,
                                                            int64_t batch_stride, int64_t row_stride,
                                                            uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                            uint8_t *__restrict__ t_codes,
                                                            uint8_t *__restrict__ t_scales) {
    __shared__ T s[128][128 + (sizeof(T) == 4 ? 1 : 2)];
    const int lane = threadIdx.x & 63, frag = threadIdx.x >> 6;
    const int i = (frag >> 1) * 32 + (lane & 31), j = (frag & 1) * 64 + (lane >> 5) * 32;
    for_tiles(t_col_tiles, col_tiles, batch, first_col, [&](int64_t, int64_t b, int64_t rb, int64_t kb) {
        auto put = [&](const float (&v)[32], uint8_t *c, uint8_t *sc, int64_t tile) {
            uint4 q;
            const uint32_t byte = encode_block(v, q);
            *reinterpret_cast<uint4 *>(c + tile * kMx4CodeBytes + frag * 1024 + lane * 16) = q;
            sc[tile * kMx4ScaleBytes + lane * 4 + frag] = static_cast<uint8_t>(byte);
        };
        const int64_t k0 = kb * 128 + j;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t rt = 2 * rb + h, r = rt * kMx4TileRows + i;
            float v[32];
            load_block(x + b * batch_stride + r * row_stride + k0, r < rows ? cols - k0 : 0, v);
#pragma unroll
            for (int e = 0; e < 32; ++e) s[h * 64 + i][j + e] = narrow<T>(v[e]);
            if (rt < row_tiles) put(v, codes, scales, (b * row_tiles + rt) * col_tiles + kb);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t rt = 2 * kb + h;
            if (rt >= t_row_tiles) continue;
            float v[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = widen(s[j + e][h * 64 + i]);
            put(v, t_codes, t_scales, (b * t_row_tiles + rt) * t_col_tiles + rb);
        }
        __syncthreads();
    });
}

// A tile per block of 256 threads, 16 bytes of output a thread and step, a
// tile row's by neighbouring lanes: stores of whole lines (a block of 32 per
// thread: 16-byte pieces of 64 rows at once, 2.5 TB/s).  Bound by the stores:
// 128256 x 2048 to bf16 in 95 us, 7.0 TB/s; in 121 right after the
// quantisation, whose codes have yet to leave the caches.
template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t *__restrict__ codes,
                                                         const uint8_t *__restrict__ scales, int64_t batch,
                                                         int64_t rows, int64_t cols, int64_t row_tiles,
                                                         int64_t col_tiles, int64_t first_col, T *__restrict__ out,
                                                         int64_t batch_stride, int64_t row_stride) {
    typedef float float2v __attribute__((ext_vector_type(2)));
    constexpr int kPer = 16 / sizeof(T), kLanes = kMx4TileCols / kPer, kRows = 256 / kLanes;
    const int col = static_cast<int>(threadIdx.x) % kLanes * kPer, block = col >> 5;
    for_tiles(row_tiles, col_tiles, batch, first_col, [&](int64_t tile, int64_t b, int64_t rt, int64_t kt) {
        const int64_t k = kt * kMx4TileCols + col;
#pragma unroll
        for (int i = 0; i < kMx4TileRows; i += kRows) {
            const int row = i + static_cast<int>(threadIdx.x) / kLanes, lane = (row & 31) + 32 * (block & 1),
                      frag = 2 * (row >> 5) + (block >> 1);
            const int64_t r = rt * kMx4TileRows + row;
            if (r >= rows || k >= cols) continue;
            const uint8_t *src = codes + tile * kMx4CodeBytes + frag * 1024 + lane * 16 + (col & 31) / 2;
            const uint32_t byte = scales[tile * kMx4ScaleBytes + lane * 4 + frag];
            const float scale = byte == 255 ? __uint_as_float(0x7fc00000u)
                                            : __uint_as_float(byte == 0 ? 1u << 22 : byte << 23);
            T v[kPer];
            T *dst = out + b * batch_stride + r * row_stride + k;
            if constexpr (sizeof(T) == 4) {
                const uint32_t w = *reinterpret_cast<const uint16_t *>(src);
                const float2v lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0),
                              hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
                v[0] = lo[0] * scale, v[1] = lo[1] * scale, v[2] = hi[0] * scale, v[3] = hi[1] * scale;
            } else {
                const uint32_t w = *reinterpret_cast<const uint32_t *>(src);
                const float2v p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0),
                                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2),
                                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
                // Two significant bits, multiples of 2^-128: bf16 holds them
                // as they are, its denormals included.
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = static_cast<T>(__float_as_uint(p[e >> 1][e & 1] * scale) >> 16);
            }
            if (k + kPer <= cols) {
                // Past the caches: 108 us for 242 at 128256 x 2048 to bf16.
                typedef uint32_t Out __attribute__((ext_vector_type(4), aligned(2)));
                Out q;
                __builtin_memcpy(&q, v, 16);
                __builtin_nontemporal_store(q, reinterpret_cast<Out *>(dst));
            } else {
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (k + e < cols) dst[e] = v[e];
            }
        }
    });
}

// Launches over all tiles: launch(grid, first column tile).
template <typename F>
bool for_grids(int64_t batch, int64_t row_tiles, int64_t col_tiles, F launch) {
    constexpr int64_t kMost = 1 << 22;  // a grid's threads in one direction are below 2^32
    for (int64_t k = 0; k < col_tiles; k += kMost)
        launch(dim3(static_cast<unsigned>(std::min(col_tiles - k, kMost)),
                    static_cast<unsigned>(std::min<int64_t>(row_tiles, 65535)),
                    static_cast<unsigned>(std::min<int64_t>(batch, 65535))),
               k);
    return hipGetLastError() == hipSuccess;
}

}  // namespace

bool mx4_quantize_launch(const void *x, bool bf16, int64_t batch, int64_t rows, int64_t cols, int64_t batch_stride,
                         int64_t row_stride, int64_t col_stride, void *codes, void *scales, hipStream_t stream) {
    const int64_t rt = mx4_row_tiles(rows), kt = mx4_col_tiles(cols);
    if (batch == 0 || rt == 0 || kt == 0) return true;
    auto *c = static_cast<uint8_t *>(codes), *s = static_cast<uint8_t *>(scales);
    auto go = [&](auto *p) {
        return for_grids(batch, rt, kt, [&](dim3 grid, int64_t first) {
            if (col_stride == 1 || cols == 1)
                quantize_rows_kernel<<<grid, 256, 0, stream>>>(p, batch, rows, cols, rt, kt, first, batch_stride,
                                                               row_stride, c, s);
            else
                quantize_columns_kernel<<<grid, 128, 0, stream>>>(p, batch, rows, cols, rt, kt, first, batch_stride,
                                                                  col_stride, c, s);
        });
    };
    return bf16 ? go(static_cast<const uint16_t *>(x)) : go(static_cast<const float *>(x));
}

bool mx4_quantize_both_launch(const void *x, bool bf16, int64_t batch, int64_t rows, int64_t cols,
                              int64_t batch_stride, int64_t row_stride, void *codes, void *scales, void *t_codes,
                              void *t_scales, hipStream_t stream) {
    if (batch == 0 || rows == 0 || cols == 0) return true;
    const int64_t rt = mx4_row_tiles(rows), kt = mx4_col_tiles(cols), t_rt = mx4_row_tiles(cols),
                  t_kt = mx4_col_tiles(rows);
    auto go = [&](auto *p) {
        return for_grids(batch, t_kt, kt, [&](dim3 grid, int64_t first) {
            quantize_both_kernel<<<grid, 256, 0, stream>>>(
                p, batch, rows, cols, rt, kt, first, t_rt, t_kt, batch_stride, row_stride,
                static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales), static_cast<uint8_t *>(t_codes),
                static_cast<uint8_t *>(t_scales));
        });
    };
    return bf16 ? go(static_cast<const uint16_t *>(x)) : go(static_cast<const float *>(x));
}

bool mx4_dequantize_launch(const void *codes, const void *scales, int64_t batch, int64_t rows, int64_t cols,
                           void *out, bool bf16, int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    const int64_t rt = mx4_row_tiles(rows), kt = mx4_col_tiles(cols);
    if (batch == 0 || rt == 0 || kt == 0) return true;
    auto *c = static_cast<const uint8_t *>(codes), *s = static_cast<const uint8_t *>(scales);
    auto go = [&](auto *to) {
        return for_grids(batch, rt, kt, [&](dim3 grid, int64_t first) {
            dequantize_kernel<<<grid, 256, 0, stream>>>(c, s, batch, rows, cols, rt, kt, first, to, batch_stride,
                                                        row_stride);
        });
    };
    return bf16 ? go(static_cast<uint16_t *>(out)) : go(static_cast<float *>(out));
}

}  // namespace fgd
