// mx4.hip -- matrices to and from microscaled 4-bit floating point (the
// format and its layout: mx4.hpp).
#include <hip/hip_runtime.h>

#include "mx4.hpp"
#include "mx4_block.hpp"

namespace fgd {
namespace {

template <typename T>
__device__ inline T narrow(float v);
template <>
__device__ inline float narrow<float>(float v) { return v; }
template <>
__device__ inline uint16_t narrow<uint16_t>(float v) {  // nearest, ties to even; NaN stays NaN
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return static_cast<uint16_t>((u >> 16) | 0x40u);
    return static_cast<uint16_t>((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// Rows contiguous: a 64 x 128 tile per block of 256 threads, a thread per
// block of 32.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *__restrict__ x, int64_t tiles, int64_t rows,
                                                            int64_t cols, int64_t row_tiles, int64_t col_tiles,
                                                            int64_t batch_stride, int64_t row_stride, bool vectors,
                                                            uint8_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales) {
    const int lane = threadIdx.x & 63, frag = threadIdx.x >> 6;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t kt = tile % col_tiles, rt = tile / col_tiles % row_tiles, b = tile / col_tiles / row_tiles;
        const int64_t r = rt * kMx4TileRows + (frag >> 1) * 32 + (lane & 31),
                      k0 = kt * kMx4TileCols + (frag & 1) * 64 + (lane >> 5) * 32;
        float v[32];
        load_block(x + b * batch_stride + r * row_stride + k0, r < rows ? cols - k0 : 0, vectors, v);
        uint4 c;
        const uint32_t byte = encode_block(v, c);
        *reinterpret_cast<uint4 *>(codes + tile * kMx4CodeBytes + frag * 1024 + lane * 16) = c;
        scales[tile * kMx4ScaleBytes + lane * 4 + frag] = static_cast<uint8_t>(byte);
    }
}

// Columns contiguous (blocks along the columns of the stored matrix).
template <typename T>
__global__ __launch_bounds__(256) void quantize_columns_kernel(const T *__restrict__ x, int64_t tiles, int64_t rows,
                                                               int64_t cols, int64_t row_tiles, int64_t col_tiles,
                                                               int64_t batch_stride, int64_t col_stride,
                                                               uint8_t *__restrict__ codes,
                                                               uint8_t *__restrict__ scales) {
    const int lane = threadIdx.x & 63, frag = threadIdx.x >> 6;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t kt = tile % col_tiles, rt = tile / col_tiles % row_tiles, b = tile / col_tiles / row_tiles;
        const int64_t r = rt * kMx4TileRows + (frag >> 1) * 32 + (lane & 31),
                      k0 = kt * kMx4TileCols + (frag & 1) * 64 + (lane >> 5) * 32;
        const T *src = x + b * batch_stride + r + k0 * col_stride;
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = r < rows && k0 + i < cols ? widen(src[i * col_stride]) : 0.0f;
        uint4 c;
        const uint32_t byte = encode_block(v, c);
        *reinterpret_cast<uint4 *>(codes + tile * kMx4CodeBytes + frag * 1024 + lane * 16) = c;
        scales[tile * kMx4ScaleBytes + lane * 4 + frag] = static_cast<uint8_t>(byte);
    }
}

template <typename T>
void quantize(const T *x, int64_t tiles, int64_t rows, int64_t cols, int64_t rt, int64_t kt, int64_t batch_stride,
              int64_t row_stride, int64_t col_stride, uint8_t *codes, uint8_t *scales, int grid, hipStream_t stream) {
    if (col_stride == 1 || cols == 1)
        quantize_rows_kernel<<<grid, 256, 0, stream>>>(x, tiles, rows, cols, rt, kt, batch_stride, row_stride,
                                                       mx4_rows_aligned(x, sizeof(T) == 2, batch_stride, row_stride),
                                                       codes, scales);
    else
        quantize_columns_kernel<<<grid, 256, 0, stream>>>(x, tiles, rows, cols, rt, kt, batch_stride, col_stride,
                                                          codes, scales);
}

template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t *__restrict__ codes,
                                                         const uint8_t *__restrict__ scales, int64_t tiles,
                                                         int64_t rows, int64_t cols, int64_t row_tiles,
                                                         int64_t col_tiles, T *__restrict__ out, int64_t batch_stride,
                                                         int64_t row_stride) {
    const int lane = threadIdx.x & 63, frag = threadIdx.x >> 6;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t kt = tile % col_tiles, rt = tile / col_tiles % row_tiles, b = tile / col_tiles / row_tiles;
        const int64_t r = rt * kMx4TileRows + (frag >> 1) * 32 + (lane & 31),
                      k0 = kt * kMx4TileCols + (frag & 1) * 64 + (lane >> 5) * 32;
        const uint4 c = *reinterpret_cast<const uint4 *>(codes + tile * kMx4CodeBytes + frag * 1024 + lane * 16);
        const uint32_t byte = scales[tile * kMx4ScaleBytes + lane * 4 + frag];
        const float scale = byte == 255 ? __uint_as_float(0x7fc00000u)
                                        : __uint_as_float(byte == 0 ? 1u << 22 : byte << 23);
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
        T *dst = out + b * batch_stride + r * row_stride + k0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const uint32_t code = w[i >> 3] >> (4 * (i & 7));
            const uint32_t e = (code >> 1) & 3, m = code & 1;
            const float a = e == 0 ? 0.5f * m : __uint_as_float((126 + e) << 23) * (1.0f + 0.5f * m);
            if (r < rows && k0 + i < cols) dst[i] = narrow<T>((code & 8 ? -a : a) * scale);
        }
    }
}

int grid_for(int64_t tiles) { return static_cast<int>(tiles < 1 << 20 ? tiles : 1 << 20); }

}  // namespace

bool mx4_quantize_launch(const void *x, bool bf16, int64_t batch, int64_t rows, int64_t cols, int64_t batch_stride,
                         int64_t row_stride, int64_t col_stride, void *codes, void *scales, hipStream_t stream) {
    const int64_t rt = mx4_row_tiles(rows), kt = mx4_col_tiles(cols), tiles = batch * rt * kt;
    if (tiles == 0) return true;
    auto *c = static_cast<uint8_t *>(codes), *s = static_cast<uint8_t *>(scales);
    if (bf16)
        quantize(static_cast<const uint16_t *>(x), tiles, rows, cols, rt, kt, batch_stride, row_stride, col_stride, c, s,
                 grid_for(tiles), stream);
    else
        quantize(static_cast<const float *>(x), tiles, rows, cols, rt, kt, batch_stride, row_stride, col_stride, c, s,
                 grid_for(tiles), stream);
    return hipGetLastError() == hipSuccess;
}

bool mx4_dequantize_launch(const void *codes, const void *scales, int64_t batch, int64_t rows, int64_t cols,
                           void *out, bool bf16, int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    const int64_t rt = mx4_row_tiles(rows), kt = mx4_col_tiles(cols), tiles = batch * rt * kt;
    if (tiles == 0) return true;
    auto *c = static_cast<const uint8_t *>(codes), *s = static_cast<const uint8_t *>(scales);
    if (bf16)
        dequantize_kernel<<<grid_for(tiles), 256, 0, stream>>>(c, s, tiles, rows, cols, rt, kt,
                                                              static_cast<uint16_t *>(out), batch_stride, row_stride);
    else
        dequantize_kernel<<<grid_for(tiles), 256, 0, stream>>>(c, s, tiles, rows, cols, rt, kt,
                                                              static_cast<float *>(out), batch_stride, row_stride);
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
