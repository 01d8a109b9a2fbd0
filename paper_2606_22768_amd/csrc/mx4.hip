// mx4.hip -- matrices to and from microscaled 4-bit floating point (the
// format and its layout: mx4.hpp).
#include <hip/hip_runtime.h>

#include "mx4.hpp"

namespace fgd {
namespace {

template <typename T>
__device__ inline float widen(T v);
template <>
__device__ inline float widen<float>(float v) { return v; }
template <>
__device__ inline float widen<uint16_t>(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }

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

// One block of 32 values to its 16 code bytes; returns the scale byte.
__device__ inline uint32_t encode_block(const float (&v)[32], uint4 &codes) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    const uint32_t field = top >> 23;
    if (field == 255) {
        codes = make_uint4(0, 0, 0, 0);
        return 255;
    }
    const uint32_t byte = field > 2 ? field - 2 : 0;
    // The conversion divides by its scale operand, a normal number: blocks
    // of byte 0 (scale 2^-127, a denormal) are raised by 2^64 first, exactly.
    const float lift = byte == 0 ? 0x1p64f : 1.0f;
    const float scale = __uint_as_float((byte == 0 ? 64u : byte) << 23);
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t r = 0;
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * q + 0] * lift, v[8 * q + 1] * lift, scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * q + 2] * lift, v[8 * q + 3] * lift, scale, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * q + 4] * lift, v[8 * q + 5] * lift, scale, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * q + 6] * lift, v[8 * q + 7] * lift, scale, 3);
        w[q] = r;
    }
    codes = make_uint4(w[0], w[1], w[2], w[3]);
    return byte;
}

// One 64 x 128 tile per block of 256 threads, a thread per block of 32.
template <typename T>
__global__ __launch_bounds__(256) void quantize_kernel(const T *__restrict__ x, int64_t tiles, int64_t rows,
                                                       int64_t cols, int64_t row_tiles, int64_t col_tiles,
                                                       int64_t batch_stride, int64_t row_stride, int64_t col_stride,
                                                       uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    const int lane = threadIdx.x & 63, frag = threadIdx.x >> 6;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t kt = tile % col_tiles, rt = tile / col_tiles % row_tiles, b = tile / col_tiles / row_tiles;
        const int64_t r = rt * kMx4TileRows + frag * 16 + (lane & 15), k0 = kt * kMx4TileCols + (lane >> 4) * 32;
        const T *src = x + b * batch_stride + r * row_stride + k0 * col_stride;
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
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t *__restrict__ codes,
                                                         const uint8_t *__restrict__ scales, int64_t tiles,
                                                         int64_t rows, int64_t cols, int64_t row_tiles,
                                                         int64_t col_tiles, T *__restrict__ out, int64_t batch_stride,
                                                         int64_t row_stride) {
    const int lane = threadIdx.x & 63, frag = threadIdx.x >> 6;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t kt = tile % col_tiles, rt = tile / col_tiles % row_tiles, b = tile / col_tiles / row_tiles;
        const int64_t r = rt * kMx4TileRows + frag * 16 + (lane & 15), k0 = kt * kMx4TileCols + (lane >> 4) * 32;
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
        quantize_kernel<<<grid_for(tiles), 256, 0, stream>>>(static_cast<const uint16_t *>(x), tiles, rows, cols, rt, kt,
                                                            batch_stride, row_stride, col_stride, c, s);
    else
        quantize_kernel<<<grid_for(tiles), 256, 0, stream>>>(static_cast<const float *>(x), tiles, rows, cols, rt, kt,
                                                            batch_stride, row_stride, col_stride, c, s);
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
