// mx4_gemm.hip -- products of matrices in microscaled 4-bit floating point
// (the format and its layout: mx4.hpp).
#include <hip/hip_runtime.h>

#include "mx4.hpp"

namespace fgd {
namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

// The operands' 4-bit format code, and which byte of the scale dwords.
template <int SA, int SB>
__device__ inline float4v mfma(int4v a, int4v b, float4v c, int sa, int sb) {
    const int8v x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, SA, sa, SB, sb);
}

__device__ inline uint16_t round_bf16(float v) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return static_cast<uint16_t>((u >> 16) | 0x40u);
    return static_cast<uint16_t>((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

__device__ inline void store(float *p, float v) { *p = v; }
__device__ inline void store(uint16_t *p, float v) { *p = round_bf16(v); }

// Four waves, each 64 rows of w by 16 rows of a; fragments straight from
// memory.
template <typename T>
__global__ __launch_bounds__(256) void product_kernel(const uint8_t *__restrict__ a_codes,
                                                      const uint8_t *__restrict__ a_scales,
                                                      const uint8_t *__restrict__ w_codes,
                                                      const uint8_t *__restrict__ w_scales, int64_t m, int64_t n,
                                                      int64_t kt, int64_t n_blocks, int64_t m_blocks,
                                                      T *__restrict__ out, int64_t batch_stride, int64_t row_stride) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t nb = blockIdx.x % n_blocks, mb = blockIdx.x / n_blocks % m_blocks,
                  b = blockIdx.x / n_blocks / m_blocks;
    const int64_t a_tiles = (m + 63) / 64, w_tiles = (n + 63) / 64;
    const int64_t wt = min(nb * 4 + wave, w_tiles - 1);  // a wave past the end repeats the last tile, unstored
    const int sub = mb & 3;
    const uint8_t *wc = w_codes + (b * w_tiles + wt) * kt * kMx4CodeBytes + lane * 16;
    const uint8_t *ws = w_scales + (b * w_tiles + wt) * kt * kMx4ScaleBytes + lane * 4;
    const uint8_t *ac = a_codes + (b * a_tiles + (mb >> 2)) * kt * kMx4CodeBytes + sub * 1024 + lane * 16;
    const uint8_t *as = a_scales + (b * a_tiles + (mb >> 2)) * kt * kMx4ScaleBytes + lane * 4;
    float4v acc[4] = {};
    for (int64_t k = 0; k < kt; ++k) {
        const int4v x = *reinterpret_cast<const int4v *>(ac + k * kMx4CodeBytes);
        const int sx = *reinterpret_cast<const int *>(as + k * kMx4ScaleBytes) >> (8 * sub);
        const int sw = *reinterpret_cast<const int *>(ws + k * kMx4ScaleBytes);
        const uint8_t *p = wc + k * kMx4CodeBytes;
        acc[0] = mfma<0, 0>(*reinterpret_cast<const int4v *>(p), x, acc[0], sw, sx);
        acc[1] = mfma<1, 0>(*reinterpret_cast<const int4v *>(p + 1024), x, acc[1], sw, sx);
        acc[2] = mfma<2, 0>(*reinterpret_cast<const int4v *>(p + 2048), x, acc[2], sw, sx);
        acc[3] = mfma<3, 0>(*reinterpret_cast<const int4v *>(p + 3072), x, acc[3], sw, sx);
    }
    const int64_t i = mb * 16 + (lane & 15);
    if (i >= m) return;
    T *row = out + b * batch_stride + i * row_stride;
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t j = (nb * 4 + wave) * 64 + f * 16 + (lane >> 4) * 4 + e;
            if (j < n) store(row + j, acc[f][e]);
        }
}

}  // namespace

bool mx4_matmul_launch(const void *a_codes, const void *a_scales, const void *w_codes, const void *w_scales,
                       int64_t batch, int64_t m, int64_t n, int64_t k, void *out, bool bf16, int64_t batch_stride,
                       int64_t row_stride, hipStream_t stream) {
    if (batch == 0 || m == 0 || n == 0) return true;
    const int64_t nb = (mx4_row_tiles(n) + 3) / 4, mb = (m + 15) / 16, blocks = batch * nb * mb;
    if (blocks > INT32_MAX) return false;
    auto u = [](const void *p) { return static_cast<const uint8_t *>(p); };
    if (bf16)
        product_kernel<<<static_cast<int>(blocks), 256, 0, stream>>>(
            u(a_codes), u(a_scales), u(w_codes), u(w_scales), m, n, mx4_col_tiles(k), nb, mb,
            static_cast<uint16_t *>(out), batch_stride, row_stride);
    else
        product_kernel<<<static_cast<int>(blocks), 256, 0, stream>>>(
            u(a_codes), u(a_scales), u(w_codes), u(w_scales), m, n, mx4_col_tiles(k), nb, mb,
            static_cast<float *>(out), batch_stride, row_stride);
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
