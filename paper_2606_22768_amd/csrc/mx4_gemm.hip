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

// Four consecutive outputs at an address aligned to its element only.
struct __attribute__((packed, aligned(4))) Four32 {
    float v[4];
};
struct __attribute__((packed, aligned(2))) Four16 {
    uint32_t v[2];
};
__device__ inline void store4(float *p, float4v v) {
    *reinterpret_cast<Four32 *>(p) = Four32{{v[0], v[1], v[2], v[3]}};
}
__device__ inline void store4(uint16_t *p, float4v v) {
    *reinterpret_cast<Four16 *>(p) =
        Four16{{round_bf16(v[0]) | static_cast<uint32_t>(round_bf16(v[1])) << 16,
                round_bf16(v[2]) | static_cast<uint32_t>(round_bf16(v[3])) << 16}};
}

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

// ------------------------------------------------------------ large products
//
// Four waves in a 2 x 2 square; each holds WN x WA tiles of 64 x 64 outputs
// (rows of w by rows of a) in registers.

// Tiles of one step of 128 columns, in registers on their way to LDS: a
// thread moves 16 bytes of each tile's codes and one scale dword of each
// operand.
template <int N, int A>
struct Stage {
    int4v w[N], a[A];
    int sw, sa;
};

template <int WN, int WA, typename T>
__global__ __launch_bounds__(256, 1) void tiled_kernel(const uint8_t *__restrict__ a_codes,
                                                       const uint8_t *__restrict__ a_scales,
                                                       const uint8_t *__restrict__ w_codes,
                                                       const uint8_t *__restrict__ w_scales, int64_t m, int64_t n,
                                                       int kt, int64_t batch, int n_blocks, int a_blocks, int blocks_per_xcd,
                                                       T *__restrict__ out, int64_t batch_stride,
                                                       int64_t row_stride) {
    constexpr int N = 2 * WN, A = 2 * WA;  // tiles of a block
    constexpr int kStage = (N + A) * (kMx4CodeBytes + kMx4ScaleBytes), kSlots = 3;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kSlots * kStage];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = wave & 1, wa = wave >> 1;
    // Blocks go to the eight dies in turn; each die takes a contiguous range
    // of tiles, the rows of a running fastest, so that a die's L2 serves one
    // range of w to all of them.
    const int64_t id = static_cast<int64_t>(blockIdx.x & 7) * blocks_per_xcd + (blockIdx.x >> 3);
    const int64_t per_batch = static_cast<int64_t>(n_blocks) * a_blocks, b = id / per_batch;
    const int nb = static_cast<int>(id % per_batch / a_blocks), ab = static_cast<int>(id % a_blocks);
    const int64_t a_tiles = (m + 63) / 64, w_tiles = (n + 63) / 64;
    if (b >= batch) return;

    const uint8_t *wc[N], *ac[A];
#pragma unroll
    for (int j = 0; j < N; ++j)  // tiles past the end repeat the last one, unstored
        wc[j] = w_codes + (b * w_tiles + min(static_cast<int64_t>(nb) * N + j, w_tiles - 1)) * kt * kMx4CodeBytes +
                tid * 16;
#pragma unroll
    for (int j = 0; j < A; ++j)
        ac[j] = a_codes + (b * a_tiles + min(static_cast<int64_t>(ab) * A + j, a_tiles - 1)) * kt * kMx4CodeBytes +
                tid * 16;
    const uint8_t *ws = w_scales +
                        (b * w_tiles + min(static_cast<int64_t>(nb) * N + (wave & (N - 1)), w_tiles - 1)) * kt *
                            kMx4ScaleBytes +
                        lane * 4;
    const uint8_t *as = a_scales +
                        (b * a_tiles + min(static_cast<int64_t>(ab) * A + (wave & (A - 1)), a_tiles - 1)) * kt *
                            kMx4ScaleBytes +
                        lane * 4;

    Stage<N, A> st;
    auto fetch = [&](int k) {
#pragma unroll
        for (int j = 0; j < N; ++j) st.w[j] = *reinterpret_cast<const int4v *>(wc[j] + static_cast<int64_t>(k) * kMx4CodeBytes);
#pragma unroll
        for (int j = 0; j < A; ++j) st.a[j] = *reinterpret_cast<const int4v *>(ac[j] + static_cast<int64_t>(k) * kMx4CodeBytes);
        st.sw = *reinterpret_cast<const int *>(ws + static_cast<int64_t>(k) * kMx4ScaleBytes);
        st.sa = *reinterpret_cast<const int *>(as + static_cast<int64_t>(k) * kMx4ScaleBytes);
    };
    auto put = [&](int slot) {
        uint8_t *p = lds + slot * kStage;
#pragma unroll
        for (int j = 0; j < N; ++j) *reinterpret_cast<int4v *>(p + j * kMx4CodeBytes + tid * 16) = st.w[j];
#pragma unroll
        for (int j = 0; j < A; ++j) *reinterpret_cast<int4v *>(p + (N + j) * kMx4CodeBytes + tid * 16) = st.a[j];
        uint8_t *q = p + (N + A) * kMx4CodeBytes;
        if (wave < N) *reinterpret_cast<int *>(q + tid * 4) = st.sw;
        if (wave < A) *reinterpret_cast<int *>(q + N * kMx4ScaleBytes + tid * 4) = st.sa;
    };
    auto w_frag = [&](int slot, int f) {
        return *reinterpret_cast<const int4v *>(lds + slot * kStage + wn * WN * kMx4CodeBytes + f * 1024 + lane * 16);
    };
    auto a_frag = [&](int slot, int f) {
        return *reinterpret_cast<const int4v *>(lds + slot * kStage + (N + wa * WA) * kMx4CodeBytes + f * 1024 +
                                                lane * 16);
    };
    auto w_scale = [&](int slot, int t) {
        return *reinterpret_cast<const int *>(lds + slot * kStage + (N + A) * kMx4CodeBytes +
                                              (wn * WN + t) * kMx4ScaleBytes + lane * 4);
    };
    auto a_scale = [&](int slot, int t) {
        return *reinterpret_cast<const int *>(lds + slot * kStage + (N + A) * kMx4CodeBytes +
                                              (N + wa * WA + t) * kMx4ScaleBytes + lane * 4);
    };

    float4v acc[4 * WN][4 * WA] = {};
    fetch(0);
    put(0);
    if (kt > 1) {
        fetch(1);
        put(1);
    }
    if (kt > 2) fetch(2);
    int slot = 0;
    for (int k = 0; k < kt; ++k) {
        __syncthreads();
        const int after = slot == 2 ? 0 : slot + 1, last = after == 2 ? 0 : after + 1;
        int4v y[4 * WA];
        int sy[WA];
#pragma unroll
        for (int f = 0; f < 4 * WA; ++f) y[f] = a_frag(slot, f);
#pragma unroll
        for (int t = 0; t < WA; ++t) sy[t] = a_scale(slot, t);
        if (k + 2 < kt) put(last);
        if (k + 3 < kt) fetch(k + 3);
#pragma unroll
        for (int t = 0; t < WN; ++t) {
            const int sx = w_scale(slot, t);
            int4v x[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) x[f] = w_frag(slot, 4 * t + f);
#pragma unroll
            for (int u = 0; u < WA; ++u)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    auto *c = acc[4 * t];
                    const int4v yy = y[4 * u + g];
                    const int j = 4 * u + g;
                    if (g == 0) {
                        acc[4 * t + 0][j] = mfma<0, 0>(x[0], yy, acc[4 * t + 0][j], sx, sy[u]);
                        acc[4 * t + 1][j] = mfma<1, 0>(x[1], yy, acc[4 * t + 1][j], sx, sy[u]);
                        acc[4 * t + 2][j] = mfma<2, 0>(x[2], yy, acc[4 * t + 2][j], sx, sy[u]);
                        acc[4 * t + 3][j] = mfma<3, 0>(x[3], yy, acc[4 * t + 3][j], sx, sy[u]);
                    } else if (g == 1) {
                        acc[4 * t + 0][j] = mfma<0, 1>(x[0], yy, acc[4 * t + 0][j], sx, sy[u]);
                        acc[4 * t + 1][j] = mfma<1, 1>(x[1], yy, acc[4 * t + 1][j], sx, sy[u]);
                        acc[4 * t + 2][j] = mfma<2, 1>(x[2], yy, acc[4 * t + 2][j], sx, sy[u]);
                        acc[4 * t + 3][j] = mfma<3, 1>(x[3], yy, acc[4 * t + 3][j], sx, sy[u]);
                    } else if (g == 2) {
                        acc[4 * t + 0][j] = mfma<0, 2>(x[0], yy, acc[4 * t + 0][j], sx, sy[u]);
                        acc[4 * t + 1][j] = mfma<1, 2>(x[1], yy, acc[4 * t + 1][j], sx, sy[u]);
                        acc[4 * t + 2][j] = mfma<2, 2>(x[2], yy, acc[4 * t + 2][j], sx, sy[u]);
                        acc[4 * t + 3][j] = mfma<3, 2>(x[3], yy, acc[4 * t + 3][j], sx, sy[u]);
                    } else {
                        acc[4 * t + 0][j] = mfma<0, 3>(x[0], yy, acc[4 * t + 0][j], sx, sy[u]);
                        acc[4 * t + 1][j] = mfma<1, 3>(x[1], yy, acc[4 * t + 1][j], sx, sy[u]);
                        acc[4 * t + 2][j] = mfma<2, 3>(x[2], yy, acc[4 * t + 2][j], sx, sy[u]);
                        acc[4 * t + 3][j] = mfma<3, 3>(x[3], yy, acc[4 * t + 3][j], sx, sy[u]);
                    }
                    (void)c;
                }
        }
        slot = after;
    }
    const int64_t n0 = (static_cast<int64_t>(nb) * N + wn * WN) * 64 + (lane >> 4) * 4;
    const int64_t m0 = (static_cast<int64_t>(ab) * A + wa * WA) * 64 + (lane & 15);
#pragma unroll
    for (int j = 0; j < 4 * WA; ++j) {
        const int64_t i = m0 + j * 16;
        if (i < m) {
            T *row = out + b * batch_stride + i * row_stride;
#pragma unroll
            for (int f = 0; f < 4 * WN; ++f) {
                const int64_t c = n0 + f * 16;
                if (c + 3 < n) {
                    store4(row + c, acc[f][j]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < n) store(row + c + e, acc[f][j][e]);
                }
            }
        }
    }
}

template <int WN, int WA, typename T>
bool launch_tiled(const uint8_t *ac, const uint8_t *as, const uint8_t *wc, const uint8_t *ws, int64_t batch, int64_t m,
                  int64_t n, int64_t kt, T *out, int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    const int64_t nb = (mx4_row_tiles(n) + 2 * WN - 1) / (2 * WN), ab = (mx4_row_tiles(m) + 2 * WA - 1) / (2 * WA);
    const int64_t per = (batch * nb * ab + 7) / 8;
    if (per * 8 > INT32_MAX || kt > INT32_MAX) return false;
    tiled_kernel<WN, WA, T><<<dim3(static_cast<unsigned>(per * 8), 1), 256, 0, stream>>>(
        ac, as, wc, ws, m, n, static_cast<int>(kt), batch, static_cast<int>(nb), static_cast<int>(ab), static_cast<int>(per),
        out, batch_stride, row_stride);
    return hipGetLastError() == hipSuccess;
}

template <typename T>
bool launch(const uint8_t *ac, const uint8_t *as, const uint8_t *wc, const uint8_t *ws, int64_t batch, int64_t m,
            int64_t n, int64_t kt, T *out, int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    if (m > 64) return launch_tiled<2, 2>(ac, as, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
    const int64_t nb = (mx4_row_tiles(n) + 3) / 4, mb = (m + 15) / 16, blocks = batch * nb * mb;
    if (blocks > INT32_MAX) return false;
    product_kernel<<<static_cast<int>(blocks), 256, 0, stream>>>(ac, as, wc, ws, m, n, kt, nb, mb, out, batch_stride,
                                                                 row_stride);
    return hipGetLastError() == hipSuccess;
}

}  // namespace

bool mx4_matmul_launch(const void *a_codes, const void *a_scales, const void *w_codes, const void *w_scales,
                       int64_t batch, int64_t m, int64_t n, int64_t k, void *out, bool bf16, int64_t batch_stride,
                       int64_t row_stride, hipStream_t stream) {
    if (batch == 0 || m == 0 || n == 0) return true;
    const int64_t kt = mx4_col_tiles(k);
    auto u = [](const void *p) { return static_cast<const uint8_t *>(p); };
    return bf16 ? launch(u(a_codes), u(a_scales), u(w_codes), u(w_scales), batch, m, n, kt,
                         static_cast<uint16_t *>(out), batch_stride, row_stride, stream)
                : launch(u(a_codes), u(a_scales), u(w_codes), u(w_scales), batch, m, n, kt, static_cast<float *>(out),
                         batch_stride, row_stride, stream);
}

}  // namespace fgd
