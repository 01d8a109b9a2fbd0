// mx4_gemm.hip -- products of matrices in microscaled 4-bit floating point
// (the format and its layout: mx4.hpp).
//
// out[i][j] = sum over k of a[i][k] w[j][k].  A product of two values is
// exact in float32 (four significant bits); the matrix instruction multiplies
// by both blocks' scales and adds in float32, and the sum is rounded once, to
// the output's type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "mx4.hpp"
#include "mx4_block.hpp"

namespace fgd {
namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

// 32 rows of w by 32 rows of a over 64 columns: fragments of 1 KB (lane l
// holds row l % 32 of the block l / 32), scales the bytes SW and SA of each
// lane's dwords.  Result: lane l holds row l % 32 of a and, in element i, row
// 8 (i / 4) + 4 (l / 32) + i % 4 of w.
template <int SW, int SA>
__device__ inline float16v mfma(int4v w, int4v a, float16v c, int sw, int sa) {
    const int8v x = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, y = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, SW, sw, SA, sa);  // 4, 4: both 4-bit
}

__device__ inline uint16_t round_bf16(float v) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return static_cast<uint16_t>((u >> 16) | 0x40u);
    return static_cast<uint16_t>((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// Consecutive outputs at an address aligned to its element only.
struct __attribute__((packed, aligned(4))) Four32 {
    float v[4];
};
struct __attribute__((packed, aligned(2))) Four16 {
    uint32_t v[2];
};
struct __attribute__((packed, aligned(2))) Eight16 {
    uint32_t v[4];
};

// Four columns of a row.
__device__ inline void store4(float *row, int64_t c, int64_t n, float4v v) {
    if (c + 3 < n) {
        *reinterpret_cast<Four32 *>(row + c) = Four32{{v[0], v[1], v[2], v[3]}};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < n) row[c + e] = v[e];
    }
}
__device__ inline void store4(uint16_t *row, int64_t c, int64_t n, float4v v) {
    if (c + 3 < n) {
        *reinterpret_cast<Four16 *>(row + c) =
            Four16{{round_bf16(v[0]) | static_cast<uint32_t>(round_bf16(v[1])) << 16,
                    round_bf16(v[2]) | static_cast<uint32_t>(round_bf16(v[3])) << 16}};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < n) row[c + e] = round_bf16(v[e]);
    }
}

// Stores a 32 x 32 result, whose rows are the first m of those at `rows` and
// whose columns are the first n of those there; ALL: all are, and there are
// kStores<T> stores that nothing skips.  Lanes first exchange registers, so
// that four of them, l % 16 alike, store 64 consecutive bytes of a row.
// (Whole lines by way of LDS, pieces of 32 bytes and stores past the caches
// measured no faster at 2048 x 128256 x 4096 to bf16: 4, 0 and 20% slower.)
template <typename T>
constexpr int kStores = sizeof(T);

template <bool ALL>
__device__ inline void store_rows(float *rows, int64_t stride, int64_t m, int64_t n, int lane, float16v v) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
        float4v even, odd;  // of rows r and r + 16: the 4 columns from c
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[4 * q + e]),
                                                            __float_as_uint(v[4 * q + 4 + e]), false, false);
            even[e] = __uint_as_float(x[0]), odd[e] = __uint_as_float(x[1]);
        }
        const int c = 8 * q + (g & 1) * 8 + (g >> 1) * 4;
        if (ALL) {
            *reinterpret_cast<Four32 *>(rows + r * stride + c) = Four32{{even[0], even[1], even[2], even[3]}};
            *reinterpret_cast<Four32 *>(rows + (r + 16) * stride + c) = Four32{{odd[0], odd[1], odd[2], odd[3]}};
        } else {
            if (r < m) store4(rows + r * stride, c, n, even);
            if (r + 16 < m) store4(rows + (r + 16) * stride, c, n, odd);
        }
    }
}

__device__ inline void store8(uint16_t *row, int64_t c, int64_t n, Eight16 x) {
    if (c + 7 < n) {
        *reinterpret_cast<Eight16 *>(row + c) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < n) row[c + e] = static_cast<uint16_t>(x.v[e >> 1] >> (16 * (e & 1)));
    }
}
template <bool ALL>
__device__ inline void store_rows(uint16_t *rows, int64_t stride, int64_t m, int64_t n, int lane, float16v v) {
    const int r = lane & 15, g = lane >> 4;
    uint32_t w[8];  // columns 8 i + 4 (lane / 32) .. + 3 in w[2 i ..]
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i] = round_bf16(v[2 * i]) | static_cast<uint32_t>(round_bf16(v[2 * i + 1])) << 16;
    Eight16 even, odd;  // of rows r and r + 16: the 8 columns from c
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        // Eight columns a lane, 8 (lane / 32) .. + 7 of each 16 ...
        const auto lo = __builtin_amdgcn_permlane32_swap(w[i], w[2 + i], false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(w[4 + i], w[6 + i], false, false);
        // ... then those of 16 rows.
        const auto x = __builtin_amdgcn_permlane16_swap(lo[0], hi[0], false, false);
        const auto y = __builtin_amdgcn_permlane16_swap(lo[1], hi[1], false, false);
        even.v[i] = x[0], odd.v[i] = x[1], even.v[2 + i] = y[0], odd.v[2 + i] = y[1];
    }
    const int c = (g & 1) * 16 + (g >> 1) * 8;
    if (ALL) {
        *reinterpret_cast<Eight16 *>(rows + r * stride + c) = even;
        *reinterpret_cast<Eight16 *>(rows + (r + 16) * stride + c) = odd;
    } else {
        if (r < m) store8(rows + r * stride, c, n, even);
        if (r + 16 < m) store8(rows + (r + 16) * stride, c, n, odd);
    }
}

// --------------------------------------------------------------- few tokens
//
// A block multiplies NW fragments of 32 rows of w by NA fragments of 32 rows
// of a; its waves share out the columns, tile by tile in turn, and add their
// sums through LDS in the waves' order.  Every operand goes straight from
// memory to registers: w is read once, and a comes from L2.  Bound by the
// read of w: 1 x 128256 x 2048 (140 MB) in 25 us, 5.5 TB/s (22 with w in the
// last-level cache); 9 x 16 x 32000 x 1024 (157 MB, 18 written) in 34 (26); 64 x
// 8192 x 8192 (36 MB) in 11, of which the first loads, the sums and the launch
// are half.
template <int NA>
__device__ inline void products(float16v (&acc)[1][NA], const int4v (&x)[1][2], const int4v (&y)[NA][2], int sw, int sa) {
    acc[0][0] = mfma<0, 0>(x[0][0], y[0][0], acc[0][0], sw, sa);
    if constexpr (NA == 2) acc[0][1] = mfma<0, 2>(x[0][0], y[1][0], acc[0][1], sw, sa);
    acc[0][0] = mfma<1, 1>(x[0][1], y[0][1], acc[0][0], sw, sa);
    if constexpr (NA == 2) acc[0][1] = mfma<1, 3>(x[0][1], y[1][1], acc[0][1], sw, sa);
}
template <int NA>
__device__ inline void products(float16v (&acc)[2][NA], const int4v (&x)[2][2], const int4v (&y)[NA][2], int sw, int sa) {
    acc[0][0] = mfma<0, 0>(x[0][0], y[0][0], acc[0][0], sw, sa);
    acc[1][0] = mfma<2, 0>(x[1][0], y[0][0], acc[1][0], sw, sa);
    if constexpr (NA == 2) {
        acc[0][1] = mfma<0, 2>(x[0][0], y[1][0], acc[0][1], sw, sa);
        acc[1][1] = mfma<2, 2>(x[1][0], y[1][0], acc[1][1], sw, sa);
    }
    acc[0][0] = mfma<1, 1>(x[0][1], y[0][1], acc[0][0], sw, sa);
    acc[1][0] = mfma<3, 1>(x[1][1], y[0][1], acc[1][0], sw, sa);
    if constexpr (NA == 2) {
        acc[0][1] = mfma<1, 3>(x[0][1], y[1][1], acc[0][1], sw, sa);
        acc[1][1] = mfma<3, 3>(x[1][1], y[1][1], acc[1][1], sw, sa);
    }
}

// The left operand: in the 4-bit format, or (X: float, or uint16_t for bf16)
// dense rows that the block quantises itself.
struct Packed {
    const uint8_t *codes, *scales;
};
template <typename X>
struct Dense {
    const X *x;
    int64_t batch_stride, row_stride, cols;
};

template <int NW, int NA, int WAVES, int AHEAD, typename T, typename Left>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(Left left, const uint8_t *__restrict__ w_codes,
                                                         const uint8_t *__restrict__ w_scales, int64_t m, int64_t n,
                                                         int kt, int64_t n_blocks, int64_t m_blocks,
                                                         int64_t first_batch, T *__restrict__ out, int64_t batch_stride,
                                                         int64_t row_stride) {
    constexpr bool kDense = !std::is_same<Left, Packed>::value;
    static_assert(!kDense || NA == 1, "dense rows: of one fragment");
    __shared__ float4v sums[WAVES][4 * NW * NA][64];
    // Dense rows' blocks, block by block of the columns: one per thread.
    __shared__ int4v x_codes[kDense ? 64 * WAVES : 1];
    __shared__ uint8_t x_scales[kDense ? 64 * WAVES : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t w_tiles = (n + 63) / 64, items = n_blocks * m_blocks;
    const int64_t b = first_batch + blockIdx.y;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t nb = item % n_blocks, mb = item / n_blocks;
        const int wh = NW == 2 ? 0 : nb & 1, ah = NA == 2 ? 0 : mb & 1;  // the half of a tile, where it is one
        const int64_t wt = b * w_tiles + (NW == 2 ? nb : nb >> 1);
        const uint8_t *wc = w_codes + wt * kt * kMx4CodeBytes + wh * 2048 + lane * 16;
        const uint8_t *ws = w_scales + wt * kt * kMx4ScaleBytes + lane * 4;
        const uint8_t *ac = nullptr, *as = nullptr;
        if constexpr (!kDense) {
            const int64_t at = b * ((m + 63) / 64) + (NA == 2 ? mb : mb >> 1);
            ac = left.codes + at * kt * kMx4CodeBytes + ah * 2048 + lane * 16;
            as = left.scales + at * kt * kMx4ScaleBytes + lane * 4;
        }
        // Rows past the last token are not loaded, but zero.
        bool some[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) some[i] = (mb * NA + i) * 32 + (lane & 31) < m;
        float16v acc[NW][NA] = {};
        bool fresh = kDense && item == blockIdx.x;
        for (int k0 = wave; k0 < kt || fresh; k0 += WAVES * AHEAD) {
            // AHEAD tiles' loads go out before the first product waits.
            int4v x[AHEAD][NW][2], y[AHEAD][NA][2];
            int sw[AHEAD], sa[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int k = min(k0 + u * WAVES, kt - 1);  // past the last tile: that one again, times zero
                const int64_t co = static_cast<int64_t>(k) * kMx4CodeBytes,
                              so = static_cast<int64_t>(k) * kMx4ScaleBytes;
                sw[u] = *reinterpret_cast<const int *>(ws + so) >> (16 * wh);
#pragma unroll
                for (int i = 0; i < 2 * NW; ++i)
                    x[u][i / 2][i % 2] = *reinterpret_cast<const int4v *>(wc + co + i * 1024);
                if constexpr (!kDense) {
                    sa[u] = *reinterpret_cast<const int *>(as + so) >> (16 * ah);
#pragma unroll
                    for (int i = 0; i < 2 * NA; ++i) {
                        y[u][i / 2][i % 2] = int4v{0, 0, 0, 0};
                        if (some[i / 2] && k0 + u * WAVES < kt)
                            y[u][i / 2][i % 2] = *reinterpret_cast<const int4v *>(ac + co + i * 1024);
                    }
                }
            }
            if constexpr (kDense) {
                const int tokens = static_cast<int>(m);
                if (fresh) {  // with the first weights on their way
                    const int row = threadIdx.x % tokens, block = threadIdx.x / tokens;
                    if (block < 4 * kt) {
                        const int64_t c0 = 32 * static_cast<int64_t>(block);
                        float v[32];
                        load_block(left.x + b * left.batch_stride + row * left.row_stride + c0, left.cols - c0,
                                   v);
                        uint4 c;
                        x_scales[threadIdx.x] = static_cast<uint8_t>(encode_block(v, c));
                        x_codes[threadIdx.x] = int4v{static_cast<int>(c.x), static_cast<int>(c.y),
                                                     static_cast<int>(c.z), static_cast<int>(c.w)};
                    }
                    __syncthreads();
                    fresh = false;
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    sa[u] = 0;
                    y[u][0][0] = y[u][0][1] = int4v{0, 0, 0, 0};
                    if (some[0] && k0 + u * WAVES < kt) {
                        const int at = (4 * (k0 + u * WAVES) + (lane >> 5)) * tokens + (lane & 31);
                        y[u][0][0] = x_codes[at];
                        y[u][0][1] = x_codes[at + 2 * tokens];
                        sa[u] = x_scales[at] | x_scales[at + 2 * tokens] << 8;
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) products(acc, x[u], y[u], sw[u], sa[u]);
        }
        // Each wave leaves its sums in LDS, and adds up its share of the
        // groups of four columns.
#pragma unroll
        for (int i = 0; i < NW * NA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float16v &v = acc[i / NA][i % NA];
                sums[wave][4 * i + q][lane] = float4v{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
            }
        __syncthreads();
#pragma unroll
        for (int g = wave; g < 4 * NW * NA; g += WAVES) {
            float4v v = sums[0][g][lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v += sums[w][g][lane];
            const int64_t i = (mb * NA + g / 4 % NA) * 32 + (lane & 31);
            const int64_t c = (nb * NW + g / 4 / NA) * 32 + (g & 3) * 8 + (lane >> 5) * 4;
            if (i < m) store4(out + b * batch_stride + i * row_stride, c, n, v);
        }
        if (item + gridDim.x < items) __syncthreads();  // before the sums' room is used again
    }
}

// A tile of w (its fragments x) by a tile of a (y) over 128 columns.
template <int NW, int NA>
__device__ inline void outer(float16v (&acc)[NW][NA], int i, int j, const int4v *x, const int4v *y, int sx,
                             int sy) {
    acc[i][j] = mfma<0, 0>(x[0], y[0], acc[i][j], sx, sy);
    acc[i + 1][j] = mfma<2, 0>(x[2], y[0], acc[i + 1][j], sx, sy);
    acc[i][j + 1] = mfma<0, 2>(x[0], y[2], acc[i][j + 1], sx, sy);
    acc[i + 1][j + 1] = mfma<2, 2>(x[2], y[2], acc[i + 1][j + 1], sx, sy);
    acc[i][j] = mfma<1, 1>(x[1], y[1], acc[i][j], sx, sy);
    acc[i + 1][j] = mfma<3, 1>(x[3], y[1], acc[i + 1][j], sx, sy);
    acc[i][j + 1] = mfma<1, 3>(x[1], y[3], acc[i][j + 1], sx, sy);
    acc[i + 1][j + 1] = mfma<3, 3>(x[3], y[3], acc[i + 1][j + 1], sx, sy);
}

// Waits until at most N of this wave's loads and stores are on their way.
template <int N>
__device__ inline void outstanding() {
    static_assert(N < 64, "the counter's range");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
    asm volatile("" ::: "memory");
}
// The same, and until all that it read from LDS has come, then for the
// block's other waves.
template <int LOADS>
__device__ inline void arrive() {
    static_assert(LOADS < 64, "the counter's range");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LOADS & 15) | 7 << 4 | (LOADS >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Orders a step's instructions: products with the reads of LDS and the loads
// spread evenly between them, since a wave issues in order and would wait at
// a full LDS queue with its matrix unit idle.
template <int PRODUCTS, int READS, int LOADS>
__device__ inline void interleave() {
    constexpr int kOther = READS + LOADS;
#pragma unroll
    for (int i = 0, done = 0; i < PRODUCTS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        const int upto = (i + 1) * kOther / PRODUCTS;
#pragma unroll
        for (; done < upto; ++done) {
            if (done < READS)
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            else
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
    }
}

// ------------------------------------------------------------ large products
//
// GN x GA waves, each holding WN x WA tiles of 64 x 64 outputs (rows of w by
// rows of a) in registers.  A block takes block after block of the outputs,
// as one run of steps: the first tiles of the next are on their way while the
// last products of one are stored (6% less time than a block each at 2048 x
// 128256 x 4096 to bf16, 3% at 8192^3).  8192^3 takes 255 to 270 us, 4.1 to 4.3
// PFLOP/s, 2048 x 128256 x 4096 to bf16 564 to 591, from card to card.  Bound by
// the matrix units: busy for 57% of the cycles of a clock that their power
// lowers to 1.8 GHz (operands of zeros: 181 us at 2.46 GHz; without a step's
// loads and reads: 232 to 242), and, where n is large, by stores that the steps
// do not hide (without them 2048 x 128256 x 4096 takes 7% less).
template <int GN, int GA, int WN, int WA, typename T>
__global__ __launch_bounds__(64 * GN * GA, (WN * WA >= 4 ? 1 : 2)) void tiled_kernel(
    const uint8_t *__restrict__ a_codes, const uint8_t *__restrict__ a_scales, const uint8_t *__restrict__ w_codes,
    const uint8_t *__restrict__ w_scales, int64_t m, int64_t n, int kt, int64_t batch, int n_blocks, int a_blocks,
    int blocks_per_xcd, T *__restrict__ out, int64_t batch_stride, int64_t row_stride) {
    constexpr int N = GN * WN, A = GA * WA, kThreads = 64 * GN * GA;  // tiles of a block
    constexpr int kCodes = (N + A) * 256 / kThreads, kScales = ((N + A) * 64 + kThreads - 1) / kThreads;
    constexpr int kLoads = kCodes + kScales, kSlots = 3;
    // Every wave issues the same loads, so that it can count them: scales
    // past the last tile's repeat its, behind them.
    constexpr int kStage = (N + A) * kMx4CodeBytes + kScales * kThreads * 4;
    static_assert(kCodes * kThreads == (N + A) * 256, "whole chunks per thread");
    __shared__ __attribute__((aligned(16))) uint8_t lds[kSlots * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = wave % GN,
              wa = wave / GN;
    // Blocks go to the eight dies in turn; each die takes a contiguous range
    // of the order below, in which 32 neighbours (a die's compute units) are
    // 4 blocks of a by 8 of w: what its L2 serves to all of them is least, as
    // with 8 by 4, and the pieces of a row that are written at a time are
    // longer (2048 x 131072 x 4096: 607 us for 668 with 8 by 4 on one card; the
    // same time at 128256, whose rows start off the lines).
    const uint32_t per_batch = static_cast<uint32_t>(n_blocks) * a_blocks, first = (blockIdx.x & 7) * blocks_per_xcd;
    const int count = static_cast<int>(min(static_cast<int64_t>(blocks_per_xcd), batch * per_batch - first));
    const int stride = gridDim.x >> 3;
    const int64_t a_tiles = (m + 63) / 64, w_tiles = (n + 63) / 64;
    struct Place {
        int64_t b, nb, ab;
    };
    auto place_of = [&](int item) {
        const uint32_t id = first + item, b = id / per_batch, in_batch = id - b * per_batch, across = 4u * n_blocks;
        const uint32_t strip = in_batch / across * 4, in_strip = in_batch % across,
                       width = min(4u, static_cast<uint32_t>(a_blocks) - strip);
        auto uniform = [](uint32_t v) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(v)); };
        return Place{uniform(b), uniform(in_strip / width), uniform(strip + in_strip % width)};
    };

    // What is loaded next: step `ahead` of a block of the outputs.  A wave's
    // chunks of 64 lanes lie within a tile.
    const uint8_t *code_src[kCodes], *scale_src[kScales];
    int item = blockIdx.x >> 3, loading = item, ahead = 0;
    if (item >= count) return;
    auto aim = [&] {
        const Place at = place_of(loading);
        // Tiles past the end repeat the last one, unstored.
        auto tile_of = [&](int j) {
            return j < N ? at.b * w_tiles + min(at.nb * N + j, w_tiles - 1)
                         : at.b * a_tiles + min(at.ab * A + (j - N), a_tiles - 1);
        };
#pragma unroll
        for (int i = 0; i < kCodes; ++i) {
            const int c = i * kThreads + wave * 64, j = c >> 8;
            code_src[i] = (j < N ? w_codes : a_codes) + tile_of(j) * kt * kMx4CodeBytes + (c & 255) * 16;
        }
#pragma unroll
        for (int i = 0; i < kScales; ++i) {
            const int j = min(i * (kThreads / 64) + wave, N + A - 1);
            scale_src[i] = (j < N ? w_scales : a_scales) + tile_of(j) * kt * kMx4ScaleBytes;
        }
    };
    // Copies its tiles to a slot: 16 (or 4) bytes a lane, straight to LDS.
    const uint32_t lane16 = lane * 16, lane4 = lane * 4;
    auto fetch = [&](int slot) {
        uint8_t *p = lds + slot * kStage, *q = p + (N + A) * kMx4CodeBytes;
#pragma unroll
        for (int i = 0; i < kCodes; ++i)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)(code_src[i] +
                                                                 static_cast<int64_t>(ahead) * kMx4CodeBytes + lane16),
                (__attribute__((address_space(3))) void *)(p + (i * kThreads + wave * 64) * 16), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < kScales; ++i)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)(scale_src[i] +
                                                                 static_cast<int64_t>(ahead) * kMx4ScaleBytes + lane4),
                (__attribute__((address_space(3))) void *)(q + (i * kThreads + wave * 64) * 4), 4, 0, 0);
    };
    // Past the last step that one is loaded again, and unused: a branch
    // around the loads would cost the registers that hold the result.
    auto advance = [&] {
        if (++ahead < kt) return;
        ahead = kt - 1;
        if (loading + stride >= count) return;
        ahead = 0;
        loading += stride;
        aim();
    };
    auto frag = [&](int slot, int tile, int f) {
        return *reinterpret_cast<const int4v *>(lds + slot * kStage + tile * kMx4CodeBytes + f * 1024 + lane * 16);
    };
    auto scales = [&](int slot, int tile) {
        return *reinterpret_cast<const int *>(lds + slot * kStage + (N + A) * kMx4CodeBytes + tile * kMx4ScaleBytes +
                                              lane * 4);
    };

    float16v acc[2 * WN][2 * WA];
    // A step's operands in registers.
    struct Operands {
        int4v w[4 * WN], a[4 * WA];
        int sw[WN], sa[WA];
    } held[2];
    auto read = [&](Operands &r, int slot) {
#pragma unroll
        for (int t = 0; t < WA; ++t) r.sa[t] = scales(slot, N + wa * WA + t);
#pragma unroll
        for (int t = 0; t < WN; ++t) r.sw[t] = scales(slot, wn * WN + t);
#pragma unroll
        for (int f = 0; f < 4 * WA; ++f) r.a[f] = frag(slot, N + wa * WA, f);
#pragma unroll
        for (int f = 0; f < 4 * WN; ++f) r.w[f] = frag(slot, wn * WN, f);
    };
    auto multiply = [&](const Operands &r) {
#pragma unroll
        for (int t = 0; t < WN; ++t)
#pragma unroll
            for (int u = 0; u < WA; ++u) outer(acc, 2 * t, 2 * u, r.w + 4 * t, r.a + 4 * u, r.sw[t], r.sa[u]);
        // Keeps the products on their side of the next barrier.
#pragma unroll
        for (int t = 0; t < 2 * WN; ++t)
#pragma unroll
            for (int u = 0; u < 2 * WA; ++u) asm volatile("" : "+v"(acc[t][u]));
    };

    // The ring of slots.  While a step multiplies, its own slot, already read,
    // takes the step kSlots after it, and the next one's operands are read
    // from theirs; the barrier before says that this step is read and the
    // next one has arrived everywhere.  Loads and stores complete in their
    // order: what has to have arrived was issued two steps before, so behind
    // it are one step's loads and, for two steps, the stores of a block.
    constexpr int kBehind = 4 * WN * WA * kStores<T>;
    aim();
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
        fetch(i);
        advance();
    }
    arrive<(kSlots - 1) * kLoads>();
    read(held[0], 0);
    int slot = 0, stored = 0;
    auto step = [&](int p) {
        const int after = slot == kSlots - 1 ? 0 : slot + 1;
        if (stored) {
            --stored;
            outstanding<(kSlots - 2) * kLoads + kBehind>();
        } else {
            outstanding<(kSlots - 2) * kLoads>();
        }
        arrive<(kSlots - 2) * kLoads + kBehind>();
        __builtin_amdgcn_sched_barrier(0);
        read(held[p ^ 1], after);
        fetch(slot);
        multiply(held[p]);
        interleave<8 * WN * WA, 5 * (WN + WA), kLoads>();
        __builtin_amdgcn_sched_barrier(0);
        slot = after;
        advance();
    };
    for (; item < count; item += stride) {
#pragma unroll
        for (int f = 0; f < 2 * WN; ++f)
#pragma unroll
            for (int j = 0; j < 2 * WA; ++j) acc[f][j] = float16v{};
        int k = 0;
        for (; k + 1 < kt; k += 2) {
            step(0);
            step(1);
        }
        if (k < kt) {
            step(0);
            held[0] = held[1];
        }
        const Place at = place_of(item);
        const int64_t n0 = (at.nb * N + wn * WN) * 64,
                      m0 = (at.ab * A + wa * WA) * 64;
        T *to = out + at.b * batch_stride + m0 * row_stride + n0;
        auto store = [&](auto all) {
#pragma unroll
            for (int j = 0; j < 2 * WA; ++j)
#pragma unroll
                for (int f = 0; f < 2 * WN; ++f)
                    store_rows<decltype(all)::value>(to + j * 32 * row_stride + f * 32, row_stride, m - m0 - j * 32,
                                                     n - n0 - f * 32, lane, acc[f][j]);
        };
        if (n0 + 64 * WN <= n && m0 + 64 * WA <= m) {
            store(std::true_type());
            stored = 2;
        } else {
            store(std::false_type());
            outstanding<0>();  // an unknown number of them
        }
    }
    outstanding<0>();  // nothing may still be on its way to this block's LDS
}

template <int GN, int GA, int WN, int WA, typename T>
bool launch_tiled(const uint8_t *ac, const uint8_t *as, const uint8_t *wc, const uint8_t *ws, int64_t batch, int64_t m,
                  int64_t n, int64_t kt, T *out, int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    // A die's range: whole groups of neighbours in either direction.
    const int64_t nb = (mx4_row_tiles(n) + GN * WN - 1) / (GN * WN), ab = (mx4_row_tiles(m) + GA * WA - 1) / (GA * WA);
    const int64_t per = (batch * nb * ab + 63) / 64 * 8;
    if (nb * ab > INT32_MAX / 8 || per > INT32_MAX / 8 || kt > INT32_MAX) return false;
    // As many blocks as the card holds: one of 512 threads a compute unit, two
    // of 256.
    const int64_t held = 32 * 512 / (64 * GN * GA);
    tiled_kernel<GN, GA, WN, WA, T><<<static_cast<unsigned>(std::min(per, held) * 8), 64 * GN * GA, 0, stream>>>(
        ac, as, wc, ws, m, n, static_cast<int>(kt), batch, static_cast<int>(nb), static_cast<int>(ab),
        static_cast<int>(per), out, batch_stride, row_stride);
    return hipGetLastError() == hipSuccess;
}

template <int NW, int NA, int WAVES, int AHEAD, typename T, typename Left>
bool launch_few(Left left, const uint8_t *wc, const uint8_t *ws, int64_t batch, int64_t m, int64_t n, int64_t kt,
                T *out, int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    const int64_t nb = (n + 32 * NW - 1) / (32 * NW), mb = (m + 32 * NA - 1) / (32 * NA);
    if (kt > INT32_MAX / 64) return false;
    // Dense rows are quantised once a block, so there are two blocks a compute
    // unit, which go round (1 x 128256 x 2048 by 256, 512, 768 and 1024
    // blocks: 32, 26, 27 and 29 us).
    const int64_t most = std::is_same<Left, Packed>::value ? 1 << 20 : std::max<int64_t>(1, 512 / batch);
    for (int64_t b = 0; b < batch; b += 65535) {  // a grid's most
        const dim3 grid(static_cast<unsigned>(std::min(nb * mb, most)),
                        static_cast<unsigned>(std::min<int64_t>(batch - b, 65535)));
        few_kernel<NW, NA, WAVES, AHEAD, T, Left><<<grid, 64 * WAVES, 0, stream>>>(
            left, wc, ws, m, n, static_cast<int>(kt), nb, mb, b, out, batch_stride, row_stride);
    }
    return hipGetLastError() == hipSuccess;
}

// Which kernel a product takes.
enum Shape { kFew2x1, kFew2x1Deep, kFew1x1Deep, kFew1x2Deep, kFew2x2, kFew2x2Deep, kTiled128, kTiled256 };

Shape shape_of(int64_t batch, int64_t m, int64_t n, int64_t kt) {
    constexpr int64_t kCus = 256;
    auto blocks = [&](int64_t rows, int64_t cols) { return batch * ((m + rows - 1) / rows) * ((n + cols - 1) / cols); };
    const int64_t small = blocks(128, 128), large = blocks(256, 256);
    if (m > 32 && small >= kCus && kt > 0)
        // Steps of the fullest compute unit: one of a 256 x 256 block costs
        // 3.3 times one of a 128 x 128 block (1.1 and 0.33 us, the card full).
        return 10 * ((small + kCus - 1) / kCus) >= 33 * ((large + kCus - 1) / kCus) ? kTiled256 : kTiled128;
    // Below that a compute unit's block is the smaller, the fewer there are,
    // and its waves share out the columns: eight where there are no more
    // blocks than compute units (5.2 us for four waves' 5.9 at 1 x 2048 x 8192;
    // 11.7 for 14.2 at 1 x 9000 x 8192; 11.8 for 12.8 at 128 x 8192 x 8192),
    // else four (17.0 for 20.2 at 16 x 128256 x 1024, 19.3 for 21.5 at 256 x
    // 8192 x 8192; blocks of 32 rows of w for 64: 19.6).  Over few columns there is
    // little to share, and 128 x 128 tiles are faster: 10.4 us for 16.3 at 777
    // x 4100 x 1000, 10.3 for 15.6 at 64 x 50257 x 768; at 2048 x 1024 x 4096
    // they take 13.6 for 12.0.
    if (blocks(32, 32) <= kCus) return kFew1x1Deep;
    if (m <= 32) return blocks(32, 64) <= kCus ? kFew2x1Deep : kFew2x1;
    if (blocks(64, 32) <= kCus) return kFew1x2Deep;
    if (blocks(64, 64) <= kCus) return kFew2x2Deep;
    return kt > 0 && kt <= 16 ? kTiled128 : kFew2x2;
}

template <typename T>
bool launch(Packed a, const uint8_t *wc, const uint8_t *ws, int64_t batch, int64_t m, int64_t n, int64_t kt, T *out,
            int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    switch (shape_of(batch, m, n, kt)) {
        case kFew2x1:
            return launch_few<2, 1, 4, 2>(a, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        case kFew2x1Deep:
            return launch_few<2, 1, 8, 2>(a, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        case kFew1x1Deep:
            return launch_few<1, 1, 8, 4>(a, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        case kFew1x2Deep:
            return launch_few<1, 2, 8, 2>(a, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        case kFew2x2:
            return launch_few<2, 2, 4, 2>(a, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        case kFew2x2Deep:
            return launch_few<2, 2, 8, 2>(a, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        case kTiled128:
            return launch_tiled<2, 2, 1, 1>(a.codes, a.scales, wc, ws, batch, m, n, kt, out, batch_stride, row_stride,
                                            stream);
        default:
            return launch_tiled<2, 4, 2, 1>(a.codes, a.scales, wc, ws, batch, m, n, kt, out, batch_stride, row_stride,
                                            stream);
    }
}

template <typename T, typename X>
bool launch_dense(Dense<X> x, const uint8_t *wc, const uint8_t *ws, int64_t batch, int64_t m, int64_t n, int64_t kt,
                  T *out, int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    switch (shape_of(batch, m, n, kt)) {
        case kFew2x1:
            return launch_few<2, 1, 4, 2>(x, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        case kFew2x1Deep:
            return launch_few<2, 1, 8, 2>(x, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
        default:
            return launch_few<1, 1, 8, 4>(x, wc, ws, batch, m, n, kt, out, batch_stride, row_stride, stream);
    }
}

}  // namespace

bool mx4_matmul_launch(const void *a_codes, const void *a_scales, const void *w_codes, const void *w_scales,
                       int64_t batch, int64_t m, int64_t n, int64_t k, void *out, bool bf16, int64_t batch_stride,
                       int64_t row_stride, hipStream_t stream) {
    if (batch == 0 || m == 0 || n == 0) return true;
    const int64_t kt = mx4_col_tiles(k);
    auto u = [](const void *p) { return static_cast<const uint8_t *>(p); };
    const Packed a = {u(a_codes), u(a_scales)};
    return bf16 ? launch(a, u(w_codes), u(w_scales), batch, m, n, kt, static_cast<uint16_t *>(out), batch_stride,
                         row_stride, stream)
                : launch(a, u(w_codes), u(w_scales), batch, m, n, kt, static_cast<float *>(out), batch_stride,
                         row_stride, stream);
}

bool mx4_linear_fuses(int64_t batch, int64_t m, int64_t n, int64_t k) {
    if (batch == 0 || m == 0 || n == 0 || k == 0 || m > 32) return false;
    const int64_t kt = mx4_col_tiles(k);
    const Shape shape = shape_of(batch, m, n, kt);
    // A thread quantises a block of x at most.
    return (shape == kFew2x1 && m * 4 * kt <= 256) ||
           ((shape == kFew2x1Deep || shape == kFew1x1Deep) && m * 4 * kt <= 512);
}

bool mx4_linear_launch(const void *x, bool x_bf16, int64_t x_batch_stride, int64_t x_row_stride, const void *w_codes,
                       const void *w_scales, int64_t batch, int64_t m, int64_t n, int64_t k, void *out, bool bf16,
                       int64_t batch_stride, int64_t row_stride, hipStream_t stream) {
    const int64_t kt = mx4_col_tiles(k);
    auto *wc = static_cast<const uint8_t *>(w_codes), *ws = static_cast<const uint8_t *>(w_scales);
    auto go = [&](auto dense) {
        return bf16 ? launch_dense(dense, wc, ws, batch, m, n, kt, static_cast<uint16_t *>(out), batch_stride,
                                   row_stride, stream)
                    : launch_dense(dense, wc, ws, batch, m, n, kt, static_cast<float *>(out), batch_stride, row_stride,
                                   stream);
    };
    return x_bf16 ? go(Dense<uint16_t>{static_cast<const uint16_t *>(x), x_batch_stride, x_row_stride, k})
                  : go(Dense<float>{static_cast<const float *>(x), x_batch_stride, x_row_stride, k});
}

}  // namespace fgd
