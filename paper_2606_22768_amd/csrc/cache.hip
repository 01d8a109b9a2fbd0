// cache.hip -- tokens into and out of a paged 4-bit cache (layout: cache.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.hpp"
#include "mx4_block.hpp"

namespace fgd {
namespace {

typedef float float2v __attribute__((ext_vector_type(2)));

// A thread per block of 32 elements of a token's key or value.
template <typename T>
__global__ __launch_bounds__(256) void write_kernel(CacheView c, HeadRows k, HeadRows v, int64_t tokens,
                                                    const int64_t *__restrict__ slots, int64_t blocks) {
    const int nb = c.dim / 32;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < blocks;
         i += static_cast<int64_t>(gridDim.x) * 256) {
        const int b = static_cast<int>(i % nb);
        int64_t j = i / nb;
        const int h = static_cast<int>(j % c.heads);
        j /= c.heads;
        const bool value = j >= tokens;
        const int64_t t = value ? j - tokens : j, slot = slots[t];
        if (slot < 0 || slot >= c.slots()) continue;
        const HeadRows &x = value ? v : k;
        float e[32];
        load_block(static_cast<const T *>(x.p) + t * x.token_stride + h * x.head_stride + 32 * b, 32, e);
        uint4 code;
        const uint32_t scale = encode_block(e, code);
        const int token = static_cast<int>(slot & 15);
        uint8_t *g = c.data + c.group(slot >> c.page_shift, h, (slot & ((1 << c.page_shift) - 1)) >> 4);
        const uint32_t w[4] = {code.x, code.y, code.z, code.w};
        if (!value) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int piece = 4 * b + p, quarter = piece / nb;
                *reinterpret_cast<uint32_t *>(g + (token + 16 * quarter) * 4 * nb + (piece - quarter * nb) * 4) = w[p];
            }
            g[16 * c.dim + token * nb + b] = static_cast<uint8_t>(scale);
        } else {
            uint8_t *d = g + 8 * c.dim + (token >> 2) * 64 * nb + 4 * b + (token & 3);
#pragma unroll
            for (int n = 0; n < 16; ++n) d[n * 4 * nb] = static_cast<uint8_t>(w[n >> 2] >> (8 * (n & 3)));
            g[16 * c.dim + c.dim / 2 + (token >> 2) * 4 * nb + 4 * b + (token & 3)] = static_cast<uint8_t>(scale);
        }
    }
}

// A thread per 8 elements of a token's key or value.
template <typename T>
__global__ __launch_bounds__(256) void read_kernel(CacheView c, HeadRows k, HeadRows v, int64_t tokens,
                                                   const int64_t *__restrict__ slots, int64_t pieces) {
    const int nb = c.dim / 32;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < pieces;
         i += static_cast<int64_t>(gridDim.x) * 256) {
        const int piece = static_cast<int>(i % (4 * nb));
        int64_t j = i / (4 * nb);
        const int h = static_cast<int>(j % c.heads);
        j /= c.heads;
        const bool value = j >= tokens;
        const int64_t t = value ? j - tokens : j, slot = slots[t];
        uint32_t w = 0, byte = 0;
        if (slot >= 0 && slot < c.slots()) {
            const int token = static_cast<int>(slot & 15), b = piece >> 2;
            const uint8_t *g = c.data + c.group(slot >> c.page_shift, h, (slot & ((1 << c.page_shift) - 1)) >> 4);
            if (!value) {
                const int quarter = piece / nb;
                w = *reinterpret_cast<const uint32_t *>(g + (token + 16 * quarter) * 4 * nb +
                                                        (piece - quarter * nb) * 4);
                byte = g[16 * c.dim + token * nb + b];
            } else {
                const uint8_t *d = g + 8 * c.dim + (token >> 2) * 64 * nb + 4 * b + (token & 3);
#pragma unroll
                for (int n = 0; n < 4; ++n) w |= static_cast<uint32_t>(d[(4 * (piece & 3) + n) * 4 * nb]) << (8 * n);
                byte = g[16 * c.dim + c.dim / 2 + (token >> 2) * 4 * nb + 4 * b + (token & 3)];
            }
        }
        const float scale = byte == 255 ? __uint_as_float(0x7fc00000u)
                                        : __uint_as_float(byte == 0 ? 1u << 22 : byte << 23);
        const float2v p[4] = {
            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
        const HeadRows &x = value ? v : k;
        Pack<T> *dst = reinterpret_cast<Pack<T> *>(static_cast<T *>(x.p) + t * x.token_stride + h * x.head_stride +
                                                   8 * piece);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                Pack<T> o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o.w[e] = __float_as_uint(p[2 * q + (e >> 1)][e & 1] * scale);
                dst[q] = o;
            }
        } else {  // two significant bits: bf16 holds them as they are
            Pack<T> o;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o.w[e] = __float_as_uint(p[e][0] * scale) >> 16 | (__float_as_uint(p[e][1] * scale) & 0xffff0000u);
            *dst = o;
        }
    }
}

unsigned grid_of(int64_t threads) { return static_cast<unsigned>(std::min<int64_t>((threads + 255) / 256, 1 << 22)); }

}  // namespace

bool cache_write_launch(const CacheView &cache, const HeadRows &k, const HeadRows &v, bool bf16, int64_t tokens,
                        const int64_t *slots, hipStream_t stream) {
    const int64_t blocks = 2 * tokens * cache.heads * (cache.dim / 32);
    if (blocks == 0) return true;
    if (bf16)
        write_kernel<uint16_t><<<grid_of(blocks), 256, 0, stream>>>(cache, k, v, tokens, slots, blocks);
    else
        write_kernel<float><<<grid_of(blocks), 256, 0, stream>>>(cache, k, v, tokens, slots, blocks);
    return hipGetLastError() == hipSuccess;
}

bool cache_read_launch(const CacheView &cache, const HeadRows &k, const HeadRows &v, bool bf16, int64_t tokens,
                       const int64_t *slots, hipStream_t stream) {
    const int64_t pieces = 2 * tokens * cache.heads * (cache.dim / 8);
    if (pieces == 0) return true;
    if (bf16)
        read_kernel<uint16_t><<<grid_of(pieces), 256, 0, stream>>>(cache, k, v, tokens, slots, pieces);
    else
        read_kernel<float><<<grid_of(pieces), 256, 0, stream>>>(cache, k, v, tokens, slots, pieces);
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
