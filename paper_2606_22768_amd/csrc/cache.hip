// cache.hip -- tokens into and out of a paged 4-bit cache (layout: cache.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "cache.hpp"
#include "mx4_block.hpp"

namespace fgd {
namespace {

typedef float float2v __attribute__((ext_vector_type(2)));

// A thread takes 8 elements (a piece) of a token's key or value, four
// neighbouring lanes the same piece of four neighbouring tokens: loads and
// stores of the dense side are whole lines, and where the four tokens' slots
// are four of the cache that share its dwords (a prompt's are, but for its
// ends), four lanes turn their values' bytes among each other and each moves
// a dword; else a byte at a time.
//
// A block has eight fours of one head: 29 tokens, behind as many places that
// stay empty (3 at most) that a run of slots falls in fours as the cache's
// dwords do.
constexpr int kChunk = 29;

// Byte r of lane j of every four to byte j of lane r.
__device__ inline uint32_t turn(uint32_t w, int lane) {
    const uint32_t x = __shfl_xor(w, 1);
    const uint32_t a = __builtin_amdgcn_perm(x, w, lane & 1 ? 0x03070105u : 0x06020400u);
    const uint32_t y = __shfl_xor(a, 2);
    return __builtin_amdgcn_perm(y, a, lane & 2 ? 0x03020706u : 0x05040100u);
}

// Where a thread's piece is.
struct Piece {
    int64_t token, slot;
    int head, piece;
    bool value, real, held, whole;  // of a token; with a slot in the cache; its four share dwords
};

// f(pieces, lane) with the kTimes pieces of each thread.
template <int NB, typename F>
__device__ inline void for_pieces(const CacheView &c, int64_t tokens, const int64_t *__restrict__ slots,
                                  int64_t chunks, F f) {
    constexpr int kTimes = (128 * NB + 255) / 256;
    const int lane = threadIdx.x & 63;
    for (int64_t i = blockIdx.x; i < 2 * chunks * c.heads; i += gridDim.x) {
        const bool value = i >= chunks * c.heads;
        const int64_t j = i - (value ? chunks * c.heads : 0), chunk = j / c.heads, first = chunk * kChunk;
        const int before = static_cast<int>(slots[first] & 3);
        Piece p[kTimes];
#pragma unroll
        for (int u = 0; u < kTimes; ++u) {
            const int n = threadIdx.x + 256 * u, four = (n >> 2) / (4 * NB), at = 4 * four + (n & 3) - before;
            p[u].token = first + at;
            p[u].piece = (n >> 2) % (4 * NB);
            p[u].head = static_cast<int>(j - chunk * c.heads);
            p[u].value = value;
            p[u].real = four < 8 && at >= 0 && at < kChunk && p[u].token < tokens;
            p[u].slot = p[u].real ? slots[p[u].token] : -1;
        }
        f(p, lane);
    }
}

// What a piece's slot says of it; for whole waves.
__device__ inline void place(const CacheView &c, Piece &p, int lane) {
    p.held = p.slot >= 0 && p.slot < c.slots();
    const int64_t four = __shfl(static_cast<long long>(p.slot >> 2), lane & ~3);
    const bool fits = p.held && (p.slot & 3) == (lane & 3) && p.slot >> 2 == four;
    p.whole = (__ballot(fits) >> (lane & ~3) & 15) == 15;
}

// A token's group, its key's code dword or the first byte of its value's
// codes, and its scale.
template <int NB>
struct Spot {
    uint8_t *key, *value, *scale;
    __device__ Spot(const CacheView &c, const Piece &p) {
        constexpr int D = 32 * NB;
        const int token = static_cast<int>(p.slot & 15), b = p.piece >> 2, quarter = p.piece / NB;
        uint8_t *g = c.data + c.group(p.slot >> c.page_shift, p.head, (p.slot & ((1 << c.page_shift) - 1)) >> 4);
        key = g + (token + 16 * quarter) * 4 * NB + (p.piece - quarter * NB) * 4;
        value = g + 8 * D + (token >> 2) * 64 * NB + 4 * b + 16 * NB * (p.piece & 3);
        scale = g + 16 * D + (p.value ? D / 2 + (token >> 2) * 4 * NB + 4 * b + (token & 3) : token * NB + b);
    }
};

// Bound by memory, or by its latency where tokens are few: 8191 tokens of 8
// heads of 128 bf16 in 12 us (a thread per block of 32, values byte by byte:
// 19).
template <typename T, int NB>
__global__ __launch_bounds__(256) void write_kernel(CacheView c, HeadRows k, HeadRows v, int64_t tokens,
                                                    const int64_t *__restrict__ slots, int64_t chunks) {
    for_pieces<NB>(c, tokens, slots, chunks, [&](auto &pieces, int lane) {
        constexpr int kTimes = sizeof(pieces) / sizeof(Piece), kPacks = 8 * sizeof(T) / 16;
        Pack<T> raw[kTimes][kPacks];
#pragma unroll
        for (int u = 0; u < kTimes; ++u) {
            const Piece &p = pieces[u];
            const HeadRows &x = p.value ? v : k;
            const T *src = static_cast<const T *>(x.p) + p.token * x.token_stride + p.head * x.head_stride + 8 * p.piece;
#pragma unroll
            for (int i = 0; i < kPacks; ++i) {
                raw[u][i] = {};
                if (p.real) raw[u][i] = reinterpret_cast<const Pack<T> *>(src)[i];
            }
        }
#pragma unroll
        for (int u = 0; u < kTimes; ++u) {
            Piece &p = pieces[u];
            place(c, p, lane);
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (sizeof(T) == 4) {
                    e[j] = __uint_as_float(raw[u][j / 4 % kPacks].w[j & 3]);
                } else {
                    const uint32_t w = raw[u][0].w[j >> 1];
                    e[j] = __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
                }
            }
            // The largest magnitude of the block's four pieces, 4 lanes apart.
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(e[i]) & 0x7fffffffu);
            top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 4)));
            top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 8)));
            uint32_t byte;
            const uint32_t w = encode_eight(e, top, byte), turned = turn(w, lane);
            if (!p.held) continue;
            const Spot<NB> at(c, p);
            if (!p.value) {
                *reinterpret_cast<uint32_t *>(at.key) = w;
            } else if (p.whole) {
                *reinterpret_cast<uint32_t *>(at.value + (lane & 3) * 4 * NB) = turned;
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n) at.value[n * 4 * NB + (p.slot & 3)] = static_cast<uint8_t>(w >> (8 * n));
            }
            if ((p.piece & 3) == 0) *at.scale = static_cast<uint8_t>(byte);
        }
    });
}

// The same: 14 us (values byte by byte: 16).
template <typename T, int NB>
__global__ __launch_bounds__(256) void read_kernel(CacheView c, HeadRows k, HeadRows v, int64_t tokens,
                                                   const int64_t *__restrict__ slots, int64_t chunks) {
    for_pieces<NB>(c, tokens, slots, chunks, [&](auto &pieces, int lane) {
        constexpr int kTimes = sizeof(pieces) / sizeof(Piece);
        uint32_t codes[kTimes], scales[kTimes];
#pragma unroll
        for (int u = 0; u < kTimes; ++u) {
            Piece &p = pieces[u];
            place(c, p, lane);
            codes[u] = scales[u] = 0;
            if (!p.held) continue;
            const Spot<NB> at(c, p);
            if (!p.value) {
                codes[u] = *reinterpret_cast<const uint32_t *>(at.key);
            } else if (p.whole) {
                codes[u] = *reinterpret_cast<const uint32_t *>(at.value + (lane & 3) * 4 * NB);
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    codes[u] |= static_cast<uint32_t>(at.value[n * 4 * NB + (p.slot & 3)]) << (8 * n);
            }
            scales[u] = *at.scale;
        }
#pragma unroll
        for (int u = 0; u < kTimes; ++u) {
            const Piece &p = pieces[u];
            uint32_t w = codes[u];
            const uint32_t byte = scales[u], turned = turn(w, lane);
            if (p.value && p.whole) w = turned;
            if (!p.real) continue;
            const float scale = byte == 255 ? __uint_as_float(0x7fc00000u)
                                            : __uint_as_float(byte == 0 ? 1u << 22 : byte << 23);
            const float2v e[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0),
                                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2),
                                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
            const HeadRows &x = p.value ? v : k;
            Pack<T> *dst = reinterpret_cast<Pack<T> *>(static_cast<T *>(x.p) + p.token * x.token_stride +
                                                       p.head * x.head_stride + 8 * p.piece);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    Pack<T> o;
#pragma unroll
                    for (int i = 0; i < 4; ++i) o.w[i] = __float_as_uint(e[2 * q + (i >> 1)][i & 1] * scale);
                    dst[q] = o;
                }
            } else {  // two significant bits: bf16 holds them as they are
                Pack<T> o;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o.w[i] = __float_as_uint(e[i][0] * scale) >> 16 | (__float_as_uint(e[i][1] * scale) & 0xffff0000u);
                *dst = o;
            }
        }
    });
}

// launch(blocks count) of the kernel for the cache's heads.
template <typename F>
bool for_blocks(const CacheView &cache, int64_t tokens, F launch) {
    if (tokens == 0) return true;
    const int64_t chunks = (tokens + kChunk - 1) / kChunk;
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(2 * chunks * cache.heads, 1 << 22));
    switch (cache.dim / 32) {
        case 1: launch(std::integral_constant<int, 1>(), grid, chunks); break;
        case 2: launch(std::integral_constant<int, 2>(), grid, chunks); break;
        case 3: launch(std::integral_constant<int, 3>(), grid, chunks); break;
        case 4: launch(std::integral_constant<int, 4>(), grid, chunks); break;
        case 5: launch(std::integral_constant<int, 5>(), grid, chunks); break;
        case 6: launch(std::integral_constant<int, 6>(), grid, chunks); break;
        case 7: launch(std::integral_constant<int, 7>(), grid, chunks); break;
        default: launch(std::integral_constant<int, 8>(), grid, chunks); break;
    }
    return hipGetLastError() == hipSuccess;
}

}  // namespace

bool cache_write_launch(const CacheView &cache, const HeadRows &k, const HeadRows &v, bool bf16, int64_t tokens,
                        const int64_t *slots, hipStream_t stream) {
    return for_blocks(cache, tokens, [&](auto nb, unsigned grid, int64_t chunks) {
        if (bf16)
            write_kernel<uint16_t, nb.value><<<grid, 256, 0, stream>>>(cache, k, v, tokens, slots, chunks);
        else
            write_kernel<float, nb.value><<<grid, 256, 0, stream>>>(cache, k, v, tokens, slots, chunks);
    });
}

bool cache_read_launch(const CacheView &cache, const HeadRows &k, const HeadRows &v, bool bf16, int64_t tokens,
                       const int64_t *slots, hipStream_t stream) {
    return for_blocks(cache, tokens, [&](auto nb, unsigned grid, int64_t chunks) {
        if (bf16)
            read_kernel<uint16_t, nb.value><<<grid, 256, 0, stream>>>(cache, k, v, tokens, slots, chunks);
        else
            read_kernel<float, nb.value><<<grid, 256, 0, stream>>>(cache, k, v, tokens, slots, chunks);
    });
}

}  // namespace fgd
