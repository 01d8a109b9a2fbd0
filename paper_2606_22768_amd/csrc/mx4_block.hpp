// mx4_block.hpp -- one block of the 4-bit format (mx4.hpp) in a thread.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fgd {
namespace {

template <typename T>
__device__ inline float widen(T v);
template <>
__device__ inline float widen<float>(float v) { return v; }
template <>
__device__ inline float widen<uint16_t>(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }

// A widened value back in its type.
template <typename T>
__device__ inline T narrow(float v);
template <>
__device__ inline float narrow<float>(float v) { return v; }
template <>
__device__ inline uint16_t narrow<uint16_t>(float v) { return static_cast<uint16_t>(__float_as_uint(v) >> 16); }

// Sixteen bytes of elements at an address aligned to its element only.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    uint32_t w[4];
};

// `valid` (32 at most) values from src, zeros behind them.
template <typename T>
__device__ inline void load_block(const T *src, int64_t valid, float (&v)[32]) {
    constexpr int kPer = 16 / sizeof(T);
    if (valid >= 32) {
#pragma unroll
        for (int i = 0; i < 32 / kPer; ++i) {
            const Pack<T> u = reinterpret_cast<const Pack<T> *>(src)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) {
                    v[4 * i + j] = __uint_as_float(u.w[j]);
                } else {
                    v[8 * i + 2 * j] = __uint_as_float(u.w[j] << 16);
                    v[8 * i + 2 * j + 1] = __uint_as_float(u.w[j] & 0xffff0000u);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = i < valid ? widen(src[i]) : 0.0f;
    }
}

// Eight values of a block whose largest magnitude has the bits `top` to their
// four code bytes, and the block's scale byte.
__device__ inline uint32_t encode_eight(const float (&v)[8], uint32_t top, uint32_t &byte) {
    const uint32_t field = top >> 23;
    if (field == 255) {
        byte = 255;
        return 0;
    }
    byte = field > 2 ? field - 2 : 0;
    const float lift = byte == 0 ? 0x1p64f : 1.0f;  // as in encode_block
    const float scale = __uint_as_float((byte == 0 ? 64u : byte) << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0] * lift, v[1] * lift, scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2] * lift, v[3] * lift, scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4] * lift, v[5] * lift, scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6] * lift, v[7] * lift, scale, 3);
    return r;
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

}  // namespace
}  // namespace fgd
