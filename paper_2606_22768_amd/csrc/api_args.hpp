// api_args.hpp -- argument checks that the C ABI's operators share.
#pragma once

#include <stdint.h>

#include "api.hpp"

namespace fgd {

typedef __int128 wide;

constexpr wide kMostBytes = static_cast<wide>(1) << 60;  // largest element or byte count of one array

inline bool api_aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline int api_elem_size(int32_t dtype) { return dtype == FGD_BF16 ? 2 : 4; }

inline bool api_overlap(const void *a, int64_t na, const void *b, int64_t nb) {
    if (!a || !b || na <= 0 || nb <= 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + static_cast<uint64_t>(nb) && b0 < a0 + static_cast<uint64_t>(na);
}

inline fgd_status api_check_dtype(int32_t dtype) {
    if (dtype != FGD_F32 && dtype != FGD_BF16) return api_fail(FGD_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    return FGD_OK;
}

// An array of n values of `size` bytes.
inline fgd_status api_check_array(const char *what, const void *p, int64_t n, int size) {
    if (n <= 0) return FGD_OK;
    if (!p) return api_fail(FGD_ERR_INVALID_ARG, "%s: NULL array", what);
    if (!api_aligned(p, size))
        return api_fail(FGD_ERR_INVALID_ARG, "%s must be aligned to its element size", what);
    return FGD_OK;
}

// An array batch x tokens x heads x dim with element strides of the first
// three (heads of contiguous elements): aligned to its element, no stride
// negative; *bytes is the span from the first to the last element.  An
// output's elements must not overlap each other (`output`).
inline fgd_status api_check_heads(const char *what, const void *p, int32_t dtype, int64_t batch, int64_t tokens,
                                  int64_t heads, int64_t dim, int64_t batch_stride, int64_t token_stride,
                                  int64_t head_stride, bool output, int64_t *bytes) {
    *bytes = 0;
    if (batch == 0 || tokens == 0 || heads == 0 || dim == 0) return FGD_OK;
    if (!p) return api_fail(FGD_ERR_INVALID_ARG, "%s: NULL array", what);
    if (!api_aligned(p, api_elem_size(dtype)))
        return api_fail(FGD_ERR_INVALID_ARG, "%s must be aligned to its element size", what);
    if (batch_stride < 0 || token_stride < 0 || head_stride < 0)
        return api_fail(FGD_ERR_INVALID_ARG, "%s: negative stride", what);
    const wide last = static_cast<wide>(batch - 1) * batch_stride + static_cast<wide>(tokens - 1) * token_stride +
                      static_cast<wide>(heads - 1) * head_stride + (dim - 1);
    if (last >= kMostBytes / 4) return api_fail(FGD_ERR_INVALID_ARG, "%s: strides are too large", what);
    *bytes = (static_cast<int64_t>(last) + 1) * api_elem_size(dtype);
    if (!output) return FGD_OK;
    // In the order of their strides each axis steps over all of those below.
    struct {
        int64_t stride, n;
    } axes[3] = {{batch_stride, batch}, {token_stride, tokens}, {head_stride, heads}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            if (axes[j].stride > axes[j + 1].stride || (axes[j].stride == axes[j + 1].stride && axes[j].n > axes[j + 1].n)) {
                const auto t = axes[j];
                axes[j] = axes[j + 1];
                axes[j + 1] = t;
            }
    wide span = dim;
    for (const auto &x : axes) {
        if (x.n <= 1) continue;
        if (x.stride < span) return api_fail(FGD_ERR_INVALID_ARG, "%s: its elements overlap", what);
        span += static_cast<wide>(x.n - 1) * x.stride;
    }
    return FGD_OK;
}

}  // namespace fgd
