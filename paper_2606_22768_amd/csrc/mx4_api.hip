// mx4_api.hip -- the C ABI of the 4-bit operators: argument checks and
// launches of the kernels in mx4.hip and mx4_gemm.hip.  No engine is
// involved; the calls run on the caller's current device.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "../../include/fgd.h"
#include "api.hpp"
#include "mx4.hpp"

namespace {

using fgd::api_fail;
typedef __int128 wide;

constexpr wide kMost = static_cast<wide>(1) << 60;  // largest element or byte count of one array

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int elem_size(int32_t dtype) { return dtype == FGD_BF16 ? 2 : 4; }

bool ranges_overlap(const void *a, int64_t na, const void *b, int64_t nb) {
    if (!a || !b || na <= 0 || nb <= 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + static_cast<uint64_t>(nb) && b0 < a0 + static_cast<uint64_t>(na);
}

fgd_status check_dtype(int32_t dtype) {
    if (dtype != FGD_F32 && dtype != FGD_BF16) return api_fail(FGD_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    return FGD_OK;
}

// Sizes of a matrix in the 4-bit format; its padded size stays far below 2^63.
fgd_status check_matrix(const char *what, int32_t batch, int64_t rows, int64_t cols) {
    if (batch < 0 || rows < 0 || cols < 0) return api_fail(FGD_ERR_INVALID_ARG, "%s: negative size", what);
    if (static_cast<wide>(batch) * (static_cast<wide>(rows) + 63) * (static_cast<wide>(cols) + 127) > kMost)
        return api_fail(FGD_ERR_INVALID_ARG, "%s: sizes are too large", what);
    return FGD_OK;
}

// A dense array seen as batch x rows x cols with element strides: every
// stride non-negative, the last element's offset in range; *bytes is the
// span from the first to the last element.
fgd_status check_strided(const char *what, const void *p, int32_t dtype, int32_t batch, int64_t rows, int64_t cols,
                         int64_t batch_stride, int64_t row_stride, int64_t col_stride, int64_t *bytes) {
    *bytes = 0;
    if (batch == 0 || rows == 0 || cols == 0) return FGD_OK;
    if (!p) return api_fail(FGD_ERR_INVALID_ARG, "%s: NULL array", what);
    if (!aligned(p, elem_size(dtype)))
        return api_fail(FGD_ERR_INVALID_ARG, "%s must be aligned to its element size", what);
    if (batch_stride < 0 || row_stride < 0 || col_stride < 0)
        return api_fail(FGD_ERR_INVALID_ARG, "%s: negative stride", what);
    const wide last = static_cast<wide>(batch - 1) * batch_stride + static_cast<wide>(rows - 1) * row_stride +
                      static_cast<wide>(cols - 1) * col_stride;
    if (last >= kMost) return api_fail(FGD_ERR_INVALID_ARG, "%s: strides are too large", what);
    *bytes = (static_cast<int64_t>(last) + 1) * elem_size(dtype);
    return FGD_OK;
}

// An output: rows of contiguous elements, no two of which may overlap.
fgd_status check_output(const char *what, const void *p, int32_t dtype, int32_t batch, int64_t rows, int64_t cols,
                        int64_t batch_stride, int64_t row_stride, int64_t *bytes) {
    if (fgd_status st = check_strided(what, p, dtype, batch, rows, cols, batch_stride, row_stride, 1, bytes))
        return st;
    if (rows > 1 && row_stride < cols)
        return api_fail(FGD_ERR_INVALID_ARG, "%s: row_stride is below the row length", what);
    if (batch > 1 && rows > 0 && static_cast<wide>(batch_stride) < static_cast<wide>(rows - 1) * row_stride + cols)
        return api_fail(FGD_ERR_INVALID_ARG, "%s: batch_stride is below one matrix", what);
    return FGD_OK;
}

struct Spans {  // of a matrix in the 4-bit format
    int64_t codes, scales;
};

fgd_status check_packed(const char *what, const void *codes, const void *scales, int32_t batch, int64_t rows,
                        int64_t cols, Spans *s) {
    if (fgd_status st = check_matrix(what, batch, rows, cols)) return st;
    const int64_t tiles = fgd::mx4_tiles(batch, rows, cols);
    s->codes = tiles * fgd::kMx4CodeBytes;
    s->scales = tiles * fgd::kMx4ScaleBytes;
    if (tiles == 0) return FGD_OK;
    if (!codes || !scales) return api_fail(FGD_ERR_INVALID_ARG, "%s: NULL array", what);
    if (!aligned(codes, 16) || !aligned(scales, 16))
        return api_fail(FGD_ERR_INVALID_ARG, "%s: codes and scales must be 16-byte aligned", what);
    return FGD_OK;
}

fgd_status check_quantize_input(const char *what, const void *x, int32_t dtype, int32_t batch, int64_t rows,
                                int64_t cols, int64_t batch_stride, int64_t row_stride, int64_t col_stride,
                                int64_t *bytes) {
    if (fgd_status st = check_dtype(dtype)) return st;
    if (fgd_status st = check_matrix(what, batch, rows, cols)) return st;
    if (fgd_status st =
            check_strided(what, x, dtype, batch, rows, cols, batch_stride, row_stride, col_stride, bytes))
        return st;
    if (batch > 0 && rows > 0 && cols > 0 && row_stride != 1 && col_stride != 1)
        return api_fail(FGD_ERR_INVALID_ARG, "%s: its rows or its columns must be contiguous", what);
    return FGD_OK;
}

// The product's sizes and output, shared by the product and the layer.
fgd_status check_product(const void *w_codes, const void *w_scales, int32_t batch, int64_t m, int64_t n, int64_t k,
                         const void *out, int32_t out_dtype, int64_t out_batch_stride, int64_t out_row_stride,
                         Spans *w, int64_t *out_bytes) {
    if (fgd_status st = check_dtype(out_dtype)) return st;
    if (fgd_status st = check_packed("weights", w_codes, w_scales, batch, n, k, w)) return st;
    if (m < 0) return api_fail(FGD_ERR_INVALID_ARG, "negative size");
    if (static_cast<wide>(batch) * (m + 255) * (static_cast<wide>(n) + 255) > kMost)
        return api_fail(FGD_ERR_INVALID_ARG, "output: sizes are too large");
    if (fgd_status st =
            check_output("output", out, out_dtype, batch, m, n, out_batch_stride, out_row_stride, out_bytes))
        return st;
    if (ranges_overlap(out, *out_bytes, w_codes, w->codes) || ranges_overlap(out, *out_bytes, w_scales, w->scales))
        return api_fail(FGD_ERR_INVALID_ARG, "the output must not overlap the weights");
    return FGD_OK;
}

}  // namespace

extern "C" {

fgd_status fgd_mx4_size(int32_t batch, int64_t rows, int64_t cols, int64_t *code_bytes, int64_t *scale_bytes) {
    fgd::api_clear();
    if (!code_bytes || !scale_bytes) return api_fail(FGD_ERR_INVALID_ARG, "NULL size");
    if (fgd_status st = check_matrix("matrix", batch, rows, cols)) return st;
    const int64_t tiles = fgd::mx4_tiles(batch, rows, cols);
    *code_bytes = tiles * fgd::kMx4CodeBytes;
    *scale_bytes = tiles * fgd::kMx4ScaleBytes;
    return FGD_OK;
}

fgd_status fgd_mx4_quantize(const void *x, int32_t dtype, int32_t batch, int64_t rows, int64_t cols,
                            int64_t batch_stride, int64_t row_stride, int64_t col_stride, void *codes, void *scales,
                            void *stream) {
    fgd::api_clear();
    int64_t x_bytes;
    Spans q;
    if (fgd_status st = check_quantize_input("x", x, dtype, batch, rows, cols, batch_stride, row_stride, col_stride,
                                             &x_bytes))
        return st;
    if (fgd_status st = check_packed("quantised matrix", codes, scales, batch, rows, cols, &q)) return st;
    if (ranges_overlap(codes, q.codes, x, x_bytes) || ranges_overlap(scales, q.scales, x, x_bytes) ||
        ranges_overlap(codes, q.codes, scales, q.scales))
        return api_fail(FGD_ERR_INVALID_ARG, "x, codes and scales must not overlap");
    if (!fgd::mx4_quantize_launch(x, dtype == FGD_BF16, batch, rows, cols, batch_stride, row_stride, col_stride,
                                  codes, scales, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "4-bit quantisation launch failed");
    return FGD_OK;
}

fgd_status fgd_mx4_quantize_both(const void *x, int32_t dtype, int32_t batch, int64_t rows, int64_t cols,
                                 int64_t batch_stride, int64_t row_stride, void *codes, void *scales, void *t_codes,
                                 void *t_scales, void *stream) {
    fgd::api_clear();
    int64_t x_bytes;
    Spans q, t;
    if (fgd_status st = check_quantize_input("x", x, dtype, batch, rows, cols, batch_stride, row_stride, 1, &x_bytes))
        return st;
    if (fgd_status st = check_packed("quantised matrix", codes, scales, batch, rows, cols, &q)) return st;
    if (fgd_status st = check_packed("quantised transpose", t_codes, t_scales, batch, cols, rows, &t)) return st;
    const struct {
        const void *p;
        int64_t bytes;
    } arrays[] = {{x, x_bytes}, {codes, q.codes}, {scales, q.scales}, {t_codes, t.codes}, {t_scales, t.scales}};
    for (int i = 0; i < 5; ++i)
        for (int j = i + 1; j < 5; ++j)
            if (ranges_overlap(arrays[i].p, arrays[i].bytes, arrays[j].p, arrays[j].bytes))
                return api_fail(FGD_ERR_INVALID_ARG, "x, codes and scales must not overlap");
    if (!fgd::mx4_quantize_both_launch(x, dtype == FGD_BF16, batch, rows, cols, batch_stride, row_stride, codes,
                                       scales, t_codes, t_scales, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "4-bit quantisation launch failed");
    return FGD_OK;
}

fgd_status fgd_mx4_dequantize(const void *codes, const void *scales, int32_t batch, int64_t rows, int64_t cols,
                              void *out, int32_t dtype, int64_t batch_stride, int64_t row_stride, void *stream) {
    fgd::api_clear();
    int64_t out_bytes;
    Spans q;
    if (fgd_status st = check_dtype(dtype)) return st;
    if (fgd_status st = check_packed("quantised matrix", codes, scales, batch, rows, cols, &q)) return st;
    if (fgd_status st = check_output("output", out, dtype, batch, rows, cols, batch_stride, row_stride, &out_bytes))
        return st;
    if (ranges_overlap(codes, q.codes, out, out_bytes) || ranges_overlap(scales, q.scales, out, out_bytes))
        return api_fail(FGD_ERR_INVALID_ARG, "the output must not overlap codes or scales");
    if (!fgd::mx4_dequantize_launch(codes, scales, batch, rows, cols, out, dtype == FGD_BF16, batch_stride,
                                    row_stride, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "4-bit read-back launch failed");
    return FGD_OK;
}

fgd_status fgd_mx4_matmul(const void *a_codes, const void *a_scales, const void *w_codes, const void *w_scales,
                          int32_t batch, int64_t m, int64_t n, int64_t k, void *out, int32_t out_dtype,
                          int64_t out_batch_stride, int64_t out_row_stride, void *stream) {
    fgd::api_clear();
    int64_t out_bytes;
    Spans a, w;
    if (fgd_status st = check_packed("left operand", a_codes, a_scales, batch, m, k, &a)) return st;
    if (fgd_status st = check_product(w_codes, w_scales, batch, m, n, k, out, out_dtype, out_batch_stride,
                                      out_row_stride, &w, &out_bytes))
        return st;
    if (ranges_overlap(out, out_bytes, a_codes, a.codes) || ranges_overlap(out, out_bytes, a_scales, a.scales))
        return api_fail(FGD_ERR_INVALID_ARG, "the output must not overlap the operands");
    if (!fgd::mx4_matmul_launch(a_codes, a_scales, w_codes, w_scales, batch, m, n, k, out, out_dtype == FGD_BF16,
                                out_batch_stride, out_row_stride, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "4-bit product launch failed");
    return FGD_OK;
}

fgd_status fgd_mx4_linear_workspace_size(int32_t batch, int64_t tokens, int64_t k, int64_t *bytes) {
    fgd::api_clear();
    if (!bytes) return api_fail(FGD_ERR_INVALID_ARG, "NULL bytes");
    if (fgd_status st = check_matrix("x", batch, tokens, k)) return st;
    *bytes = fgd::mx4_tiles(batch, tokens, k) * (fgd::kMx4CodeBytes + fgd::kMx4ScaleBytes);
    return FGD_OK;
}

fgd_status fgd_mx4_linear(const void *x, int32_t x_dtype, int64_t x_batch_stride, int64_t x_row_stride,
                          const void *w_codes, const void *w_scales, int32_t batch, int64_t tokens, int64_t n,
                          int64_t k, void *out, int32_t out_dtype, int64_t out_batch_stride, int64_t out_row_stride,
                          void *workspace, int64_t workspace_bytes, void *stream) {
    fgd::api_clear();
    int64_t x_bytes, out_bytes;
    Spans a, w;
    if (fgd_status st =
            check_quantize_input("x", x, x_dtype, batch, tokens, k, x_batch_stride, x_row_stride, 1, &x_bytes))
        return st;
    if (fgd_status st = check_product(w_codes, w_scales, batch, tokens, n, k, out, out_dtype, out_batch_stride,
                                      out_row_stride, &w, &out_bytes))
        return st;
    const int64_t tiles = fgd::mx4_tiles(batch, tokens, k);
    a.codes = tiles * fgd::kMx4CodeBytes;
    const int64_t need = a.codes + tiles * fgd::kMx4ScaleBytes;
    if (need > 0 && !workspace) return api_fail(FGD_ERR_INVALID_ARG, "NULL workspace");
    if (!aligned(workspace, 16)) return api_fail(FGD_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
    if (workspace_bytes < need)
        return api_fail(FGD_ERR_INVALID_ARG, "workspace of %lld bytes is below the %lld this call needs",
                        static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    if (ranges_overlap(out, out_bytes, x, x_bytes) || ranges_overlap(out, out_bytes, workspace, need) ||
        ranges_overlap(workspace, need, x, x_bytes) || ranges_overlap(workspace, need, w_codes, w.codes) ||
        ranges_overlap(workspace, need, w_scales, w.scales))
        return api_fail(FGD_ERR_INVALID_ARG, "x, the weights, the output and the workspace must not overlap");
    if (fgd::mx4_linear_fuses(batch, tokens, n, k)) {
        if (!fgd::mx4_linear_launch(x, x_dtype == FGD_BF16, x_batch_stride, x_row_stride, w_codes, w_scales, batch,
                                    tokens, n, k, out, out_dtype == FGD_BF16, out_batch_stride, out_row_stride,
                                    static_cast<hipStream_t>(stream)))
            return api_fail(FGD_ERR_HIP, "4-bit layer launch failed");
        return FGD_OK;
    }
    uint8_t *codes = static_cast<uint8_t *>(workspace), *scales = codes + a.codes;
    if (!fgd::mx4_quantize_launch(x, x_dtype == FGD_BF16, batch, tokens, k, x_batch_stride, x_row_stride, 1, codes,
                                  scales, static_cast<hipStream_t>(stream)) ||
        !fgd::mx4_matmul_launch(codes, scales, w_codes, w_scales, batch, tokens, n, k, out, out_dtype == FGD_BF16,
                                out_batch_stride, out_row_stride, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "4-bit layer launch failed");
    return FGD_OK;
}

fgd_status fgd_mx4_linear_grads_workspace_size(int32_t batch, int64_t tokens, int64_t n, int64_t k, int64_t *bytes) {
    fgd::api_clear();
    if (!bytes) return api_fail(FGD_ERR_INVALID_ARG, "NULL bytes");
    if (fgd_status st = check_matrix("dy", batch, tokens, n)) return st;
    if (fgd_status st = check_matrix("dy", batch, n, tokens)) return st;
    if (fgd_status st = check_matrix("x", batch, k, tokens)) return st;
    *bytes = (fgd::mx4_tiles(batch, tokens, n) + fgd::mx4_tiles(batch, n, tokens) + fgd::mx4_tiles(batch, k, tokens)) *
             (fgd::kMx4CodeBytes + fgd::kMx4ScaleBytes);
    return FGD_OK;
}

fgd_status fgd_mx4_linear_grads(const void *dy, int32_t dy_dtype, int64_t dy_batch_stride, int64_t dy_row_stride,
                                const void *x, int32_t x_dtype, int64_t x_batch_stride, int64_t x_row_stride,
                                const void *wt_codes, const void *wt_scales, int32_t batch, int64_t tokens, int64_t n,
                                int64_t k, void *dx, int32_t dx_dtype, int64_t dx_batch_stride, int64_t dx_row_stride,
                                void *dw, int32_t dw_dtype, int64_t dw_batch_stride, int64_t dw_row_stride,
                                void *workspace, int64_t workspace_bytes, void *stream) {
    fgd::api_clear();
    int64_t dy_bytes, x_bytes, dx_bytes, dw_bytes, need;
    Spans w;
    if (fgd_status st =
            check_quantize_input("dy", dy, dy_dtype, batch, tokens, n, dy_batch_stride, dy_row_stride, 1, &dy_bytes))
        return st;
    if (fgd_status st =
            check_quantize_input("x", x, x_dtype, batch, tokens, k, x_batch_stride, x_row_stride, 1, &x_bytes))
        return st;
    if (fgd_status st = fgd_mx4_linear_grads_workspace_size(batch, tokens, n, k, &need)) return st;
    if (fgd_status st = check_product(wt_codes, wt_scales, batch, tokens, k, n, dx, dx_dtype, dx_batch_stride,
                                      dx_row_stride, &w, &dx_bytes))
        return st;
    if (fgd_status st = check_dtype(dw_dtype)) return st;
    if (static_cast<wide>(batch) * (static_cast<wide>(n) + 255) * (static_cast<wide>(k) + 255) > kMost)
        return api_fail(FGD_ERR_INVALID_ARG, "dw: sizes are too large");
    if (fgd_status st = check_output("dw", dw, dw_dtype, batch, n, k, dw_batch_stride, dw_row_stride, &dw_bytes))
        return st;
    if (need > 0 && !workspace) return api_fail(FGD_ERR_INVALID_ARG, "NULL workspace");
    if (!aligned(workspace, 16)) return api_fail(FGD_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
    if (workspace_bytes < need)
        return api_fail(FGD_ERR_INVALID_ARG, "workspace of %lld bytes is below the %lld this call needs",
                        static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    // What is written, then what is read.
    const struct {
        const void *p;
        int64_t bytes;
    } arrays[] = {{dx, dx_bytes}, {dw, dw_bytes},          {workspace, need},     {dy, dy_bytes},
                  {x, x_bytes},   {wt_codes, w.codes}, {wt_scales, w.scales}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 7; ++j)
            if (ranges_overlap(arrays[i].p, arrays[i].bytes, arrays[j].p, arrays[j].bytes))
                return api_fail(FGD_ERR_INVALID_ARG,
                                "the gradients and the workspace must overlap neither each other nor an input");
    const int64_t dy_tiles = fgd::mx4_tiles(batch, tokens, n), dyt_tiles = fgd::mx4_tiles(batch, n, tokens),
                  xt_tiles = fgd::mx4_tiles(batch, k, tokens);
    uint8_t *dy_codes = static_cast<uint8_t *>(workspace), *dyt_codes = dy_codes + dy_tiles * fgd::kMx4CodeBytes,
            *xt_codes = dyt_codes + dyt_tiles * fgd::kMx4CodeBytes,
            *dy_scales = xt_codes + xt_tiles * fgd::kMx4CodeBytes,
            *dyt_scales = dy_scales + dy_tiles * fgd::kMx4ScaleBytes,
            *xt_scales = dyt_scales + dyt_tiles * fgd::kMx4ScaleBytes;
    const hipStream_t on = static_cast<hipStream_t>(stream);
    if (!fgd::mx4_quantize_launch(x, x_dtype == FGD_BF16, batch, k, tokens, x_batch_stride, 1, x_row_stride, xt_codes,
                                  xt_scales, on) ||
        !fgd::mx4_quantize_both_launch(dy, dy_dtype == FGD_BF16, batch, tokens, n, dy_batch_stride, dy_row_stride,
                                       dy_codes, dy_scales, dyt_codes, dyt_scales, on) ||
        !fgd::mx4_matmul_launch(dy_codes, dy_scales, wt_codes, wt_scales, batch, tokens, k, n, dx,
                                dx_dtype == FGD_BF16, dx_batch_stride, dx_row_stride, on) ||
        !fgd::mx4_matmul_launch(dyt_codes, dyt_scales, xt_codes, xt_scales, batch, n, k, tokens, dw,
                                dw_dtype == FGD_BF16, dw_batch_stride, dw_row_stride, on))
        return api_fail(FGD_ERR_HIP, "4-bit gradients' launch failed");
    return FGD_OK;
}

}  // extern "C"
