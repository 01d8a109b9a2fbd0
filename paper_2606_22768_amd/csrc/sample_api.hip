// sample_api.hip -- the C ABI of sampling: argument checks and the launch of
// the kernels in sample.hip.  No engine is involved; the call runs on the
// caller's current device.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "../../include/fgd.h"
#include "api.hpp"
#include "sample.hpp"

namespace {

using fgd::api_fail;

bool misaligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

bool ranges_overlap(const void *a, int64_t na, const void *b, int64_t nb) {
    if (!a || !b || na <= 0 || nb <= 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + static_cast<uint64_t>(nb) && b0 < a0 + static_cast<uint64_t>(na);
}

fgd_status check_sizes(int32_t dtype, int64_t num_rows, int64_t vocab) {
    if (dtype != FGD_F32 && dtype != FGD_BF16) return api_fail(FGD_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (num_rows < 0 || num_rows > INT32_MAX)
        return api_fail(FGD_ERR_INVALID_ARG, "num_rows must be in [0, 2^31)");
    if (vocab < 1 || vocab > FGD_MAX_SAMPLE_VOCAB)
        return api_fail(FGD_ERR_INVALID_ARG, "vocab %lld is outside [1, %d]", static_cast<long long>(vocab),
                        FGD_MAX_SAMPLE_VOCAB);
    return FGD_OK;
}

}  // namespace

extern "C" {

fgd_status fgd_sample_workspace_size(int32_t dtype, int64_t num_rows, int64_t vocab, int64_t *bytes) {
    fgd::api_clear();
    if (!bytes) return api_fail(FGD_ERR_INVALID_ARG, "NULL bytes");
    if (fgd_status st = check_sizes(dtype, num_rows, vocab)) return st;
    *bytes = fgd::sample_workspace_bytes(dtype == FGD_BF16, num_rows, static_cast<int32_t>(vocab));
    return FGD_OK;
}

fgd_status fgd_sample(const void *logits, int32_t dtype, int64_t num_rows, int64_t vocab, int64_t ldk,
                      const float *uniform, const fgd_sampling *settings, int32_t *tokens_out, float *probs_out,
                      void *workspace, int64_t workspace_bytes, void *stream) {
    fgd::api_clear();
    if (fgd_status st = check_sizes(dtype, num_rows, vocab)) return st;
    const int64_t es = dtype == FGD_BF16 ? 2 : 4;
    if (!settings || settings->struct_size != sizeof(fgd_sampling))
        return api_fail(FGD_ERR_INVALID_ARG, "settings: NULL or of another size");
    if (settings->reserved != 0) return api_fail(FGD_ERR_INVALID_ARG, "settings: reserved must be 0");
    if (ldk < vocab || ldk > (INT64_C(1) << 40)) return api_fail(FGD_ERR_INVALID_ARG, "need vocab <= ldk <= 2^40");
    if (num_rows == 0) return FGD_OK;
    if (!logits || !uniform || !tokens_out) return api_fail(FGD_ERR_INVALID_ARG, "NULL array");
    if (misaligned(logits, es) || misaligned(uniform, 4) || misaligned(tokens_out, 4) || misaligned(probs_out, 4) ||
        misaligned(settings->temperature_rows, 4) || misaligned(settings->top_k_rows, 4) ||
        misaligned(settings->top_p_rows, 4) || misaligned(settings->min_p_rows, 4) || misaligned(workspace, 16))
        return api_fail(FGD_ERR_INVALID_ARG,
                        "arrays must be aligned to their element size and the workspace to 16 bytes");
    const __int128 span = (static_cast<__int128>(num_rows - 1) * ldk + vocab) * es;
    if (span > (INT64_C(1) << 60)) return api_fail(FGD_ERR_INVALID_ARG, "logits: sizes are too large");
    int64_t need = 0;
    if (fgd_status st = fgd_sample_workspace_size(dtype, num_rows, vocab, &need)) return st;
    if (workspace_bytes < need || (need > 0 && !workspace))
        return api_fail(FGD_ERR_INVALID_ARG, "workspace of %lld bytes is below the %lld this call needs",
                        static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    const struct {
        const void *p;
        int64_t n;
    } in[] = {{logits, static_cast<int64_t>(span)},       {uniform, num_rows * 4},
              {settings->temperature_rows, num_rows * 4}, {settings->top_k_rows, num_rows * 4},
              {settings->top_p_rows, num_rows * 4},       {settings->min_p_rows, num_rows * 4}},
      out[] = {{tokens_out, num_rows * 4}, {probs_out, num_rows * 4}, {workspace, need}};
    for (int i = 0; i < 3; ++i) {
        for (const auto &a : in)
            if (ranges_overlap(out[i].p, out[i].n, a.p, a.n))
                return api_fail(FGD_ERR_INVALID_ARG, "outputs and the workspace must not overlap the inputs");
        for (int j = 0; j < i; ++j)
            if (ranges_overlap(out[i].p, out[i].n, out[j].p, out[j].n))
                return api_fail(FGD_ERR_INVALID_ARG, "outputs and the workspace must not overlap each other");
    }
    const fgd::SampleSettings s = {settings->temperature_rows, settings->top_p_rows, settings->min_p_rows,
                                   settings->top_k_rows,       settings->temperature, settings->top_p,
                                   settings->min_p,            settings->top_k};
    if (!fgd::sample_launch(logits, dtype == FGD_BF16, num_rows, static_cast<int32_t>(vocab), ldk, uniform, s,
                            tokens_out, probs_out, workspace, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "sampling launch failed");
    return FGD_OK;
}

}  // extern "C"
