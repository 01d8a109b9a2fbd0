// sample.hpp -- launcher of the sampling kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fgd {

// The settings of a call: each array holds one value per row, or is NULL and
// the scalar beside it holds for every row.
struct SampleSettings {
    const float *temperature_rows, *top_p_rows, *min_p_rows;
    const int32_t *top_k_rows;
    float temperature, top_p, min_p;
    int32_t top_k;
};

// Device workspace of a call.
int64_t sample_workspace_bytes(bool bf16, int64_t rows, int32_t vocab);

// Samples one token per row of `logits` ([rows][ldk], element-aligned rows
// of `vocab` logits); probs may be NULL.  False if a launch failed.
bool sample_launch(const void *logits, bool bf16, int64_t rows, int32_t vocab, int64_t ldk, const float *uniform,
                   const SampleSettings &settings, int32_t *tokens, float *probs, void *workspace,
                   hipStream_t stream);

}  // namespace fgd
