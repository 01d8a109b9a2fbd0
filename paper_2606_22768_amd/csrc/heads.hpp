// heads.hpp -- launchers of the kernels that norm and rotate the heads of
// queries and keys, and of their gradients.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fgd {

// A dense array [batch][tokens][heads][dim], heads contiguous.
struct HeadArray {
    void *p;
    int64_t batch_stride, token_stride, head_stride;
};

// One of the two inputs: its heads, or their gradient and what that is of.
struct HeadSide {
    HeadArray x, dy, out;  // dy: gradients only
    const void *weight;    // [dim], or [batch][dim]; NULL: no norm
    float *weight_grad;
    int32_t heads;
};

struct HeadsArgs {
    HeadSide side[2];  // queries, keys
    const int32_t *positions;
    const double *freqs;
    int64_t batch, tokens, position_stride, weight_stride;
    int32_t dim, rot;
    float eps;
    bool interleaved, bf16, weight_bf16;
};

// False if a launch failed.
bool rotate_heads_launch(const HeadsArgs &a, hipStream_t stream);
int64_t rotate_heads_grads_workspace_bytes(const HeadsArgs &a);
bool rotate_heads_grads_launch(const HeadsArgs &a, float *workspace, hipStream_t stream);

}  // namespace fgd
