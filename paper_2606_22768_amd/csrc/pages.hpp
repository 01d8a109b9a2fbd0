// pages.hpp -- launchers of the kernels that give pages of a cache to
// requests and take them back.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fgd {

// The state that a program keeps on the GPU.
struct PagesView {
    int32_t *tables, *lengths, *free, *free_count;
    int64_t table_stride;
    int32_t requests, width, page, capacity;  // of the stack of free pages
};

// False if a launch failed.
bool pages_extend_launch(const PagesView &p, const int32_t *counts, int64_t tokens, int32_t *starts,
                         int32_t *positions, int64_t *slots, hipStream_t stream);
bool pages_truncate_launch(const PagesView &p, const int32_t *keep, hipStream_t stream);

}  // namespace fgd
