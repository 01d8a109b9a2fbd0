// cache.hpp -- layout of a paged cache of keys and values in microscaled
// 4-bit floating point (the format: mx4.hpp), and the launchers of the
// kernels that write, read and attend to it.
//
// The layout is that of the matrix instruction's operands.  A page holds
// `page` tokens of every head; a head's 16 consecutive tokens are a group of
// 17 D contiguous bytes (D the head's elements, NB = D / 32 its blocks):
//
//   keys' codes    8 D bytes: lane l = token + 16 h holds the token's elements
//                  [h D/4, (h + 1) D/4), low nibble first, in D/8 bytes, as
//                  the products' left operand (16 tokens, four lanes each)
//   values' codes  8 D bytes: lane l = n + 16 h holds the elements 32 b + 2 n
//                  (low nibble) and 32 b + 2 n + 1 of tokens 4 h .. 4 h + 3,
//                  byte 4 b + token % 4 of the lane's D/8
//   keys' scales   D/2 bytes: block b of a token is byte token NB + b
//   values' scales D/2 bytes: block b of a token is byte
//                  (token / 4) 4 NB + 4 b + token % 4
//
// The group of token t of page p, head h is at index (p heads + h) (page /
// 16) + t / 16.  A byte belongs to one token, so tokens are written without
// reading what is there.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fgd {

constexpr int kCacheGroup = 16;  // tokens

struct CacheView {
    uint8_t *data;
    int64_t pages;
    int32_t heads, dim, page_shift;  // page = 1 << page_shift tokens

    __host__ __device__ int64_t group_bytes() const { return 17 * static_cast<int64_t>(dim); }
    __host__ __device__ int64_t slots() const { return pages << page_shift; }
    __host__ __device__ int64_t group(int64_t page, int64_t head, int64_t g) const {
        return (((page * heads + head) << (page_shift - 4)) + g) * group_bytes();
    }
};

// A dense array [tokens][heads][dim], heads contiguous.
struct HeadRows {
    void *p;
    int64_t token_stride, head_stride;
};

// False if a launch failed.
bool cache_write_launch(const CacheView &cache, const HeadRows &k, const HeadRows &v, bool bf16, int64_t tokens,
                        const int64_t *slots, hipStream_t stream);
bool cache_read_launch(const CacheView &cache, const HeadRows &k, const HeadRows &v, bool bf16, int64_t tokens,
                       const int64_t *slots, hipStream_t stream);

struct AttendArgs {
    CacheView cache;
    HeadRows q, out;
    const int32_t *tables, *lengths, *starts;  // starts NULL: one query per sequence
    int64_t table_stride, tokens;
    int32_t sequences, width, q_heads, most_queries, window;
    float scale;
    bool bf16;
};

int64_t attend_workspace_bytes(const AttendArgs &a);
bool attend_launch(const AttendArgs &a, void *workspace, hipStream_t stream);

}  // namespace fgd
