// pages.hip -- block tables and slot maps from the requests' lengths.
//
// Bound by latency: a decoding turn moves a few bytes per request.  One block
// sums the requests' needs, hands out pages from the top of the stack and
// writes the tables; the tokens' positions and slots follow in the same
// launch where they are few, else in a second over the card.
// 64 requests of a token each: 4 us, given back in 3; 513 of up to 256: 9, 4 for
// the tokens' slots, 9 (the pages' searches of two requests side by side in
// a thread took 28 us for the three's 22).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pages.hpp"

namespace fgd {
namespace {

constexpr int kMostThreads = 1024;
// Tokens that the first block still fills by itself.
constexpr int64_t kFewTokens = 4096;

struct Pair {
    int64_t a, b;
};

// Inclusive sums over the block's threads.
__device__ inline Pair scan(Pair v, Pair *waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t a = __shfl_up(static_cast<long long>(v.a), o), b = __shfl_up(static_cast<long long>(v.b), o);
        if (lane >= o) v.a += a, v.b += b;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = v;
    __syncthreads();
    for (int i = 0; i < wave; ++i) v.a += waves[i].a, v.b += waves[i].b;
    return v;
}

// The last of n ascending sums that is not above x (sums[0] <= x).
template <typename I>
__device__ inline int last_at(const I *sums, int n, I x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (sums[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

__device__ inline int pages_for(int64_t tokens, int page) { return static_cast<int>((tokens + page - 1) / page); }

// Positions and slots of tokens [first, tokens) in steps; lengths are the new ones.
__device__ inline void fill(const PagesView &p, int64_t first, int64_t step, int64_t tokens, const int32_t *starts,
                            int32_t *positions, int64_t *slots) {
    const int64_t real = starts[p.requests];
    for (int64_t t = first; t < tokens; t += step) {
        int32_t position = 0;
        int64_t slot = -1;
        if (t < real) {
            const int b = last_at(starts, p.requests, static_cast<int32_t>(t));
            position = p.lengths[b] - starts[b + 1] + static_cast<int32_t>(t);
            const int at = position / p.page;
            const int32_t page = p.tables[b * p.table_stride + at];
            if (page >= 0) slot = static_cast<int64_t>(page) * p.page + (position - at * p.page);
        }
        positions[t] = position;
        slots[t] = slot;
    }
}

__global__ __launch_bounds__(kMostThreads) void extend_kernel(PagesView p, const int32_t *__restrict__ counts,
                                                              int64_t tokens, int32_t *starts, int32_t *positions,
                                                              int64_t *slots, bool fills) {
    __shared__ Pair waves[kMostThreads / 64];
    __shared__ int32_t taken[kMostThreads + 1], have[kMostThreads];
    __shared__ Pair carry[2];
    const int n = blockDim.x, tid = threadIdx.x;
    const int32_t top = min(max(*p.free_count, 0), p.capacity);
    if (tid == 0) carry[0] = carry[1] = Pair{0, 0}, starts[0] = 0;
    for (int b0 = 0; b0 < p.requests; b0 += n) {
        const int b = b0 + tid, here = min(n, p.requests - b0);
        int64_t held = 0, asked = 0, need = 0, had = 0;
        if (b < p.requests) {
            held = max(p.lengths[b], 0);
            asked = max(counts[b], 0);
            had = pages_for(held, p.page);
            const int64_t want = (held + asked + p.page - 1) / p.page;
            if (want > p.width || held + asked > INT32_MAX)
                asked = 0;
            else
                need = max(want - had, INT64_C(0));
        }
        Pair upto = scan(Pair{need, asked}, waves);
        const Pair before = carry[0];
        const bool granted = asked > 0 && (need == 0 || before.a + upto.a <= top) && before.b + upto.b <= tokens;
        if (!granted) asked = need = 0;
        const Pair given = scan(Pair{need, asked}, waves);  // its barriers also end the readings of carry[0]
        const Pair given_before = carry[1];
        if (b < p.requests) {
            starts[b + 1] = static_cast<int32_t>(given_before.b + given.b);
            if (granted) p.lengths[b] = static_cast<int32_t>(held + asked);
            taken[tid] = static_cast<int32_t>(given.a - need);
            have[tid] = static_cast<int32_t>(had);
        }
        if (tid == n - 1) {
            taken[here] = static_cast<int32_t>(given.a);
            carry[0] = Pair{before.a + upto.a, before.b + upto.b};
        }
        __syncthreads();
        if (tid == n - 1) carry[1] = Pair{given_before.a + given.a, given_before.b + given.b};
        const int fresh = taken[here];
        for (int i = tid; i < fresh; i += n) {
            const int r = last_at(taken, here, i);
            p.tables[(b0 + r) * p.table_stride + have[r] + (i - taken[r])] =
                p.free[top - 1 - static_cast<int32_t>(given_before.a) - i];
        }
        __syncthreads();
    }
    if (tid == 0) *p.free_count = top - static_cast<int32_t>(carry[1].a);
    if (fills) {
        __syncthreads();
        fill(p, tid, n, tokens, starts, positions, slots);
    }
}

__global__ __launch_bounds__(256) void fill_kernel(PagesView p, int64_t tokens, const int32_t *__restrict__ starts,
                                                   int32_t *positions, int64_t *slots) {
    fill(p, static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, static_cast<int64_t>(gridDim.x) * 256, tokens, starts,
         positions, slots);
}

__global__ __launch_bounds__(kMostThreads) void truncate_kernel(PagesView p, const int32_t *__restrict__ keep) {
    __shared__ Pair waves[kMostThreads / 64];
    __shared__ int32_t before[kMostThreads + 1], first[kMostThreads];
    __shared__ int64_t total, carry;
    const int n = blockDim.x, tid = threadIdx.x;
    const int64_t top = min(max(*p.free_count, 0), p.capacity);
    auto of = [&](int b, int &stay) {  // how many pages request b gives back
        const int held = max(p.lengths[b], 0), left = min(held, max(keep[b], 0));
        const int have = min(pages_for(held, p.page), p.width);
        stay = min(pages_for(left, p.page), have);
        return have - stay;
    };
    if (tid == 0) carry = 0;
    int64_t mine = 0;
    for (int b = tid; b < p.requests; b += n) {
        int stay;
        mine += of(b, stay);
    }
    const Pair all = scan(Pair{mine, 0}, waves);
    if (tid == n - 1) total = all.a;
    __syncthreads();
    for (int b0 = 0; b0 < p.requests; b0 += n) {
        const int b = b0 + tid, here = min(n, p.requests - b0);
        int stay = 0, back = 0;
        if (b < p.requests) {
            back = of(b, stay);
            p.lengths[b] = min(max(p.lengths[b], 0), max(keep[b], 0));
        }
        const Pair upto = scan(Pair{back, 0}, waves);
        if (b < p.requests) before[tid] = static_cast<int32_t>(upto.a - back), first[tid] = stay;
        if (tid == n - 1) before[here] = static_cast<int32_t>(upto.a);
        __syncthreads();
        const int given = before[here];
        for (int i = tid; i < given; i += n) {
            const int r = last_at(before, here, i);
            int32_t *entry = p.tables + (b0 + r) * p.table_stride + first[r] + (i - before[r]);
            const int64_t at = top + total - 1 - (carry + i);
            if (at < p.capacity) p.free[at] = *entry;
            *entry = -1;
        }
        __syncthreads();
        if (tid == 0) carry += given;
    }
    if (tid == 0) *p.free_count = static_cast<int32_t>(min(top + total, static_cast<int64_t>(p.capacity)));
}

unsigned threads_for(int requests) { return std::clamp((requests + 63) / 64 * 64, 64, kMostThreads); }

}  // namespace

bool pages_extend_launch(const PagesView &p, const int32_t *counts, int64_t tokens, int32_t *starts,
                         int32_t *positions, int64_t *slots, hipStream_t stream) {
    const bool fills = tokens <= kFewTokens;
    const unsigned n = fills ? std::max(threads_for(p.requests), static_cast<unsigned>(std::min<int64_t>(
                                                                     (tokens + 63) / 64 * 64, kMostThreads)))
                             : threads_for(p.requests);
    extend_kernel<<<1, n, 0, stream>>>(p, counts, tokens, starts, positions, slots, fills);
    if (!fills)
        fill_kernel<<<static_cast<unsigned>(std::min<int64_t>((tokens + 255) / 256, 1 << 20)), 256, 0, stream>>>(
            p, tokens, starts, positions, slots);
    return hipGetLastError() == hipSuccess;
}

bool pages_truncate_launch(const PagesView &p, const int32_t *keep, hipStream_t stream) {
    if (p.requests == 0) return true;
    truncate_kernel<<<1, threads_for(p.requests), 0, stream>>>(p, keep);
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
