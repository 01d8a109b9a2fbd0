// sample.hip -- one token per row of logits by temperature, top-k, top-p
// and min-p, from given random numbers.
//
// A token's weight is w = 2^t, t = (z - max z) c, c = (1 / T) log2(e), each
// operation rounded to float32, and its mass the whole number
// floor(w 2^31 + 1/2).  Masses add exactly in any order, so a row's token
// depends on its logits, settings and random number alone: not on the batch,
// the number of blocks or the order of their sums.  2^-31 of the largest
// probability is far below the 2^-24 that separates float32 random numbers.
//
// The tokens stand in descending order of their logits, the lower index
// first among equal ones.  Top-k, top-p and min-p each keep a prefix of that
// order, so their intersection is the shortest of the three and its mass the
// least of theirs; the drawn token is the one whose span of mass holds
// floor(u mass).  Both searches (where top-k or top-p cuts, and the draw)
// are for the group of equal logits at a given count or mass of the order,
// found by radix descent over the logits' order-preserving keys.
#include <hip/hip_runtime.h>

#include "sample.hpp"

namespace fgd {
namespace {

constexpr int kThreads = 1024, kBins = 2048, kBinBits = 11;

struct Shared {
    uint32_t count[kBins];
    unsigned long long mass[kBins];
    unsigned long long wave_count[kThreads / 64], wave_mass[kThreads / 64];
    // The bin found by a search, and what stands before it.
    uint32_t bin, bin_count;
    unsigned long long bin_mass, above_count, above_mass;
    float wave_max[kThreads / 64];
    int wave_nan[kThreads / 64], index;
};

__device__ inline float value(float v) { return v; }
__device__ inline float value(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }

// Larger logits have larger keys; the two zeros share one.
__device__ inline uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ inline float weight(float z, float top, float c) {
#pragma clang fp contract(off)
    const float t = z == top ? 0.0f : (z - top) * c;
    return z == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(fmaxf(t, -126.0f));
}

__device__ inline uint32_t mass_of(float w) { return static_cast<uint32_t>(fmaf(w, 0x1p31f, 0.5f)); }

// f(index, logit) for every element of a row, by the whole block.
template <typename T, typename F>
__device__ inline void scan_row(const T *row, int vocab, F f) {
    for (int i = threadIdx.x; i < vocab; i += kThreads) f(i, value(row[i]));
}

__device__ inline unsigned long long wave_sum(unsigned long long v) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Finds the first bin, from the highest, at whose end the measure (counts,
// or masses) exceeds `target`; the histogram's total does.  Each thread owns
// two bins.
__device__ void find_bin(Shared &s, bool by_mass, unsigned long long target) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int hi = kBins - 1 - 2 * t, lo = hi - 1;
    unsigned long long c = s.count[hi] + static_cast<unsigned long long>(s.count[lo]), m = s.mass[hi] + s.mass[lo];
    unsigned long long ci = c, mi = m;  // inclusive sums within the wave
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned long long cu = __shfl_up(ci, o), mu = __shfl_up(mi, o);
        if (lane >= o) ci += cu, mi += mu;
    }
    if (lane == 63) s.wave_count[wave] = ci, s.wave_mass[wave] = mi;
    __syncthreads();
    for (int w = 0; w < wave; ++w) ci += s.wave_count[w], mi += s.wave_mass[w];
    unsigned long long ce = ci - c, me = mi - m;  // before this thread's bins
    const unsigned long long before = by_mass ? me : ce, through = by_mass ? mi : ci;
    if (before <= target && target < through) {
        const unsigned long long first = by_mass ? s.mass[hi] : s.count[hi];
        const int bin = target < before + first ? hi : lo;
        if (bin == lo) ce += s.count[hi], me += s.mass[hi];
        s.bin = bin;
        s.bin_count = s.count[bin];
        s.bin_mass = s.mass[bin];
        s.above_count = ce;
        s.above_mass = me;
    }
    __syncthreads();
}

struct Group {  // the tokens of one logit in the order
    uint32_t key, count;
    unsigned long long above_count, above_mass, mass;  // mass: of one token
};

template <typename T>
__device__ Group find_group(Shared &s, const T *row, int vocab, float top, float c, bool by_mass,
                            unsigned long long target) {
    uint32_t prefix = 0;
    unsigned long long above_count = 0, above_mass = 0;
    const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
    for (int level = 0; level < 3; ++level) {
        const int shift = shifts[level];
        const uint32_t mask = (1u << bits[level]) - 1;
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = 0, s.mass[i] = 0;
        __syncthreads();
        scan_row(row, vocab, [&](int, float z) {
            const uint32_t key = key_of(z);
            if (level && (key >> (shift + bits[level])) != prefix) return;
            const uint32_t bin = (key >> shift) & mask;
            atomicAdd(&s.count[bin], 1u);
            const uint32_t m = mass_of(weight(z, top, c));
            if (m) atomicAdd(&s.mass[bin], static_cast<unsigned long long>(m));
        });
        __syncthreads();
        find_bin(s, by_mass, target);
        const unsigned long long at = by_mass ? s.above_mass : s.above_count;
        target -= at;
        above_count += s.above_count;
        above_mass += s.above_mass;
        prefix = prefix << bits[level] | s.bin;
        __syncthreads();
    }
    Group g;
    g.key = prefix;
    g.count = s.bin_count;
    g.mass = s.bin_mass / s.bin_count;
    g.above_count = above_count;
    g.above_mass = above_mass;
    __syncthreads();
    return g;
}

// The index of the n-th token of key `key`, by radix descent over indices.
template <typename T>
__device__ int find_index(Shared &s, const T *row, int vocab, uint32_t key, uint32_t n) {
    uint32_t prefix = 0;
    const int shifts[3] = {22, 11, 0};
    for (int level = 0; level < 3; ++level) {
        const int shift = shifts[level];
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = 0, s.mass[i] = 0;
        __syncthreads();
        scan_row(row, vocab, [&](int i, float z) {
            const uint32_t r = ~static_cast<uint32_t>(i);  // find_bin counts from the highest bin
            if (key_of(z) != key || (level && (r >> (shift + kBinBits)) != prefix)) return;
            atomicAdd(&s.count[(r >> shift) & (kBins - 1)], 1u);
        });
        __syncthreads();
        find_bin(s, false, n);
        n -= static_cast<uint32_t>(s.above_count);
        prefix = prefix << kBinBits | s.bin;
        __syncthreads();
    }
    return static_cast<int>(~prefix & 0xffffffffu);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const T *__restrict__ logits, int64_t rows, int vocab,
                                                          int64_t ldk, const float *__restrict__ uniform,
                                                          SampleSettings set, int32_t *__restrict__ tokens,
                                                          float *__restrict__ probs) {
    __shared__ Shared s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = logits + r * ldk;
        float best = -__builtin_inff();
        int bad = 0;
        scan_row(row, vocab, [&](int, float z) {
            bad |= z != z;
            best = fmaxf(best, z);
        });
        for (int o = 32; o; o >>= 1) best = fmaxf(best, __shfl_xor(best, o)), bad |= __shfl_xor(bad, o);
        if (lane == 0) s.wave_max[wave] = best, s.wave_nan[wave] = bad;
        __syncthreads();
        for (int w = 0; w < kThreads / 64; ++w) best = fmaxf(best, s.wave_max[w]), bad |= s.wave_nan[w];
        __syncthreads();
        if (bad || best == -__builtin_inff()) {
            if (threadIdx.x == 0) {
                tokens[r] = -1;
                if (probs) probs[r] = bad ? __builtin_nanf("") : 0.0f;
            }
            continue;
        }
        const float temperature = set.temperature_rows ? set.temperature_rows[r] : set.temperature;
        float c = 1.0f / temperature;
        c = c * 1.44269504088896340736f;
        const bool greedy = !(temperature > 0.0f) || c == __builtin_inff();
        if (greedy) c = 1.0f;
        int k = greedy ? 1 : set.top_k_rows ? set.top_k_rows[r] : set.top_k;
        if (k <= 0 || k > vocab) k = vocab;
        const float top_p = set.top_p_rows ? set.top_p_rows[r] : set.top_p;
        float min_p = set.min_p_rows ? set.min_p_rows[r] : set.min_p;
        if (min_p > 1.0f) min_p = 1.0f;

        // Masses of everything, and of what min-p keeps.
        unsigned long long all = 0, kept = 0;
        scan_row(row, vocab, [&](int, float z) {
            const float w = weight(z, best, c);
            const unsigned long long m = mass_of(w);
            all += m;
            if (!(w < min_p)) kept += m;
        });
        all = wave_sum(all), kept = wave_sum(kept);
        if (lane == 0) s.wave_count[wave] = all, s.wave_mass[wave] = kept;
        __syncthreads();
        all = kept = 0;
        for (int w = 0; w < kThreads / 64; ++w) all += s.wave_count[w], kept += s.wave_mass[w];
        __syncthreads();

        unsigned long long total = all;
        if (k < vocab) {
            const Group g = find_group(s, row, vocab, best, c, false, k - 1);
            total = g.above_mass + (k - g.above_count) * g.mass;
        }
        if (top_p < 1.0f) {
            const double want = ceil(static_cast<double>(top_p) * static_cast<double>(total));
            const unsigned long long limit = want >= 1.0 ? static_cast<unsigned long long>(want) : 1;
            if (limit < total) {
                const Group g = find_group(s, row, vocab, best, c, true, limit - 1);
                total = g.above_mass + ((limit - 1 - g.above_mass) / g.mass + 1) * g.mass;
            }
        }
        total = min(total, kept);
        const double at = static_cast<double>(uniform[r]) * static_cast<double>(total);
        unsigned long long target = at > 0.0 ? static_cast<unsigned long long>(at) : 0;
        target = min(target, total - 1);
        const Group g = find_group(s, row, vocab, best, c, true, target);
        const int index = find_index(s, row, vocab, g.key, static_cast<uint32_t>((target - g.above_mass) / g.mass));
        if (threadIdx.x == 0) {
            tokens[r] = index;
            if (probs) probs[r] = static_cast<float>(g.mass) / static_cast<float>(total);
        }
        __syncthreads();
    }
}

}  // namespace

bool sample_launch(const void *logits, bool bf16, int64_t rows, int32_t vocab, int64_t ldk, const float *uniform,
                   const SampleSettings &settings, int32_t *tokens, float *probs, hipStream_t stream) {
    if (rows == 0) return true;
    const int grid = static_cast<int>(rows < 4096 ? rows : 4096);
    if (bf16)
        sample_kernel<<<grid, kThreads, 0, stream>>>(static_cast<const uint16_t *>(logits), rows, vocab, ldk, uniform,
                                                     settings, tokens, probs);
    else
        sample_kernel<<<grid, kThreads, 0, stream>>>(static_cast<const float *>(logits), rows, vocab, ldk, uniform,
                                                     settings, tokens, probs);
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
