// sample.hip -- one token per row of logits by temperature, top-k, top-p
// and min-p, from given random numbers.
//
// A token's weight is w = 2^t, t = (z - max z) c, c = (1 / T) log2(e), each
// operation rounded to float32, and its mass the whole part of w 2^31 + 1/2,
// rounded to float32.  Masses add exactly in any order, so a row's token
// depends on its logits, settings and random number alone: not on the batch,
// the number of blocks or the order of their sums.  2^-31 of the largest
// probability is far below the 2^-24 that separates float32 random numbers.
//
// The tokens stand in descending order of their logits, the lower index
// first among equal ones.  Top-k, top-p and min-p each keep a prefix of that
// order, so their intersection is the shortest of the three and its mass the
// least of theirs; the drawn token is the one whose span of mass holds
// floor(u mass).  So a row is sampled by finding places in the order at a
// given count or mass, without sorting it:
//   1. the row's maximum;
//   2. a histogram of masses (and, for top-k, counts) over bins of t, each
//      1/64 wide: 2048 bins reach the smallest mass;
//   3. of the few bins in which a cut or the draw can fall (a cut that is
//      known to a bin gives a range for the next), the tokens, collected,
//      sorted and summed up: these give the exact places.
// Where those bins hold more than the room (thousands of nearly equal
// tokens), the row is searched by radix descent over its logits' bits
// instead, which needs no room and takes many more passes.
//
// Many rows: a block per row.  Fewer: a row's slices on several blocks, a
// kernel for each step, histogram and tokens in the workspace; the block of a
// row that ends last finds its token.  Many long bf16 rows: a pass counts the
// tokens of each 16-bit value, exact places follow from the counts, and a
// second pass finds the token.
//
// Bound by the reads of the logits: three passes over a row (two for counted
// ones), none of which the L2s serve: 2048 x 128256 f32 reads 3.16 GB for 1.05
// in 455 to 476 us (6.6 to 6.9 TB/s); bf16 1.08 for 0.53 in 196 us (5.5), 321
// in three passes; one read at 6.6 TB/s would be 159 and 80.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sample.hpp"

namespace fgd {
namespace {

typedef unsigned long long u64;

constexpr int kBins = 2048, kBinBits = 11;
constexpr int kRoom = 4096;          // tokens that a row's search can collect
constexpr int kMostSlices = 64;      // of a row
constexpr int kThreads = 512;
constexpr float kPerOctave = 64.0f;  // bins per factor of two of weight

__device__ inline float value(float v) { return v; }
__device__ inline float value(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }

// Larger logits have larger keys; the two zeros share one.
__device__ inline uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float logit_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// log2 of a token's weight; the largest logit's is 0.  NaN (an infinite
// difference times c = 0) stands for no weight.
__device__ inline float scaled(float z, float top, float c) {
#pragma clang fp contract(off)
    return (z - top) * c;
}
// The same where the largest logit may be infinite.
__device__ inline float scaled_any(float z, float top, float c) { return z == top ? 0.0f : scaled(z, top, c); }
// 2^t; where the instruction flushes its result (t < -126) there is no mass.
__device__ inline float weight(float t) { return __builtin_amdgcn_exp2f(t); }
// w 2^31 is exact, its sum with 1/2 rounded: a whole number from 2^23 to 2^24
// and a half is a tie, which goes to the even one.
__device__ inline uint32_t mass_of(float w) { return static_cast<uint32_t>(fmaf(w, 0x1p31f, 0.5f)); }
// The bin of a token that has mass (t >= -32).
__device__ inline uint32_t bin_of(float t) {
    return min(static_cast<uint32_t>(-kPerOctave * t), static_cast<uint32_t>(kBins - 1));
}
// The same of any; kBins where there is no mass.
__device__ inline int bin_of_any(float t) { return t >= -32.0f ? static_cast<int>(bin_of(t)) : kBins; }

// f(index of the first, logits[n]) for the elements [lo, hi) of a row, some
// at a time so that their steps interleave, by a block of TH threads.
template <int TH, typename T, typename F>
__device__ inline void scan_row(const T *row, int lo, int hi, F f) {
    constexpr int kPer = 16 / sizeof(T), kAhead = 2;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + lo);
    const int head = min(hi - lo, static_cast<int>((16 - (at & 15)) & 15) / static_cast<int>(sizeof(T)));
    const int vectors = (hi - lo - head) / kPer, first = lo + head, tail = first + vectors * kPer;
    const uint4 *v = reinterpret_cast<const uint4 *>(row + first);
    auto each = [&](int i, uint4 u) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        float z[kPer];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) {
                z[j] = __uint_as_float(w[j]);
            } else {
                z[2 * j] = __uint_as_float(w[j] << 16);
                z[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
        }
        f(first + i * kPer, z);
    };
    int i = threadIdx.x;
    for (; i + (kAhead - 1) * TH < vectors; i += kAhead * TH) {
        uint4 u[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) u[a] = v[i + a * TH];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) each(i + a * TH, u[a]);
    }
    for (; i < vectors; i += TH) each(i, v[i]);
    const int rest = static_cast<int>(threadIdx.x);
    const int at_end = rest < head ? lo + rest : tail + rest - head;
    if (at_end < hi) {
        const float z[1] = {value(row[at_end])};
        f(at_end, z);
    }
}

// f(index, logit), one by one.
template <int TH, typename T, typename F>
__device__ inline void scan_row_singly(const T *row, int lo, int hi, F f) {
    scan_row<TH>(row, lo, hi, [&](int i, const auto &z) {
#pragma unroll
        for (int j = 0; j < static_cast<int>(sizeof(z) / sizeof(float)); ++j) f(i + j, z[j]);
    });
}

// A value that is the same in a wave, in a scalar register.
__device__ inline float uniform_value(float v) {
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

// A row's settings, made definite.
struct Settings {
    float c, top_p, min_p;
    int k;  // 1..vocab
};

__device__ inline Settings settings_of(const SampleSettings &set, int64_t r, int vocab) {
    Settings s;
    const float temperature = set.temperature_rows ? set.temperature_rows[r] : set.temperature;
    s.c = 1.0f / temperature;
    s.c = s.c * 1.44269504088896340736f;
    const bool greedy = !(temperature > 0.0f) || s.c == __builtin_inff();
    if (greedy) s.c = 1.0f;
    s.k = greedy ? 1 : set.top_k_rows ? set.top_k_rows[r] : set.top_k;
    if (s.k <= 0 || s.k > vocab) s.k = vocab;
    s.top_p = set.top_p_rows ? set.top_p_rows[r] : set.top_p;
    s.min_p = set.min_p_rows ? set.min_p_rows[r] : set.min_p;
    if (s.min_p > 1.0f) s.min_p = 1.0f;
    s.c = uniform_value(s.c), s.top_p = uniform_value(s.top_p), s.min_p = uniform_value(s.min_p);
    s.k = __builtin_amdgcn_readfirstlane(s.k);
    return s;
}

// The mass that top-p asks for, of a total.
__device__ inline u64 nucleus(float top_p, u64 total) {
    if (!(top_p < 1.0f)) return total;
    const double want = ceil(static_cast<double>(top_p) * static_cast<double>(total));
    return min(want >= 1.0 ? static_cast<u64>(want) : u64{1}, total);
}
// The place of the draw, of a total of at least 1.
__device__ inline u64 place(float u, u64 total) {
    const double at = static_cast<double>(u) * static_cast<double>(total);
    return min(at > 0.0 ? static_cast<u64>(at) : u64{0}, total - 1);
}

// The tokens a row's search needs: three ranges of logits.
struct Wanted {
    float lo[3], hi[3];
    __device__ bool has(float z) const {
        return (z >= lo[0] & z <= hi[0]) | (z >= lo[1] & z <= hi[1]) | (z >= lo[2] & z <= hi[2]);  // no branches
    }
};

template <int TH>
struct Bins {
    u64 mass[kBins + 1];  // a histogram, then the sums before each bin; the total
    uint32_t count[kBins + 1];
    u64 wave_a[TH / 64], wave_b[TH / 64], found_mass, found_count;
    uint32_t found;
    float wave_max[TH / 64];
};
template <int TH, int ROOM = kRoom>
struct Shared : Bins<TH> {
    __attribute__((aligned(16))) u64 list[ROOM];  // key, then ~index: the larger is the earlier in the order
    u64 total;
    uint32_t listed, first, last;
    Wanted wanted;
};

// The largest value of the block's, NaN if one is.
template <int TH>
__device__ inline float block_max(Bins<TH> &s, float best, bool bad) {
    for (int o = 32; o; o >>= 1) best = fmaxf(best, __shfl_xor(best, o));
    if (__any(bad)) best = __builtin_nanf("");
    if ((threadIdx.x & 63) == 0) s.wave_max[threadIdx.x >> 6] = best;
    __syncthreads();
    best = s.wave_max[0];
    for (int w = 1; w < TH / 64; ++w) {
        const float v = s.wave_max[w];
        best = v != v || best != best ? __builtin_nanf("") : fmaxf(best, v);
    }
    __syncthreads();
    return uniform_value(best);
}

// Sums over the lanes up to this one.
template <int CTRL, int ROWS>
__device__ inline u64 moved(u64 v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0u, static_cast<uint32_t>(v), CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0u, static_cast<uint32_t>(v >> 32), CTRL, ROWS, 0xf, false);
    return static_cast<u64>(hi) << 32 | lo;
}
__device__ inline u64 wave_scan(u64 v) {
    v += moved<0x111, 0xf>(v);  // from 1, 2, 4 and 8 lanes before, in rows of 16
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);  // a row's last lane to the next row
    v += moved<0x143, 0xc>(v);  // lane 31 to the upper half
    return v;
}

// Sums of a and b over the threads before this one; the totals in ta, tb.
template <int TH>
__device__ inline void scan_threads(u64 *wave_a, u64 *wave_b, u64 &a, u64 &b, u64 &ta, u64 &tb) {
    const int wave = threadIdx.x >> 6;
    const u64 ia = wave_scan(a), ib = wave_scan(b);
    if ((threadIdx.x & 63) == 63) wave_a[wave] = ia, wave_b[wave] = ib;
    __syncthreads();
    a = ia - a, b = ib - b;
    ta = tb = 0;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) {
        const u64 x = wave_a[w], y = wave_b[w];
        a += w < wave ? x : 0, b += w < wave ? y : 0;
        ta += x, tb += y;
    }
    __syncthreads();
}

template <int TH>
__device__ inline void scan_threads(Bins<TH> &s, u64 &a, u64 &b, u64 &ta, u64 &tb) {
    scan_threads<TH>(s.wave_a, s.wave_b, a, b, ta, tb);
}

template <int TH>
__device__ inline void clear_bins(Bins<TH> &s) {
    for (int i = threadIdx.x; i < kBins; i += TH) s.mass[i] = 0, s.count[i] = 0;
    __syncthreads();
}

// The sums before each bin, of a histogram whose bins thread i holds kOwn
// of, from kOwn i.
template <int TH>
__device__ inline void scan_bins(Bins<TH> &s, const u64 (&m)[kBins / TH], const uint32_t (&c)[kBins / TH]) {
    constexpr int kOwn = kBins / TH;
    u64 a = 0, b = 0, ta, tb;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) a += m[i], b += c[i];
    scan_threads<TH>(s, a, b, ta, tb);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        s.mass[threadIdx.x * kOwn + i] = a, s.count[threadIdx.x * kOwn + i] = static_cast<uint32_t>(b);
        a += m[i], b += c[i];
    }
    if (threadIdx.x == 0) s.mass[kBins] = ta, s.count[kBins] = static_cast<uint32_t>(tb);
    __syncthreads();
}

// The bin that holds the place x (below the total); by a wave.
template <typename U>
__device__ inline int bin_at(const U *before, U x) {
    static_assert(kBins == 64 * 32, "two steps");
    const int lane = threadIdx.x & 63;
    const int part = __ffsll(static_cast<u64>(__ballot(before[32 * lane] <= x && x < before[32 * lane + 32]))) - 1;
    const int bin = 32 * part + (lane & 31);
    return 32 * part + ((__ffsll(static_cast<u64>(__ballot(before[bin] <= x && x < before[bin + 1]))) - 1) & 31);
}

// The smallest key whose bin is `bin` or an earlier one; each lane its own.
// pred(key) is monotone, false at -infinity and true at the largest logit.
__device__ inline uint32_t first_key(int bin, float top, float c) {
    uint32_t lo = key_of(-__builtin_inff()), hi = key_of(top);
    auto pred = [&](uint32_t key) { return bin_of_any(scaled(logit_of(key), top, c)) <= bin; };
    if (bin < 0) return hi + 1;
    // Where the inverse puts it, give or take its rounding.
    const float guess = top - static_cast<float>(bin + 1) / (kPerOctave * c);
    if (guess == guess && guess > -__builtin_inff()) {
        const uint32_t g = key_of(guess), a = g - 64, b = g + 64;
        if (a > lo && a < hi) (pred(a) ? hi : lo) = a;
        if (b > lo && b < hi) (pred(b) ? hi : lo) = b;
    }
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        (pred(mid) ? hi : lo) = mid;
    }
    return hi;
}

// What to collect, from the summed histogram; by the block's first wave.  A
// step's total, with which the next one works, is known to a range lo..hi:
// of top-k's cut its bin is wanted, of top-p's and the draw's the bins from
// one end's to the other's.  kept: the mass that min-p keeps.
template <int TH, int ROOM>
__device__ inline void find_wanted(Shared<TH, ROOM> &s, const Settings &set, float u, u64 kept, float top) {
    if (threadIdx.x >= 64) return;
    int first[3] = {0, 0, 0}, last[3] = {-1, -1, -1};  // none
    u64 lo = s.mass[kBins], hi = lo;
    const uint32_t k = static_cast<uint32_t>(set.k);
    if (k < s.count[kBins]) {
        first[0] = last[0] = bin_at<uint32_t>(s.count, k - 1);
        lo = s.mass[first[0]], hi = s.mass[first[0] + 1];
    }
    if (set.top_p < 1.0f) {
        const u64 p0 = max(nucleus(set.top_p, lo), u64{1}), p1 = nucleus(set.top_p, hi);
        first[1] = bin_at<u64>(s.mass, p0 - 1), last[1] = bin_at<u64>(s.mass, p1 - 1);
        lo = p0, hi = min(hi, s.mass[last[1] + 1]);
    }
    lo = max(min(lo, kept), u64{1}), hi = min(hi, kept);
    first[2] = bin_at<u64>(s.mass, place(u, lo)), last[2] = bin_at<u64>(s.mass, place(u, hi));
    const int lane = threadIdx.x, i = lane >> 1;
    if (lane < 6) {
        const int from = i == 0 ? first[0] : i == 1 ? first[1] : first[2],
                  to = i == 0 ? last[0] : i == 1 ? last[1] : last[2];
        const uint32_t key = first_key(lane & 1 ? from - 1 : to, top, set.c);
        if (lane & 1)
            s.wanted.hi[i] = to < from ? -1.0f : logit_of(key - 1);
        else
            s.wanted.lo[i] = to < from ? 1.0f : logit_of(key);
    }
}

// Sorts list[0, n), n a power of two above 64, from the largest.  A wave's 64
// pairs at a distance of up to 64 are 128 neighbours, which no other wave
// touches: between such steps, a wave's own order is enough.
template <int TH>
__device__ inline void sort_list(u64 *list, int n) {
    for (int size = 2; size <= n; size <<= 1)
        for (int step = size >> 1; step; step >>= 1) {
            for (int i = threadIdx.x; i < n / 2; i += TH) {
                const int a = 2 * i - (i & (step - 1)), b = a + step;
                const u64 x = list[a], y = list[b];
                if ((x < y) == ((a & size) == 0)) list[a] = y, list[b] = x;
            }
            const int next = step > 1 ? step >> 1 : size;
            if (max(step, next) > 64)
                __syncthreads();
            else
                asm volatile("" ::: "memory");
        }
}

// Finds the token among those collected, which are all of the wanted bins':
// at most one a thread, each against each.
template <int TH, int ROOM>
__device__ inline void finish_few(Shared<TH, ROOM> &s, const Settings &set, float u, u64 kept, float top, int listed,
                                  int32_t *token, float *prob) {
    static_assert(4 * TH <= ROOM, "the pairs' room");
    const int i = threadIdx.x;
    const bool some = i < listed;
    const u64 own = some ? s.list[i] : 0;
    const float t = scaled(logit_of(static_cast<uint32_t>(own >> 32)), top, set.c);
    const uint32_t m = some ? mass_of(weight(t)) : 0, bin = some ? bin_of(t) : kBins;
    // Beside each other: a token, its bin and mass.
    u64 *pairs = s.list + ROOM / 2;
    if (some) pairs[2 * i] = own, pairs[2 * i + 1] = static_cast<u64>(bin) << 32 | m;
    __syncthreads();
    u64 before = s.mass[bin];
    uint32_t rank = s.count[bin];
    if (i < (listed + 63) / 64 * 64) {  // the others' waves go on
#pragma unroll 4
        for (int j = 0; j < listed; ++j) {
            const u64 other = pairs[2 * j], what = pairs[2 * j + 1];
            const bool ahead = static_cast<uint32_t>(what >> 32) == bin && other > own;
            before += ahead ? static_cast<uint32_t>(what) : 0u;
            rank += ahead;
        }
    }
    u64 total = s.mass[kBins];
    if (static_cast<uint32_t>(set.k) < s.count[kBins]) {
        if (some && rank == static_cast<uint32_t>(set.k) - 1) s.total = before + m;
        __syncthreads();
        total = s.total;
        __syncthreads();
    }
    const u64 limit = nucleus(set.top_p, total);
    if (limit < total) {
        if (some && before < limit && limit <= before + m) s.total = before + m;
        __syncthreads();
        total = s.total;
    }
    total = min(total, kept);
    const u64 target = place(u, total);
    if (some && before <= target && target < before + m) {
        *token = static_cast<int32_t>(~static_cast<uint32_t>(own));
        if (prob) *prob = static_cast<float>(m) / static_cast<float>(total);
    }
}

// The same, of any number, sorted by the block.
template <int TH, int ROOM>
__device__ inline void finish(Shared<TH, ROOM> &s, const Settings &set, float u, u64 kept, float top, int listed,
                              int32_t *token, float *prob) {
    if (listed <= TH) {
        finish_few(s, set, u, kept, top, listed, token, prob);
        return;
    }
    int n = 1;
    while (n < listed) n <<= 1;
    for (int i = listed + threadIdx.x; i < n; i += TH) s.list[i] = 0;
    __syncthreads();
    sort_list<TH>(s.list, n);
    const int own = (n + TH - 1) / TH, base = threadIdx.x * own, end = min(base + own, listed);
    auto t_at = [&](int i) { return scaled(logit_of(static_cast<uint32_t>(s.list[i] >> 32)), top, set.c); };
    u64 sum = 0, none = 0, t0, t1;
    for (int i = base; i < end; ++i) sum += mass_of(weight(t_at(i)));
    scan_threads<TH>(s, sum, none, t0, t1);
    // A bin's sums become those to add to a place in the list.
    u64 at = sum;
    for (int i = base; i < end; ++i) {
        const float t = t_at(i);
        const uint32_t bin = bin_of(t);
        if (i == 0 || bin_of(t_at(i - 1)) != bin) s.mass[bin] -= at, s.count[bin] -= i;
        at += mass_of(weight(t));
    }
    u64 total = s.mass[kBins];
    __syncthreads();
    if (static_cast<uint32_t>(set.k) < s.count[kBins]) {
        at = sum;
        for (int i = base; i < end; ++i) {
            const float t = t_at(i);
            const uint32_t bin = bin_of(t), m = mass_of(weight(t));
            at += m;
            if (s.count[bin] + i == static_cast<uint32_t>(set.k) - 1) s.total = s.mass[bin] + at;
        }
        __syncthreads();
        total = s.total;
        __syncthreads();
    }
    const u64 limit = nucleus(set.top_p, total);
    if (limit < total) {
        at = sum;
        for (int i = base; i < end; ++i) {
            const float t = t_at(i);
            const uint32_t bin = bin_of(t), m = mass_of(weight(t));
            const u64 before = s.mass[bin] + at;
            if (before < limit && limit <= before + m) s.total = before + m;
            at += m;
        }
        __syncthreads();
        total = s.total;
    }
    total = min(total, kept);
    const u64 target = place(u, total);
    at = sum;
    for (int i = base; i < end; ++i) {
        const float t = t_at(i);
        const uint32_t bin = bin_of(t), m = mass_of(weight(t));
        const u64 before = s.mass[bin] + at;
        if (before <= target && target < before + m) {
            *token = static_cast<int32_t>(~static_cast<uint32_t>(s.list[i]));
            if (prob) *prob = static_cast<float>(m) / static_cast<float>(total);
        }
        at += m;
    }
}

// ------------------------------------------------------- by radix descent

struct Group {  // the tokens of one logit in the order
    uint32_t key;
    u64 above_count, above_mass, mass;  // mass: of one token
};

// The first bin, from the highest, through which the measure exceeds
// `target`.
template <int TH>
__device__ inline void find_bin(Bins<TH> &s, bool by_mass, u64 target) {
    constexpr int kOwn = kBins / TH;
    u64 a = 0, b = 0, ta, tb;
    for (int i = 0; i < kOwn; ++i) {
        const int bin = kBins - 1 - (threadIdx.x * kOwn + i);
        a += s.count[bin], b += s.mass[bin];
    }
    scan_threads<TH>(s, a, b, ta, tb);
    for (int i = 0; i < kOwn; ++i) {
        const int bin = kBins - 1 - (threadIdx.x * kOwn + i);
        const u64 before = by_mass ? b : a, own = by_mass ? s.mass[bin] : s.count[bin];
        if (before <= target && target < before + own) s.found = bin, s.found_count = a, s.found_mass = b;
        a += s.count[bin], b += s.mass[bin];
    }
    __syncthreads();
}

template <int TH, typename T>
__device__ Group find_group(Bins<TH> &s, const T *row, int vocab, float top, float c, bool by_mass, u64 target) {
    Group g = {0, 0, 0, 0};
    const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
    for (int level = 0; level < 3; ++level) {
        const int shift = shifts[level];
        const uint32_t mask = (1u << bits[level]) - 1;
        clear_bins<TH>(s);
        scan_row_singly<TH>(row, 0, vocab, [&](int, float z) {
            const uint32_t key = key_of(z);
            if (level && (key >> (shift + bits[level])) != g.key) return;
            const uint32_t bin = (key >> shift) & mask, m = mass_of(weight(scaled_any(z, top, c)));
            if (!m) return;  // no place falls on it
            atomicAdd(&s.count[bin], 1u);
            atomicAdd(&s.mass[bin], static_cast<u64>(m));
        });
        __syncthreads();
        find_bin<TH>(s, by_mass, target);
        const uint32_t bin = s.found;
        target -= by_mass ? s.found_mass : s.found_count;
        g.above_count += s.found_count;
        g.above_mass += s.found_mass;
        g.key = g.key << bits[level] | bin;
        g.mass = s.mass[bin] / s.count[bin];
        __syncthreads();
    }
    return g;
}

// The index of the n-th token of key `key`.
template <int TH, typename T>
__device__ int find_index(Bins<TH> &s, const T *row, int vocab, uint32_t key, u64 n) {
    uint32_t prefix = 0;
    for (int shift = 22; shift >= 0; shift -= kBinBits) {
        clear_bins<TH>(s);
        scan_row_singly<TH>(row, 0, vocab, [&](int i, float z) {
            const uint32_t r = ~static_cast<uint32_t>(i);  // find_bin counts from the highest bin
            if (key_of(z) != key || (shift < 22 && (r >> (shift + kBinBits)) != prefix)) return;
            atomicAdd(&s.count[(r >> shift) & (kBins - 1)], 1u);
        });
        __syncthreads();
        find_bin<TH>(s, false, n);
        n -= s.found_count;
        prefix = prefix << kBinBits | s.found;
        __syncthreads();
    }
    return static_cast<int>(~prefix);
}

template <int TH, typename T>
__device__ __noinline__ void search_row(Bins<TH> &s, const T *row, int vocab, Settings set, float u, float top,
                                        int32_t *token, float *prob) {
    u64 total = 0, kept = 0, counted = 0, none = 0, t0, t1;
    scan_row_singly<TH>(row, 0, vocab, [&](int, float z) {
        const float w = weight(scaled_any(z, top, set.c));
        const uint32_t m = mass_of(w);
        total += m, counted += m != 0;
        if (!(w < set.min_p)) kept += m;
    });
    scan_threads<TH>(s, total, kept, t0, t1);
    total = t0, kept = t1;
    scan_threads<TH>(s, counted, none, t0, t1);
    if (static_cast<u64>(set.k) < t0) {
        const Group g = find_group<TH>(s, row, vocab, top, set.c, false, set.k - 1);
        total = g.above_mass + (set.k - g.above_count) * g.mass;
    }
    const u64 limit = nucleus(set.top_p, total);
    if (limit < total) {
        const Group g = find_group<TH>(s, row, vocab, top, set.c, true, limit - 1);
        total = g.above_mass + ((limit - 1 - g.above_mass) / g.mass + 1) * g.mass;
    }
    total = min(total, kept);
    const u64 target = place(u, total);
    const Group g = find_group<TH>(s, row, vocab, top, set.c, true, target);
    const int index = find_index<TH>(s, row, vocab, g.key, (target - g.above_mass) / g.mass);
    if (threadIdx.x == 0) {
        *token = index;
        if (prob) *prob = static_cast<float>(g.mass) / static_cast<float>(total);
    }
    __syncthreads();
}

// ------------------------------------------------------------------ steps

template <int TH, typename T>
__device__ inline float slice_max(Bins<TH> &s, const T *row, int lo, int hi) {
    float best = -__builtin_inff();
    bool bad = false;
    scan_row<TH>(row, lo, hi, [&](int, const auto &z) {
#pragma unroll
        for (float v : z) {
            bad |= v != v;
            best = fmaxf(best, v);
        }
    });
    return block_max<TH>(s, best, bad);
}

// Adds [lo, hi) to the histogram; returns this thread's mass of what min-p
// keeps (FLOORS).
template <int TH, bool COUNTS, bool FLOORS, typename T>
__device__ inline u64 add_slice(Bins<TH> &s, const T *row, int lo, int hi, float top, float c, float min_p) {
    u64 kept = 0;
    scan_row<TH>(row, lo, hi, [&](int, const auto &z) {
        constexpr int n = sizeof(z) / sizeof(float);
        uint32_t m[n], bin[n];
#pragma unroll
        for (int j = 0; j < n; ++j) {
            const float t = scaled(z[j], top, c), w = weight(t);
            m[j] = mass_of(w), bin[j] = bin_of(t);
            if (FLOORS) kept += w >= min_p ? m[j] : 0u;
        }
#pragma unroll
        for (int j = 0; j < n; ++j)
            if (m[j]) {
                atomicAdd(&s.mass[bin[j]], static_cast<u64>(m[j]));
                if (COUNTS) atomicAdd(&s.count[bin[j]], 1u);
            }
    });
    return kept;
}
template <int TH, typename T>
__device__ inline u64 slice_histogram(Bins<TH> &s, const T *row, int lo, int hi, float top, const Settings &set,
                                      bool counts) {
    if (counts)
        return set.min_p > 0.0f ? add_slice<TH, true, true>(s, row, lo, hi, top, set.c, set.min_p)
                                : add_slice<TH, true, false>(s, row, lo, hi, top, set.c, set.min_p);
    return set.min_p > 0.0f ? add_slice<TH, false, true>(s, row, lo, hi, top, set.c, set.min_p)
                            : add_slice<TH, false, false>(s, row, lo, hi, top, set.c, set.min_p);
}

// Calls add(key and ~index) for the wanted tokens of [lo, hi).
template <int TH, typename T, typename F>
__device__ inline void slice_collect(const T *row, int lo, int hi, const Wanted &wanted, F add) {
    Wanted w;
#pragma unroll
    for (int i = 0; i < 3; ++i) w.lo[i] = uniform_value(wanted.lo[i]), w.hi[i] = uniform_value(wanted.hi[i]);
    scan_row<TH>(row, lo, hi, [&](int i, const auto &z) {
        constexpr int n = sizeof(z) / sizeof(float);
        bool some = false;
#pragma unroll
        for (int j = 0; j < n; ++j) some |= w.has(z[j]);
        if (!some) return;
#pragma unroll
        for (int j = 0; j < n; ++j)
            if (w.has(z[j])) add(static_cast<u64>(key_of(z[j])) << 32 | ~static_cast<uint32_t>(i + j));
    });
}

// A row's histogram and token, where its largest logit is finite.  ONE_LOOP:
// one form of the histogram's loop for all settings, in fewer registers.
template <bool ONE_LOOP, int TH, int ROOM, typename T>
__device__ inline void sample_row_by_bins(Shared<TH, ROOM> &s, const T *row, int vocab, const Settings &set, float u,
                                          float top, int32_t *token, float *prob) {
    clear_bins<TH>(s);
    u64 kept = 0, none = 0, t0, t1;
    if constexpr (ONE_LOOP)
        kept = add_slice<TH, true, true>(s, row, 0, vocab, top, set.c, set.min_p);
    else
        kept = slice_histogram<TH>(s, row, 0, vocab, top, set, set.k < vocab);
    __syncthreads();
    u64 m[kBins / TH];
    uint32_t c[kBins / TH];
#pragma unroll
    for (int i = 0; i < kBins / TH; ++i)
        m[i] = s.mass[threadIdx.x * (kBins / TH) + i], c[i] = s.count[threadIdx.x * (kBins / TH) + i];
    scan_bins<TH>(s, m, c);
    if (set.min_p > 0.0f) {
        scan_threads<TH>(s, kept, none, t0, t1);
        kept = t0;
    } else {
        kept = s.mass[kBins];
    }
    find_wanted(s, set, u, kept, top);
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    slice_collect<TH>(row, 0, vocab, s.wanted, [&](u64 v) {
        const uint32_t at = atomicAdd(&s.listed, 1u);
        if (at < ROOM) s.list[at] = v;
    });
    __syncthreads();
    const uint32_t listed = s.listed;
    if (listed <= ROOM)
        finish(s, set, u, kept, top, listed, token, prob);
    else
        search_row<TH>(s, row, vocab, set, u, top, token, prob);
}

// -------------------------------------------------------------- block a row
//
// The three steps of a row, one after the other: two blocks of 512 threads a
// compute unit, so that one's reads run beside the other's searches.

template <typename T>
__global__ __launch_bounds__(kThreads, 4) void sample_rows_kernel(const T *__restrict__ logits, int64_t rows, int vocab,
                                                                  int64_t ldk, const float *__restrict__ uniform,
                                                                  SampleSettings settings,
                                                                  int32_t *__restrict__ tokens,
                                                                  float *__restrict__ probs) {
    constexpr int TH = kThreads;
    __shared__ Shared<TH> s;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = logits + r * ldk;
        const float top = slice_max<TH>(s, row, 0, vocab);
        if (!(top > -__builtin_inff())) {
            if (threadIdx.x == 0) {
                tokens[r] = -1;
                if (probs) probs[r] = top != top ? top : 0.0f;
            }
            continue;
        }
        const Settings set = settings_of(settings, r, vocab);
        const float u = uniform_value(uniform[r]);
        float *prob = probs ? probs + r : nullptr;
        if (top == __builtin_inff()) {
            search_row<TH>(s, row, vocab, set, u, top, tokens + r, prob);
            continue;
        }
        sample_row_by_bins<false>(s, row, vocab, set, u, top, tokens + r, prob);
        __syncthreads();
    }
}

// ------------------------------------------------------- bf16: a block a row
//
// 16-bit logits need no bins: a pass counts the tokens of every value, in
// LDS.  The rest follows from the counts, place by place in descending order
// of the values, and a second pass finds the token among those of the drawn
// value.  Three blocks a compute unit, so that one row's loads run beside
// another's sums (the row held in registers, read once, at a block a compute
// unit: 330 us for the 200 of 2048 x 128256; four blocks of 64 registers, 214).

// A dword counts a magnitude, from 2^-55 to 2^9: the positive value in its
// lower half, the negative in its upper.  A count that overflows its half
// shows in the sum of all.  Zeros are counted apart; values of -2^9 and below
// are taken for masks, without counters, where they have no mass beside the
// largest (counted, a mask's atomics meet on one address: 64 x 128256 with 60%
// at -1e4 137 us for 48).
constexpr int kValues = 64 * 128, kGroups = kValues / 64;
constexpr uint32_t kSmallest = 72 << 7, kBeyond = kSmallest + kValues, kInfinity = 0x7f80;
constexpr float kMask = -0x1p9f;
// Places in the order of the values: the positive groups downwards, zero, the
// negative groups; padded.
constexpr int kZeroPlace = kGroups, kPlaces = 512;

typedef Shared<kThreads, 4 * kThreads> BinsBeside;  // three blocks a compute unit fit
struct ValueShared {
    union {
        uint32_t counts[kValues + 64];  // the last: of each lane's tokens elsewhere, unused
        uint32_t matches[kValues];      // a bit per token beside the row's ends: it has the drawn value
        BinsBeside bins;
    };
    u64 mass[kPlaces + 1];  // sums before each place
    uint32_t count[kPlaces + 1];
    u64 wave_a[kThreads / 64], wave_b[kThreads / 64], in_head, in_tail;
    uint32_t highest, lowest, sum, zeros, outside, odd, bits, nth;
    float prob;
};

// The counted values of a group, in their order: positive ones downwards,
// negative ones upwards.
struct Value {
    uint32_t bits, count;
};
__device__ inline Value value_at(const ValueShared &s, int place) {
    const int lane = threadIdx.x & 63;
    if (place == kZeroPlace) return {0, lane == 0 ? s.zeros : 0};
    const bool negative = place > kZeroPlace;
    const uint32_t i = negative ? (place - kZeroPlace - 1) * 64 + lane : (kGroups - 1 - place) * 64 + 63 - lane;
    const uint32_t c = s.counts[i];
    return negative ? Value{0x8000u | (i + kSmallest), c >> 16} : Value{i + kSmallest, c & 0xffff};
}
__device__ inline float logit_of_bits(uint32_t bits) { return __uint_as_float(bits << 16); }

__device__ inline u64 last_lane(u64 v) {
    return static_cast<u64>(__builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), 63)) << 32 |
           static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(v), 63));
}

// The place of the n-th set bit.
__device__ inline int nth_bit(u64 v, int n) {
    for (; n; --n) v &= v - 1;
    return __ffsll(v) - 1;
}

// A value at a given count or mass of the order: one token's mass, and what
// is before the value.
struct Found {
    uint32_t bits, m;
    u64 count_before, mass_before;
};

// The value at x below the total, by a wave; before: s.count or s.mass.
template <typename U>
__device__ inline Found find_value(const ValueShared &s, const U *before, float top, float c, U x) {
    static_assert(kPlaces == 64 * 8, "two steps");
    const int lane = threadIdx.x & 63;
    const int part = __ffsll(static_cast<u64>(__ballot(before[8 * lane] <= x && x < before[8 * lane + 8]))) - 1;
    const int at = 8 * part + (lane & 7);
    const int place =
        8 * part + ((__ffsll(static_cast<u64>(__ballot(before[at] <= x && x < before[at + 1]))) - 1) & 7);
    const Value v = value_at(s, place);
    const uint32_t m = v.count ? mass_of(weight(scaled(logit_of_bits(v.bits), top, c))) : 0;
    const u64 gc = m ? v.count : 0, gm = static_cast<u64>(m) * v.count;
    const u64 ic = s.count[place] + wave_scan(gc), im = s.mass[place] + wave_scan(gm);
    const int l = __ffsll(static_cast<u64>(__ballot(x < (sizeof(U) == 8 ? im : ic)))) - 1;
    return {static_cast<uint32_t>(__shfl(v.bits, l)), static_cast<uint32_t>(__shfl(m, l)), __shfl(ic - gc, l),
            __shfl(im - gm, l)};
}

// A row that the counts cannot tell, by bins: four reads of it in all (2048 x
// 128256 with 60% at -100: 783 us, of which half are counts on one address;
// by radix descent 1565; with -inf for -100, counted, 230).  A function of its
// own keeps its registers out of the counting loops.
__device__ __noinline__ void sample_row_apart(BinsBeside &s, const uint16_t *row, int vocab, Settings set, float u,
                                              int32_t *token, float *prob) {
    const float top = slice_max<kThreads>(s, row, 0, vocab);
    if (!(top > -__builtin_inff())) {
        if (threadIdx.x == 0) {
            *token = -1;
            if (prob) *prob = top != top ? top : 0.0f;
        }
    } else if (top == __builtin_inff()) {
        search_row<kThreads>(s, row, vocab, set, u, top, token, prob);
    } else {
        sample_row_by_bins<true>(s, row, vocab, set, u, top, token, prob);
    }
}

__global__ __launch_bounds__(kThreads, 6) void sample_values_kernel(const uint16_t *__restrict__ logits, int64_t rows,
                                                                    int vocab, int64_t ldk,
                                                                    const float *__restrict__ uniform,
                                                                    SampleSettings settings,
                                                                    int32_t *__restrict__ tokens,
                                                                    float *__restrict__ probs) {
    constexpr int TH = kThreads, kAhead = 4;
    typedef uint16_t Half2 __attribute__((ext_vector_type(2)));
    __shared__ ValueShared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const uint16_t *row = logits + r * ldk;
        const int head = min(vocab, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / 2);
        const int vectors = (vocab - head) / 8, tail = head + vectors * 8;
        const uint4 *src = reinterpret_cast<const uint4 *>(row + head);
        const int edge = tid < head ? tid : tail + tid - head;  // one of the few tokens beside the vectors
        const uint32_t edge_bits = edge < vocab ? row[edge] : 0;
        const Settings set = settings_of(settings, r, vocab);
        const float u = uniform_value(uniform[r]);
        for (int i = tid; i < kValues / 4; i += TH)
            reinterpret_cast<uint4 *>(s.counts)[i] = make_uint4(0, 0, 0, 0);
        if (tid == 0) s.highest = s.sum = s.zeros = s.outside = s.odd = 0, s.lowest = kValues;
        __syncthreads();

        uint32_t outside = 0, zeros = 0, odd = 0;
        auto classify = [&](uint32_t bits) {  // of a value that has no counter
            const uint32_t magnitude = bits & 0x7fff;
            if (magnitude - kSmallest < static_cast<uint32_t>(kValues)) return;
            ++outside;
            if (magnitude == 0)
                ++zeros;
            else if (!(bits > 0x8000u && magnitude >= kBeyond && magnitude <= kInfinity))
                odd = 1;
        };
        auto each = [&](uint4 v) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t h = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffff;
                const uint32_t i = (h & 0x7fff) - kSmallest;
                most = max(most, i);
                atomicAdd(&s.counts[min(i, static_cast<uint32_t>(kValues + lane))], 1u + (h >> 15) * 0xffffu);
            }
            if (most >= static_cast<uint32_t>(kValues)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) classify(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffff);
            }
        };
        int at = tid;
        for (; at + (kAhead - 1) * TH < vectors; at += kAhead * TH) {
            uint4 v[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) v[a] = src[at + a * TH];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) each(v[a]);
        }
        for (; at < vectors; at += TH) each(src[at]);
        if (edge < vocab) {
            const uint32_t i = (edge_bits & 0x7fff) - kSmallest;
            if (i < static_cast<uint32_t>(kValues)) atomicAdd(&s.counts[i], 1u + (edge_bits >> 15) * 0xffffu);
            classify(edge_bits);
        }
        if (outside) atomicAdd(&s.outside, outside);
        if (zeros) atomicAdd(&s.zeros, zeros);
        if (odd) s.odd = 1;
        __syncthreads();

        // The largest value, and whether every token is accounted for.  The
        // waves take groups in turn; which of them hold a token: a bit each.
        uint32_t sum = 0, some = 0, highest = 0, lowest = kValues;  // highest: plus 1
#pragma unroll 4
        for (int i = 0; i < kGroups / (TH / 64); ++i) {
            const uint32_t magnitude = (i * (TH / 64) + wave) * 64 + lane, c = s.counts[magnitude];
            if (!__any(c != 0)) continue;
            some |= 1u << i;
            sum += (c & 0xffff) + (c >> 16);
            if (c & 0xffff) highest = magnitude + 1;
            if (c >> 16) lowest = min(lowest, magnitude);
        }
        if (sum) atomicAdd(&s.sum, sum);
        if (highest) atomicMax(&s.highest, highest);
        if (lowest < kValues) atomicMin(&s.lowest, lowest);
        for (int i = tid; i <= kPlaces; i += TH) s.mass[i] = 0, s.count[i] = 0;
        __syncthreads();
        const uint32_t top_bits = s.highest ? s.highest - 1 + kSmallest : s.zeros ? 0 : 0x8000u | (s.lowest + kSmallest);
        const float top = uniform_value(logit_of_bits(top_bits));
        float *prob = probs ? probs + r : nullptr;
        // Rows that the counts cannot tell: over 65535 tokens of a value,
        // values without a counter, none with one, or masks that may have mass.
        if (__builtin_amdgcn_readfirstlane(s.sum + s.outside != static_cast<uint32_t>(vocab) || s.odd ||
                                           s.sum + s.zeros == 0 ||
                                           (s.outside > s.zeros && !(scaled(kMask, top, set.c) <= -33.0f)))) {
            __syncthreads();
            sample_row_apart(s.bins, row, vocab, set, u, tokens + r, prob);
            __syncthreads();
            continue;
        }

        // The places' masses and counts, then the sums before them.
        u64 kept = 0;
        auto add_place = [&](int place) {
            const Value x = value_at(s, place);
            if (!__any(x.count != 0)) return;
            const float w = weight(scaled(logit_of_bits(x.bits), top, set.c));
            const uint32_t one = x.count ? mass_of(w) : 0;
            const u64 m = static_cast<u64>(one) * x.count;
            if (!(w < set.min_p)) kept += m;
            const u64 mass = last_lane(wave_scan(m)), counted = last_lane(wave_scan(one ? x.count : 0));
            if (lane == 0) s.mass[place] = mass, s.count[place] = static_cast<uint32_t>(counted);
        };
        for (uint32_t left = __builtin_amdgcn_readfirstlane(some); left; left &= left - 1) {
            const int group = (__ffs(left) - 1) * (TH / 64) + wave;
            add_place(kGroups - 1 - group);
            add_place(kZeroPlace + 1 + group);
        }
        if (wave == 0) add_place(kZeroPlace);
        __syncthreads();
        static_assert(kPlaces == TH, "a place each");
        u64 mass = s.mass[tid], counted = s.count[tid], none = 0, all, all_counted, t0;
        scan_threads<TH>(s.wave_a, s.wave_b, mass, counted, all, all_counted);
        s.mass[tid] = mass, s.count[tid] = static_cast<uint32_t>(counted);
        if (tid == 0) s.mass[kPlaces] = all, s.count[kPlaces] = static_cast<uint32_t>(all_counted);
        scan_threads<TH>(s.wave_a, s.wave_b, kept, none, t0, none);
        kept = t0;
        if (wave == 0) {
            u64 total = all;
            if (static_cast<u64>(set.k) < all_counted) {
                const Found f = find_value<uint32_t>(s, s.count, top, set.c, set.k - 1);
                total = f.mass_before + (set.k - f.count_before) * f.m;
            }
            const u64 limit = nucleus(set.top_p, total);
            if (limit < total) {
                const Found f = find_value<u64>(s, s.mass, top, set.c, limit - 1);
                total = f.mass_before + ((limit - 1 - f.mass_before) / f.m + 1) * f.m;
            }
            total = min(total, kept);
            const u64 target = place(u, total);
            const Found f = find_value<u64>(s, s.mass, top, set.c, target);
            if (lane == 0) {
                s.bits = f.bits;
                s.nth = static_cast<uint32_t>((target - f.mass_before) / f.m);
                if (prob) *prob = static_cast<float>(f.m) / static_cast<float>(total);
            }
        }
        __syncthreads();

        // The n-th token of the drawn value: a bit for each token.
        const int words = (vectors + 3) / 4;
        for (int i = tid; i < words; i += TH) s.matches[i] = 0;
        __syncthreads();
        const uint32_t bits = s.bits, both = bits == 0 ? 0x7fffu : 0xffffu;  // the zeros are one value
        const uint32_t mask = both | both << 16, want = (bits & both) * 0x10001u;
        auto match = [&](int i, uint4 v) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t differ[4], all_differ = 0xffffffffu;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t x = (w[e] & mask) ^ want;
                differ[e] = __builtin_bit_cast(
                    uint32_t, __builtin_elementwise_min(__builtin_bit_cast(Half2, x), Half2{1, 1}));
                all_differ &= differ[e];
            }
            if (all_differ == 0x10001u) return;
            uint32_t found = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) found |= ((~differ[e] & 1) | (~differ[e] >> 15 & 2)) << (2 * e);
            reinterpret_cast<uint8_t *>(s.matches)[i] = static_cast<uint8_t>(found);
        };
        at = tid;
        for (; at + (kAhead - 1) * TH < vectors; at += kAhead * TH) {
            uint4 v[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) v[a] = src[at + a * TH];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) match(at + a * TH, v[a]);
        }
        for (; at < vectors; at += TH) match(at, src[at]);
        if (wave == 0) {
            const bool hit = edge < vocab && ((edge_bits ^ bits) & both) == 0;
            const u64 in_head = __ballot(hit && tid < head), in_tail = __ballot(hit && tid >= head);
            if (lane == 0) s.in_head = in_head, s.in_tail = in_tail;
        }
        __syncthreads();
        const int own = (words + TH - 1) / TH, from = min(tid * own, words), to = min(from + own, words);
        u64 before = 0, t1;
        none = 0;
        for (int i = from; i < to; ++i) before += __popc(s.matches[i]);
        const u64 mine = before;
        scan_threads<TH>(s.wave_a, s.wave_b, before, none, t0, t1);
        const u64 nth = s.nth, heads = __popcll(s.in_head);
        if (tid == 0) {
            if (nth < heads) tokens[r] = nth_bit(s.in_head, static_cast<int>(nth));
            if (nth >= heads + t0) tokens[r] = tail - head + nth_bit(s.in_tail, static_cast<int>(nth - heads - t0));
        }
        if (nth >= heads && nth - heads - before < mine) {
            u64 left = nth - heads - before;
            for (int i = from; i < to; ++i) {
                const uint32_t have = __popc(s.matches[i]);
                if (left < have) {
                    tokens[r] = head + i * 32 + nth_bit(s.matches[i], static_cast<int>(left));
                    break;
                }
                left -= have;
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------- several blocks a row
//
// Three kernels: the slices' maxima; the row's histogram, of the slices'; the
// wanted tokens of each slice, and from all of them the row's.  Bound by
// latency: 1 x 128256 f32 takes 3, 5 and 10 us, the last one's for reading the
// histogram and its sums (2.3), the search of the bins (2.2), the slice (1.2),
// the meeting (1.7) and the token (1.3).

struct RowSpace {
    u64 mass[kBins], list[kRoom], kept;
    uint32_t count[kBins], listed, done;
    float top[kMostSlices];
};

// The row's largest logit, NaN if one is; every wave by itself.
__device__ inline float row_top(const RowSpace &space, int slices) {
    static_assert(kMostSlices <= 64, "a lane each");
    const int lane = threadIdx.x & 63;
    float best = lane < slices ? space.top[lane] : -__builtin_inff();
    const bool bad = __any(best != best);
    for (int o = 32; o; o >>= 1) best = fmaxf(best, __shfl_xor(best, o));
    return uniform_value(bad ? __builtin_nanf("") : best);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void slice_max_kernel(const T *__restrict__ logits, int vocab, int64_t ldk,
                                                                  int slice, RowSpace *__restrict__ spaces) {
    __shared__ Shared<kThreads> s;
    const int64_t r = blockIdx.y;
    RowSpace &space = spaces[r];
    const int lo = blockIdx.x * slice, hi = min(vocab, lo + slice);
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < kBins; i += gridDim.x * kThreads)
        space.mass[i] = 0, space.count[i] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) space.kept = 0, space.listed = 0, space.done = 0;
    const float top = slice_max<kThreads>(s, logits + r * ldk, lo, hi);
    if (threadIdx.x == 0) space.top[blockIdx.x] = top;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void slice_histogram_kernel(const T *__restrict__ logits, int vocab,
                                                                        int64_t ldk, int slice,
                                                                        SampleSettings settings,
                                                                        RowSpace *__restrict__ spaces) {
    constexpr int TH = kThreads;
    __shared__ Shared<TH> s;
    const int64_t r = blockIdx.y;
    RowSpace &space = spaces[r];
    const Settings set = settings_of(settings, r, vocab);
    const float top = row_top(space, gridDim.x);
    if (!(top > -__builtin_inff() && top < __builtin_inff())) return;
    const int lo = blockIdx.x * slice, hi = min(vocab, lo + slice);
    clear_bins<TH>(s);
    u64 kept = slice_histogram<TH>(s, logits + r * ldk, lo, hi, top, set, set.k < vocab), none = 0, t0, t1;
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += TH) {
        if (s.mass[i]) atomicAdd(&space.mass[i], s.mass[i]);
        if (s.count[i]) atomicAdd(&space.count[i], s.count[i]);
    }
    if (set.min_p > 0.0f) {
        scan_threads<TH>(s, kept, none, t0, t1);
        if (threadIdx.x == 0 && t0) atomicAdd(&space.kept, t0);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads, 4) void slice_token_kernel(const T *__restrict__ logits, int vocab,
                                                                    int64_t ldk, int slice,
                                                                    const float *__restrict__ uniform,
                                                                    SampleSettings settings,
                                                                    RowSpace *__restrict__ spaces,
                                                                    int32_t *__restrict__ tokens,
                                                                    float *__restrict__ probs) {
    constexpr int TH = kThreads;
    __shared__ Shared<TH> s;
    const int64_t r = blockIdx.y;
    const T *row = logits + r * ldk;
    RowSpace &space = spaces[r];
    const Settings set = settings_of(settings, r, vocab);
    const float u = uniform_value(uniform[r]);
    float *prob = probs ? probs + r : nullptr;
    const u64 floored = space.kept;
    u64 m[kBins / TH];
    uint32_t c[kBins / TH];
#pragma unroll
    for (int i = 0; i < kBins / TH; ++i)
        m[i] = space.mass[threadIdx.x * (kBins / TH) + i], c[i] = space.count[threadIdx.x * (kBins / TH) + i];
    const float top = row_top(space, gridDim.x);
    if (!(top > -__builtin_inff())) {
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            tokens[r] = -1;
            if (probs) probs[r] = top != top ? top : 0.0f;
        }
        return;
    }
    if (top == __builtin_inff()) {
        if (blockIdx.x == 0) search_row<TH>(s, row, vocab, set, u, top, tokens + r, prob);
        return;
    }
    scan_bins<TH>(s, m, c);
    const u64 kept = set.min_p > 0.0f ? floored : s.mass[kBins];
    find_wanted(s, set, u, kept, top);
    __syncthreads();
    const int lo = blockIdx.x * slice, hi = min(vocab, lo + slice);
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    slice_collect<TH>(row, lo, hi, s.wanted, [&](u64 v) {
        const uint32_t at = atomicAdd(&s.listed, 1u);
        if (at < kRoom) s.list[at] = v;
    });
    __syncthreads();
    // One place for the block's, found at once: a place each costs a round
    // trip to memory each time (22 us of 64 x 50257 for 18).
    const uint32_t own = s.listed;
    if (threadIdx.x == 0) s.first = own ? atomicAdd(&space.listed, own) : 0;
    __syncthreads();
    const uint32_t base = s.first;
    for (uint32_t i = threadIdx.x; i < min(own, static_cast<uint32_t>(kRoom)) && base + i < kRoom; i += TH)
        __hip_atomic_store(&space.list[base + i], s.list[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // The last of the row's blocks finds the token.  The tokens are stored
    // and read at the device's scope, past the dies' own L2s, and a wave
    // counts its block only when its stores are acknowledged; a fence would
    // write back and invalidate whole L2s (25 us of a 64-row call).
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);  // vmcnt(0)
    __syncthreads();
    if (threadIdx.x == 0) s.last = atomicAdd(&space.done, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!s.last) return;
    const uint32_t listed = __hip_atomic_load(&space.listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (listed <= kRoom) {
        for (int i = threadIdx.x; i < static_cast<int>(listed); i += TH)
            s.list[i] = __hip_atomic_load(&space.list[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        finish(s, set, u, kept, top, listed, tokens + r, prob);
    } else {
        search_row<TH>(s, row, vocab, set, u, top, tokens + r, prob);
    }
}

// Blocks per row; 1: a block per row and one kernel.  Three kernels and the
// blocks' meeting cost 6 us over one, and more the more blocks there are; a
// block reads 3000 tokens a us.  So rows are split where that takes 16384
// tokens from a block, and 128 more for every row up to 64.  Split / whole in
// us, f32, one set of logits again and again, top-k 50 and top-p 0.9, top-p
// 0.95: 1 x 16384: 15 / 13, 16 / 14; 1 x
// 32000: 15 / 18, 16 / 18; 1 x 128256: 16 / 48, 25 / 60; 8 x 24000: 16 / 17, 19 /
// 20; 32 x 32000: 20 / 19, 23 / 25; 64 x 24000: 22 / 17, 24 / 22; 64 x 32000: 23
// / 19, 26 / 26; 64 x 50257: 24 / 25, 31 / 36; 85 x 32000: 23 / 19, 27 / 26; 100 x
// 50257: 26 / 25, 36 / 37; 128 x 40000: 27 / 22, 31 / 30; 128 x 50257: 29 / 32, 37
// / 40; 128 x 128256: 52 / 68, 68 / 90.
int slices_of(int64_t rows, int32_t vocab) {
    const int64_t slices = std::min<int64_t>({256 / rows, vocab / 4096, kMostSlices});
    const int64_t pays = 16384 + 128 * std::min<int64_t>(rows, 64);
    return slices > 1 && vocab - vocab / slices >= pays ? static_cast<int>(slices) : 1;
}

// Whether a row's values are counted, with a block a row.  That costs some
// 17 us whatever the length, the histogram of weights 10 and more per token,
// most where much lies near the cuts (us, histogram / counts, of top-k 50 and
// top-p 0.9; top-p 0.95): 128 x 16384: 16 / 20, 21 / 20; 128 x 32000: 21 / 24,
// 28 / 23; 64 x 50257: 27 / 24, 37 / 24; 2048 x 16384: 70 / 83, 83 / 82;
// 2048 x 32000: 107 / 96, 126 / 94; 2048 x 128256: 321 / 200.  Few rows are
// split instead: 32 x 128256: 27 / 33, 44 / 33; 16 x 32000: 20 / 23, 25 / 22;
// 1 x 128256: 17 / 32.  The upper limit is that of the matches' bits.
bool by_values(bool bf16, int64_t rows, int32_t vocab) {
    return bf16 && rows >= 32 && vocab >= 28 * 1024 && vocab <= 32 * kValues;
}

template <typename T>
bool launch(const T *logits, int64_t rows, int32_t vocab, int64_t ldk, const float *uniform,
            const SampleSettings &settings, int32_t *tokens, float *probs, void *workspace, hipStream_t stream) {
    if constexpr (sizeof(T) == 2)
        if (by_values(true, rows, vocab)) {
            sample_values_kernel<<<static_cast<unsigned>(std::min<int64_t>(rows, 768)), kThreads, 0, stream>>>(
                logits, rows, vocab, ldk, uniform, settings, tokens, probs);
            return hipGetLastError() == hipSuccess;
        }
    const int slices = slices_of(rows, vocab);
    if (slices == 1) {
        sample_rows_kernel<<<static_cast<unsigned>(std::min<int64_t>(rows, 512)), kThreads, 0, stream>>>(
            logits, rows, vocab, ldk, uniform, settings, tokens, probs);
        return hipGetLastError() == hipSuccess;
    }
    const int slice = ((vocab + slices - 1) / slices + 7) / 8 * 8;  // whole vectors
    const dim3 grid((vocab + slice - 1) / slice, static_cast<unsigned>(rows));
    auto *spaces = static_cast<RowSpace *>(workspace);
    slice_max_kernel<<<grid, kThreads, 0, stream>>>(logits, vocab, ldk, slice, spaces);
    slice_histogram_kernel<<<grid, kThreads, 0, stream>>>(logits, vocab, ldk, slice, settings, spaces);
    slice_token_kernel<<<grid, kThreads, 0, stream>>>(logits, vocab, ldk, slice, uniform, settings, spaces, tokens,
                                                           probs);
    return hipGetLastError() == hipSuccess;
}

}  // namespace

int64_t sample_workspace_bytes(bool bf16, int64_t rows, int32_t vocab) {
    if (rows <= 0 || by_values(bf16, rows, vocab) || slices_of(rows, vocab) == 1) return 0;
    return rows * static_cast<int64_t>(sizeof(RowSpace));
}

bool sample_launch(const void *logits, bool bf16, int64_t rows, int32_t vocab, int64_t ldk, const float *uniform,
                   const SampleSettings &settings, int32_t *tokens, float *probs, void *workspace,
                   hipStream_t stream) {
    if (rows == 0) return true;
    return bf16 ? launch(static_cast<const uint16_t *>(logits), rows, vocab, ldk, uniform, settings, tokens, probs,
                         workspace, stream)
                : launch(static_cast<const float *>(logits), rows, vocab, ldk, uniform, settings, tokens, probs,
                         workspace, stream);
}

}  // namespace fgd
