// attend.hip -- attention over a paged cache in microscaled 4-bit floating
// point (layout: cache.hpp).
//
// A query head's row: t_j = scale log2(e) q.k_j over the keys j that it sees,
// o = sum_j 2^(t_j - m) v_j / sum_j 2^(t_j - m) with m their running maximum,
// in one pass over the cache.  The keys' and values' 4-bit numbers are exact
// in bf16, so both products run on the bf16 matrix instruction without
// rounding an operand: queries as they are (bf16) or as the sum of three bf16
// numbers (f32), and the weights 2^(t_j - m) as a sum of two (bf16 outputs:
// 2^-17 of a weight is left out) or three.  Sums are float32.
//
// The scores are computed transposed, S^T = K Q^T, in tiles of 16 keys x 16
// rows: a lane then holds four keys of one row, which is what the second
// product O^T = V^T P^T takes as its right operand, so that no weight crosses
// a lane.  The rows are the queries of all heads that share a key head.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.hpp"

namespace fgd {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kTile = 32;  // waves of a block; keys of a wave's step
constexpr float kLog2e = 1.44269504f;
// The running maximum is moved when a score passes it by this much (in
// powers of two): weights stay below 2^8, and most steps spare the rescaling.
constexpr float kSlack = 8.0f;

template <typename T>
struct Parts;  // how many bf16 numbers stand for a query's element and for a weight
template <>
struct Parts<uint16_t> {
    static constexpr int q = 1, p = 2;
};
template <>
struct Parts<float> {
    static constexpr int q = 3, p = 3;
};

__device__ inline uint32_t pack_bf16(float a, float b) {
    bf16x2 v;
    v[0] = static_cast<__bf16>(a);
    v[1] = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint32_t, v);
}
__device__ inline float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float high_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The leading 8 bits of a, a bf16 number in the upper half of a word; a keeps
// the rest, exactly: three such parts are all of a float32.  What is not
// finite is left whole.
__device__ inline uint32_t take_top(float &a) {
    const uint32_t w = __float_as_uint(a);
    const bool finite = (w & 0x7f800000u) != 0x7f800000u;
    const uint32_t top = (finite || (w & 0x7fffffu) == 0 ? w : w | 0x400000u) & 0xffff0000u;
    a = finite ? a - __uint_as_float(top) : 0.0f;
    return top;
}

template <int kSel>
__device__ inline uint32_t fp4_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, kSel));
}

__device__ inline f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

// Byte i of w as the float32 2^(byte - 127).
__device__ inline float scale_of(uint32_t w, int i) {
    return __uint_as_float((i < 3 ? w << (23 - 8 * i) : w >> 1) & 0x7f800000u);
}

// The blocks whose scales a lane's quarter of a key needs.
template <int NB>
constexpr int kKeyScales = NB == 7 ? 3 : NB % 4 == 0 ? NB / 4 : NB < 3 ? 1 : 2;

// 32 keys and values as they lie in the cache: a lane's part.
template <int NB>
struct Raw {
    uint32_t k[2][NB], v[2][NB], vs[2][NB];
    uint8_t ks[2][kKeyScales<NB>];
};

template <int N>
struct __attribute__((packed, aligned(4))) Words {
    uint32_t w[N];
};

template <int NB>
__device__ inline void load_keys(const uint8_t *g, int lane, int u, Raw<NB> &r) {
    const auto k = *reinterpret_cast<const Words<NB> *>(g + lane * 4 * NB);
#pragma unroll
    for (int i = 0; i < NB; ++i) r.k[u][i] = k.w[i];
    const uint8_t *ks = g + 16 * 32 * NB + (lane & 15) * NB;
    const int first = (lane >> 4) * NB / 4;
#pragma unroll
    for (int i = 0; i < kKeyScales<NB>; ++i) r.ks[u][i] = ks[min(first + i, NB - 1)];
}

template <int NB>
__device__ inline void load_values(const uint8_t *g, int lane, int u, Raw<NB> &r) {
    constexpr int D = 32 * NB;
    const auto v = *reinterpret_cast<const Words<NB> *>(g + 8 * D + lane * 4 * NB);
    const auto s = *reinterpret_cast<const Words<NB> *>(g + 16 * D + D / 2 + (lane >> 4) * 4 * NB);
#pragma unroll
    for (int i = 0; i < NB; ++i) r.v[u][i] = v.w[i], r.vs[u][i] = s.w[i];
}

// A wave's state: R tiles of 16 rows.
template <typename T, int NB, int R>
struct Rows {
    static constexpr int D = 32 * NB, kQ = Parts<T>::q, kP = Parts<T>::p;
    u32x4 q[R][kQ][NB];      // the right operand of the scores: row l & 15, elements (l >> 4) D/4 + 8 s ...
    f32x4 o[R][NB][2];       // O^T: row l & 15, elements 32 b + 8 (l >> 4) + 2 i + (0 or 1)
    float m[R], sum[R];      // the maximum that weights refer to, in scores (not scaled); the lane's part of their sum
    int lo[R], hi[R];        // the keys that the lane's row sees
    uint32_t poison[R];      // blocks in which the row sees a NaN value

    __device__ void clear() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -INFINITY, sum[r] = 0, poison[r] = 0;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[r][b][0] = o[r][b][1] = f32x4{0, 0, 0, 0};
        }
    }

    __device__ void load_query(int r, const T *src, int lane, bool real) {
#pragma unroll
        for (int s = 0; s < NB; ++s) {
            struct __attribute__((packed, aligned(sizeof(T)))) Eight {
                T e[8];
            } x;
            if (real)
                x = *reinterpret_cast<const Eight *>(src + (lane >> 4) * (D / 4) + 8 * s);
            else
                __builtin_memset(&x, 0, sizeof(x));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) {
                    q[r][0][s][i] = x.e[2 * i] | static_cast<uint32_t>(x.e[2 * i + 1]) << 16;
                } else {
                    float a = x.e[2 * i], b = x.e[2 * i + 1];
#pragma unroll
                    for (int j = 0; j < kQ; ++j) q[r][j][s][i] = take_top(a) >> 16 | take_top(b);
                }
            }
        }
    }

    // The scores of 32 keys with all rows.
    __device__ void scores(const Raw<NB> &x, int lane, f32x4 (&s)[R][2]) const {
        const int h = lane >> 4;
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][0] = s[r][1] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float ks[kKeyScales<NB>];
#pragma unroll
            for (int i = 0; i < kKeyScales<NB>; ++i) ks[i] = __uint_as_float(static_cast<uint32_t>(x.ks[u][i]) << 23);
#pragma unroll
            for (int p = 0; p < NB; ++p) {
                float scale = ks[0];
                if constexpr (NB % 4 == 0)
                    scale = ks[p / 4];
                else if constexpr (kKeyScales<NB> > 1) {
                    const int i = (h * NB + p) / 4 - h * NB / 4;
                    scale = i == 0 ? ks[0] : i == 1 ? ks[1] : ks[kKeyScales<NB> - 1];
                }
                const u32x4 a = {fp4_pair<0>(x.k[u][p], scale), fp4_pair<1>(x.k[u][p], scale),
                                 fp4_pair<2>(x.k[u][p], scale), fp4_pair<3>(x.k[u][p], scale)};
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = kQ - 1; j >= 0; --j) s[r][u] = mfma(a, q[r][j][p], s[r][u]);
            }
        }
    }

    // Scores of keys that a row does not see become -inf.  A weight of 0 does
    // not take away a NaN or an infinity (bytes above 252, which no finite
    // block has): such values are taken out as well and kept in mind for the
    // rows that see them.
    __device__ void mask(Raw<NB> &x, int first, int lane, f32x4 (&s)[R][2]) {
        const int h = lane >> 4;
        uint32_t seen[R];  // bit 4 u + i: the lane's row sees key first + 16 u + 4 h + i
#pragma unroll
        for (int r = 0; r < R; ++r) {
            seen[r] = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = first + 16 * u + 4 * h + i;
                    const bool v = key >= lo[r] && key < hi[r];
                    seen[r] |= static_cast<uint32_t>(v) << (4 * u + i);
                    if (!v) s[r][u][i] = -INFINITY;
                }
        }
        uint32_t bad = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t w = x.vs[u][b];
                bad |= ((w & 0x7f7f7f7fu) + 0x03030303u) & w & 0x80808080u;
            }
        if (!__any(bad != 0)) return;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if ((x.vs[u][b] >> (8 * i) & 255) > 252) {
                        x.vs[u][b] &= ~(255u << (8 * i));
#pragma unroll
                        for (int r = 0; r < R; ++r) poison[r] |= (seen[r] >> (4 * u + i) & 1) << b;
                    }
    }

    // Scores to weights, as the parts that the second product takes; c =
    // scale log2(e).
    __device__ void weights(const f32x4 (&s)[R][2], float c, u32x4 (&p)[R][kP]) {
        bool move = false;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float top = s[r][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, s[r][i >> 2][i & 3]);
            move |= (top - m[r]) * c > kSlack;  // infinite at first; false for two infinities
        }
        if (__any(move)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float top = s[r][0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, s[r][i >> 2][i & 3]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(m[r], fmaxf(top, __shfl_xor(top, 32)));
                const float f = top == m[r] ? 1.0f : __builtin_amdgcn_exp2f((m[r] - top) * c);
                m[r] = top;
                sum[r] *= f;
#pragma unroll
                for (int b = 0; b < NB; ++b) o[r][b][0] *= f, o[r][b][1] *= f;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            // s - m before the factor: the largest weight is 1 exactly, and
            // large scores lose nothing (m c would be rounded by itself).
            const float base = m[r] == -INFINITY ? 0.0f : m[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float a = __builtin_amdgcn_exp2f((s[r][i >> 1][2 * (i & 1)] - base) * c),
                      b = __builtin_amdgcn_exp2f((s[r][i >> 1][2 * (i & 1) + 1] - base) * c);
                sum[r] += a + b;
#pragma unroll
                for (int j = 0; j < kP; ++j) {
                    const uint32_t w = pack_bf16(a, b);
                    p[r][j][i] = w;
                    if (j + 1 < kP) a -= low_of(w), b -= high_of(w);
                }
            }
        }
    }

    __device__ void add(const Raw<NB> &x, const u32x4 (&p)[R][kP]) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            uint32_t w[8];  // (element 2 n, element 2 n + 1) of the lane's keys
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                w[4 * u] = fp4_pair<0>(x.v[u][b], scale_of(x.vs[u][b], 0));
                w[4 * u + 1] = fp4_pair<1>(x.v[u][b], scale_of(x.vs[u][b], 1));
                w[4 * u + 2] = fp4_pair<2>(x.v[u][b], scale_of(x.vs[u][b], 2));
                w[4 * u + 3] = fp4_pair<3>(x.v[u][b], scale_of(x.vs[u][b], 3));
            }
            u32x4 even, odd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                even[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
                odd[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = kP - 1; j >= 0; --j) {
                    o[r][b][0] = mfma(even, p[r][j], o[r][b][0]);
                    o[r][b][1] = mfma(odd, p[r][j], o[r][b][1]);
                }
            // Else the scheduler converts all blocks first, in twice the registers.
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

struct Span {  // a sequence's queries and keys
    int64_t first;
    int n, length;
    bool bad;
};

// Device values are held within the arrays' sizes: a length beyond the
// sequence's table makes its rows NaN.
__device__ inline Span span_of(const AttendArgs &a, int b) {
    Span s;
    int64_t end;
    if (a.starts) {
        s.first = min(max(static_cast<int64_t>(a.starts[b]), INT64_C(0)), a.tokens);
        end = min(max(static_cast<int64_t>(a.starts[b + 1]), s.first), a.tokens);
    } else {
        s.first = b, end = b + 1;
    }
    s.n = static_cast<int>(end - s.first);
    const int64_t most = static_cast<int64_t>(a.width) << a.cache.page_shift;
    const int length = max(a.lengths[b], 0);
    s.bad = length > most;
    s.length = s.bad ? static_cast<int>(most) : length;
    return s;
}

// A lane's eight elements of one block and row, scaled.
template <typename T>
__device__ inline void store_eight(T *dst, const float (&v)[8]) {
    struct __attribute__((packed, aligned(sizeof(T)))) Eight {
        T e[8];
    } x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) {
            x.e[i] = v[i];
        } else {
            x.e[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[i]));
        }
    }
    *reinterpret_cast<Eight *>(dst) = x;
}

// The output's row (token, head), or a split's part of it.
struct Place {
    int64_t token;
    int head;
};

// kShared: the block's four waves share 16 R rows and split their keys
// between them (and the grid splits them again, where splits > 1); else each
// wave has rows of its own.
// Waves of a SIMD that the registers are kept few enough for: a row tile's
// sums and queries, a step's codes and scales, and about 70 more.
template <typename T, int NB, int R>
constexpr int kRegisters = R * NB * (8 + 4 * Parts<T>::q) + 6 * NB + 60 + 10 * R;
template <typename T, int NB, int R>
constexpr int kOccupancy = kRegisters<T, NB, R> <= 110   ? 4
                           : kRegisters<T, NB, R> <= 150 ? 3
                           : kRegisters<T, NB, R> <= 235 ? 2
                                                         : 1;

template <typename T, int NB, int R, bool kShared>
__global__ __launch_bounds__(256, (kOccupancy<T, NB, R>)) void attend_kernel(AttendArgs a, int splits, float *parts, float2 *stats) {
    constexpr int D = 32 * NB;
    using State = Rows<T, NB, R>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = a.q_heads / a.cache.heads, kh = blockIdx.y;
    const int split = kShared ? blockIdx.x % splits : 0;
    const int tiles_at_once = kShared ? gridDim.x / splits : gridDim.x * kWaves;
    const float c = a.scale * kLog2e;
    const int gshift = a.cache.page_shift - 4;
    for (int b = blockIdx.z; b < a.sequences; b += gridDim.z) {
        const Span seq = span_of(a, b);
        const int64_t rows = static_cast<int64_t>(seq.n) * group;
        const int64_t row_tiles = (rows + 16 * R - 1) / (16 * R);
        const int32_t *table = a.tables + b * a.table_stride;
        for (int64_t tile = kShared ? blockIdx.x / splits : blockIdx.x * kWaves + wave; tile < row_tiles;
             tile += tiles_at_once) {
            State st;
            st.clear();
            int64_t row[R];
            Place at[R];
            const int past = seq.length - seq.n;  // keys before the first query's own
#pragma unroll
            for (int r = 0; r < R; ++r) {
                row[r] = tile * (16 * R) + 16 * r + (lane & 15);
                const bool real = row[r] < rows;
                const int i = real ? static_cast<int>(row[r] / group) : 0;
                at[r].token = seq.first + i;
                at[r].head = kh * group + (real ? static_cast<int>(row[r] - static_cast<int64_t>(i) * group) : 0);
                st.hi[r] = real ? min(max(past + i + 1, 0), seq.length) : 0;
                st.lo[r] = a.window > 0 ? max(max(past + i + 1, 0) - a.window, 0) : 0;
                st.load_query(r,
                              static_cast<const T *>(a.q.p) + at[r].token * a.q.token_stride +
                                  at[r].head * a.q.head_stride,
                              lane, real);
            }
            // The keys that any of the rows sees, and those that all see.
            const int64_t last_row = min(tile * (16 * R) + 16 * R, rows) - 1;
            const int i0 = static_cast<int>(tile * (16 * R) / group), i1 = static_cast<int>(last_row / group);
            const int lo_any = a.window > 0 ? max(max(past + i0 + 1, 0) - a.window, 0) : 0,
                      hi_any = min(max(past + i1 + 1, 0), seq.length);
            const int lo_all = a.window > 0 ? max(max(past + i1 + 1, 0) - a.window, 0) : 0, hi_all = past + i0 + 1;
            int t0 = lo_any / kTile, t1 = (hi_any + kTile - 1) / kTile;
            if (t1 < t0) t1 = t0;
            int step = 1;
            if (kShared) {
                const int64_t n = t1 - t0;
                const int e = t0 + static_cast<int>(n * (split + 1) / splits);
                t0 += static_cast<int>(n * split / splits) + wave;
                t1 = e;
                step = kWaves;
            }
            bool bad = seq.bad;
            // The groups that hold keys which some row sees: of a step's two
            // one may be outside, and the nearest is read in its place.
            const int group0 = lo_any / kCacheGroup, group1 = (hi_any - 1) / kCacheGroup;
            auto group_of = [&](int t, int u) { return min(max(2 * t + u, group0), group1); };
            auto base_of = [&](int t, int u) {
                const int g = group_of(t, u);
                int64_t p = table[g >> gshift];
                if (p < 0 || p >= a.cache.pages) bad = true, p = 0;
                return a.cache.group(p, kh, g & ((1 << gshift) - 1));
            };
            // A step's keys and values are read into the registers of the
            // step before as soon as those are free: the keys before the
            // weights and the second product, the values after it.
            if (t0 < t1) {
                Raw<NB> x;
                int64_t base[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    base[u] = base_of(t0, u);
                    load_keys<NB>(a.cache.data + base[u], lane, u, x);
                    load_values<NB>(a.cache.data + base[u], lane, u, x);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) base[u] = base_of(min(t0 + step, t1 - 1), u);
                for (int t = t0; t < t1; t += step) {
                    f32x4 s[R][2];
                    u32x4 p[R][State::kP];
                    st.scores(x, lane, s);
#pragma unroll
                    for (int u = 0; u < 2; ++u) load_keys<NB>(a.cache.data + base[u], lane, u, x);
                    const int first = t * kTile;
                    if (first < lo_all || first + kTile > hi_all) st.mask(x, first, lane, s);
                    st.weights(s, c, p);
                    st.add(x, p);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        load_values<NB>(a.cache.data + base[u], lane, u, x);
                        base[u] = base_of(min(t + 2 * step, t1 - 1), u);
                    }
                }
            }
            if (bad) {
#pragma unroll
                for (int r = 0; r < R; ++r) st.sum[r] = NAN;
            }
            float total[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                total[r] = st.sum[r] + __shfl_xor(st.sum[r], 16);
                total[r] += __shfl_xor(total[r], 32);
                st.poison[r] |= __shfl_xor(st.poison[r], 16);
                st.poison[r] |= __shfl_xor(st.poison[r], 32);
            }
            const int d0 = 8 * (lane >> 4);  // within each block
            if constexpr (!kShared) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (row[r] >= rows) continue;
                    const float inv = total[r] == 0 ? 0.0f : 1.0f / total[r];
                    T *dst = static_cast<T *>(a.out.p) + at[r].token * a.out.token_stride +
                             at[r].head * a.out.head_stride + d0;
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            v[i] = st.poison[r] >> n & 1 ? NAN : st.o[r][n][i & 1][i >> 1] * inv;
                        store_eight(dst + 32 * n, v);
                    }
                }
            } else {
                // The waves' parts are brought to one maximum and added.
                static_assert(!kShared || R == 1, "waves that share rows have one tile of them");
                __shared__ float all_m[kWaves][16], all_sum[kWaves][16];
                __shared__ float all_o[kWaves][16][D + 4];
                if (lane < 16) all_m[wave][lane] = st.m[0], all_sum[wave][lane] = total[0];
                const bool real = row[0] < rows;
                if (real) {
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            all_o[wave][lane & 15][32 * n + d0 + i] =
                                st.poison[0] >> n & 1 ? NAN : st.o[0][n][i & 1][i >> 1];
                }
                __syncthreads();
                // A thread takes some of a row's elements.
                constexpr int kPer = D / 16;
                const int rr = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * kPer;
                const int64_t rw = tile * 16 + rr;
                if (rw < rows) {
                    float m = all_m[0][rr], f[kWaves], sum = 0;
#pragma unroll
                    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, all_m[w][rr]);
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) {
                        f[w] = all_m[w][rr] == m ? 1.0f : __builtin_amdgcn_exp2f((all_m[w][rr] - m) * c);
                        sum += f[w] * all_sum[w][rr];
                    }
                    const int i = static_cast<int>(rw / group);
                    const int64_t token = seq.first + i;
                    const int head = kh * group + static_cast<int>(rw - static_cast<int64_t>(i) * group);
                    const float inv = splits > 1 ? 1.0f : sum == 0 ? 0.0f : 1.0f / sum;
                    const int64_t part = (split * a.tokens + token) * a.q_heads + head;
                    if (splits > 1 && (threadIdx.x & 15) == 0) stats[part] = make_float2(m, sum);
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        float v = 0;
#pragma unroll
                        for (int w = 0; w < kWaves; ++w) v += f[w] * all_o[w][rr][e0 + j];
                        v *= inv;
                        if (splits > 1)
                            parts[part * D + e0 + j] = v;
                        else if constexpr (sizeof(T) == 4)
                            static_cast<T *>(a.out.p)[token * a.out.token_stride + head * a.out.head_stride + e0 + j] =
                                v;
                        else
                            static_cast<T *>(a.out.p)[token * a.out.token_stride + head * a.out.head_stride + e0 + j] =
                                __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
                    }
                }
                __syncthreads();
            }
        }
    }
}

// The splits' parts of every row, joined: a block per row, its threads
// four elements of every (256 / (D / 4))th split each, so that the parts are
// read at once (a wave per row, split after split: 51 us for 64 splits of 32
// rows of 128).
template <typename T, int NB>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a, int splits, const float *__restrict__ parts,
                                                   const float2 *__restrict__ stats) {
    constexpr int D = 32 * NB, kQuads = D / 4, kSlots = 256 / kQuads;
    __shared__ float4 sums[kSlots][kQuads];
    __shared__ float totals[kSlots];
    const int quad = threadIdx.x % kQuads, slot = threadIdx.x / kQuads, lane = threadIdx.x & 63;
    const float c = a.scale * kLog2e;
    int64_t first = 0, end = a.tokens;
    if (a.starts) {  // rows behind the last sequence stay as they are
        first = min(max(static_cast<int64_t>(a.starts[0]), INT64_C(0)), a.tokens);
        end = min(max(static_cast<int64_t>(a.starts[a.sequences]), first), a.tokens);
    }
    const int64_t all = a.tokens * a.q_heads;
    for (int64_t row = first * a.q_heads + blockIdx.x; row < end * a.q_heads; row += gridDim.x) {
        float m = -INFINITY;
        for (int s = lane; s < splits; s += 64) m = fmaxf(m, stats[s * all + row].x);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
        float4 v = make_float4(0, 0, 0, 0);
        float sum = 0;
        if (slot < kSlots) {
            for (int s = slot; s < splits; s += kSlots) {
                const float2 x = stats[s * all + row];
                if (x.x == -INFINITY && x.y == 0) continue;  // no keys
                const float f = x.x == m ? 1.0f : __builtin_amdgcn_exp2f((x.x - m) * c);
                const float4 p = *reinterpret_cast<const float4 *>(parts + (s * all + row) * D + 4 * quad);
                sum += f * x.y;
                v.x += f * p.x, v.y += f * p.y, v.z += f * p.z, v.w += f * p.w;
            }
            sums[slot][quad] = v;
            if (quad == 0) totals[slot] = sum;
        }
        __syncthreads();
        if (slot == 0) {
#pragma unroll
            for (int i = 1; i < kSlots; ++i) {
                const float4 p = sums[i][quad];
                v.x += p.x, v.y += p.y, v.z += p.z, v.w += p.w;
                sum += totals[i];
            }
            const float inv = sum == 0 ? 0.0f : 1.0f / sum;
            const int64_t token = row / a.q_heads;
            T *dst = static_cast<T *>(a.out.p) + token * a.out.token_stride +
                     (row - token * a.q_heads) * a.out.head_stride + 4 * quad;
            const float o[4] = {v.x * inv, v.y * inv, v.z * inv, v.w * inv};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4)
                    dst[j] = o[j];
                else
                    dst[j] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(o[j]));
            }
        }
        __syncthreads();
    }
}

struct Plan {
    bool shared;
    int splits, tiles;  // splits of the keys; row tiles (of 16 or 32 rows) of a sequence that the grid covers at once
    size_t parts_bytes, stats_bytes;
};

constexpr int kOwnTiles = 2;  // R of waves with rows of their own

Plan plan_of(const AttendArgs &a) {
    Plan p{};
    const int64_t group = a.q_heads / a.cache.heads;
    const int64_t rows = std::max<int64_t>(1, a.most_queries) * group;
    const int64_t seqs = std::max(1, a.sequences), heads = a.cache.heads;
    const int64_t own = (rows + 16 * kOwnTiles - 1) / (16 * kOwnTiles);
    p.shared = own * heads * seqs < 1024;
    p.splits = 1;
    if (!p.shared) {
        p.tiles = static_cast<int>(std::min<int64_t>(own, 1 << 20));
        return p;
    }
    p.tiles = static_cast<int>((rows + 15) / 16);
    const int64_t blocks = p.tiles * heads * seqs;
    const int64_t keys = static_cast<int64_t>(a.width) << a.cache.page_shift;
    const int64_t most = std::max<int64_t>(1, keys / (kTile * kWaves * 2));
    p.splits = static_cast<int>(std::clamp<int64_t>(768 / blocks, 1, std::min<int64_t>(most, 64)));
    if (p.splits > 1) {
        p.parts_bytes = static_cast<size_t>(p.splits) * a.tokens * a.q_heads * a.cache.dim * 4;
        p.stats_bytes = static_cast<size_t>(p.splits) * a.tokens * a.q_heads * 8;
    }
    return p;
}

template <typename T, int NB>
void launch(const AttendArgs &a, const Plan &p, float *parts, float2 *stats, hipStream_t stream) {
    const unsigned z = std::min(a.sequences, 65535);
    if (p.shared) {
        attend_kernel<T, NB, 1, true><<<dim3(p.splits * p.tiles, a.cache.heads, z), 256, 0, stream>>>(a, p.splits, parts,
                                                                                                 stats);
        if (p.splits > 1) {
            const int64_t rows = a.tokens * a.q_heads;
            join_kernel<T, NB><<<static_cast<unsigned>(std::min<int64_t>(rows, 1 << 20)), 256, 0, stream>>>(
                a, p.splits, parts, stats);
        }
    } else {
        constexpr int R = sizeof(T) == 4 ? 1 : kOwnTiles;
        const unsigned x = static_cast<unsigned>((p.tiles * (kOwnTiles / R) + kWaves - 1) / kWaves);
        attend_kernel<T, NB, R, false><<<dim3(x, a.cache.heads, z), 256, 0, stream>>>(a, 1, nullptr, nullptr);
    }
}

template <typename T>
void launch(const AttendArgs &a, const Plan &p, float *parts, float2 *stats, hipStream_t stream) {
    switch (a.cache.dim / 32) {
        case 1: return launch<T, 1>(a, p, parts, stats, stream);
        case 2: return launch<T, 2>(a, p, parts, stats, stream);
        case 3: return launch<T, 3>(a, p, parts, stats, stream);
        case 4: return launch<T, 4>(a, p, parts, stats, stream);
        case 5: return launch<T, 5>(a, p, parts, stats, stream);
        case 6: return launch<T, 6>(a, p, parts, stats, stream);
        case 7: return launch<T, 7>(a, p, parts, stats, stream);
        default: return launch<T, 8>(a, p, parts, stats, stream);
    }
}

}  // namespace

int64_t attend_workspace_bytes(const AttendArgs &a) {
    const Plan p = plan_of(a);
    return static_cast<int64_t>(p.parts_bytes + p.stats_bytes);
}

bool attend_launch(const AttendArgs &a, void *workspace, hipStream_t stream) {
    if (a.sequences == 0 || a.tokens == 0) return true;
    const Plan p = plan_of(a);
    auto *parts = static_cast<float *>(workspace);
    auto *stats = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + p.parts_bytes);
    if (a.bf16)
        launch<uint16_t>(a, p, parts, stats, stream);
    else
        launch<float>(a, p, parts, stats, stream);
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
