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

#include <cfloat>

#include <algorithm>
#include <type_traits>

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
// powers of two): weights stay near 2^8 at most, and most steps spare the
// rescaling.
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

// The maximum m that a row's weights refer to.  f32 outputs: a score, and
// weights' exponents (s - m) c: a score equal to m has the weight 1 exactly,
// so that equal keys give their value back.  bf16 outputs: c times a score,
// rounded, and exponents c s - m in one operation: what the rounding leaves is
// a factor of all the row's weights, and the sum of two bf16 numbers is off by
// less than a bf16 output shows (4 x 512 queries: 276 us for 310).  That
// factor is near 1 only where m is not far: a wave that holds a row with m
// past kFar works with scores as f32 outputs do (its rows are `raw`), which is
// also right where c s passes the float32 numbers.  What it takes to tell costs
// 276 us for 273, or 300 for 288 where most steps move a maximum (scale 1).
template <typename T>
constexpr bool kScaled = sizeof(T) == 2;
constexpr float kFar = 0x1p20f;  // the factor is 2^(2^-4) at most

// The power of two of weights that refer to `from` where they refer to `to`
// (Rows::reference): 0 for what saw no key, where there is another.
__device__ inline float factor(double from, double to) {
    return from == to ? 1.0f : __builtin_amdgcn_exp2f(static_cast<float>(from - to));
}

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

// Byte i of w as the float32 2^(byte - 127), a scale operand.  Byte 0 gives
// 0.0: the conversions look at an operand's exponent field alone and take it
// as 2^-127, which the tests of the smallest scales pin.
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
struct __attribute__((aligned(N % 4 == 0 ? 16 : N % 2 == 0 ? 8 : 4))) Words {
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
    float m[R], sum[R];      // the maximum that weights refer to; the lane's part of their sum
    int raw;                 // 1: m are scores, those of f32 outputs always (an int: 276 us as above for 288)
    int lo[R], hi[R];        // the keys that the lane's row sees
    uint32_t poison[R];      // blocks in which the row sees a NaN value

    // c = scale log2(e).  Above 1 it may take every score of a row to -inf,
    // which its first maximum would not show: such rows begin raw.
    __device__ void clear(float c) {
        raw = !kScaled<T> || c > 1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = raw ? -INFINITY : -FLT_MAX, sum[r] = 0, poison[r] = 0;
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
                score(a, p, s, u);
            }
        }
    }

    // Adds the products of piece p of a group's keys to its scores.
    __device__ void score(const u32x4 &k, int p, f32x4 (&s)[R][2], int u) const {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = kQ - 1; j >= 0; --j) s[r][u] = mfma(k, q[r][j][p], s[r][u]);
    }

    // Adds the weighted values of block b: its even and its odd elements.
    __device__ void add_block(const u32x4 &even, const u32x4 &odd, int b, const u32x4 (&p)[R][kP]) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = kP - 1; j >= 0; --j) {
                o[r][b][0] = mfma(even, p[r][j], o[r][b][0]);
                o[r][b][1] = mfma(odd, p[r][j], o[r][b][1]);
            }
    }

    // Scores of keys that a row does not see become -inf.  A weight of 0 does
    // not take away a NaN or an infinity (bytes above 252, which no finite
    // block has): such values are taken out as well and kept in mind for the
    // rows that see them.
    __device__ void mask(uint32_t (&vs)[2][NB], int first, int lane, f32x4 (&s)[R][2]) {
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
                const uint32_t w = vs[u][b];
                bad |= ((w & 0x7f7f7f7fu) + 0x03030303u) & w & 0x80808080u;
            }
        if (!__any(bad != 0)) return;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if ((vs[u][b] >> (8 * i) & 255) > 252) {
                        vs[u][b] &= ~(255u << (8 * i));
#pragma unroll
                        for (int r = 0; r < R; ++r) poison[r] |= (seen[r] >> (4 * u + i) & 1) << b;
                    }
    }

    static __device__ float largest(const f32x4 (&x)[2]) {
        float top = x[0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i >> 2][i & 3]);
        return top;
    }

    // Moves the rows' maxima where the scores ask for it; c = scale log2(e).
    // From here on s are the weights' exponents where kScaled<T>.
    __device__ void raise(f32x4 (&s)[R][2], float c) {
        bool move = false;
        f32x4 e[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if constexpr (kScaled<T>) {
#pragma unroll
                for (int i = 0; i < 8; ++i) e[r][i >> 2][i & 3] = __builtin_fmaf(s[r][i >> 2][i & 3], c, -m[r]);
                move |= largest(e[r]) > kSlack;
            } else {
                move |= (largest(s[r]) - m[r]) * c > kSlack;  // infinite at first; false for two infinities
            }
        }
        if constexpr (kScaled<T>) {
            if ((__ballot(move) | static_cast<uint64_t>(raw)) != 0) settle(s, c, e);
#pragma unroll
            for (int r = 0; r < R; ++r) s[r][0] = e[r][0], s[r][1] = e[r][1];
        } else if (__any(move)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float top = fmaxf(m[r], of_row(largest(s[r])));
                const float f = top == m[r] ? 1.0f : __builtin_amdgcn_exp2f((m[r] - top) * c);
                m[r] = top;
                sum[r] *= f;
#pragma unroll
                for (int b = 0; b < NB; ++b) o[r][b][0] *= f, o[r][b][1] *= f;
            }
        }
    }

    // The largest of the four lanes that share a row.
    static __device__ float of_row(float x) {
        x = fmaxf(x, __shfl_xor(x, 16));
        return fmaxf(x, __shfl_xor(x, 32));
    }

    // raise() where maxima move or are raw: also the exponents e.
    __device__ void settle(const f32x4 (&s)[R][2], float c, f32x4 (&e)[R][2]) {
        float top[R], f[R];
        bool near = !raw;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            top[r] = of_row(largest(s[r]));
            f[r] = fmaxf(m[r], top[r] * c);
            near &= fabsf(f[r]) <= kFar || !(top[r] > -INFINITY);  // or has seen no key
        }
        if (__all(near)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float n = f[r];
                f[r] = __builtin_amdgcn_exp2f(m[r] - n);
                m[r] = n;
            }
        } else {
            refer(top, c, f);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sum[r] *= f[r];
#pragma unroll
            for (int b = 0; b < NB; ++b) o[r][b][0] *= f[r], o[r][b][1] *= f[r];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float x = raw && m[r] > -INFINITY ? m[r] : 0.0f, y = raw ? 0.0f : -m[r];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                e[r][i >> 2][i & 3] = __builtin_fmaf(s[r][i >> 2][i & 3] - x, c, y);
        }
    }

    // settle()'s new maxima where they were raw or one is far, and the factors
    // of the weights so far.  They are raw from here on if one is far or, of
    // those that began so, belongs to a row that will see a key and has not.
    __device__ void refer(const float (&top)[R], float c, float (&f)[R]) {
        const int was = raw;
        bool near = true;
        double from[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            from[r] = reference(was, m[r], c);
            m[r] = fmaxf(was ? m[r] : m[r] == -FLT_MAX ? -INFINITY : m[r] / c, top[r]);
            near &= fabsf(m[r] * c) <= kFar || lo[r] >= hi[r];
        }
        raw = __builtin_amdgcn_readfirstlane(__ballot(!near) != 0);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!raw) m[r] = fmaxf(m[r] * c, -FLT_MAX);
            f[r] = factor(from[r], reference(raw, m[r], c));
        }
    }

    // c times a maximum, exactly.
    static __device__ double reference(bool raw, float m, float c) {
        if (!kScaled<T> || raw) return static_cast<double>(m) * static_cast<double>(c);
        return m == -FLT_MAX ? -INFINITY : static_cast<double>(m);
    }

    // What raise() left to weights, as the parts that the second product takes.
    __device__ void weights(const f32x4 (&s)[R][2], float c, u32x4 (&p)[R][kP]) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float base = m[r] == -INFINITY ? 0.0f : m[r];
            auto weight = [&](float x) { return __builtin_amdgcn_exp2f(kScaled<T> ? x : (x - base) * c); };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float a = weight(s[r][i >> 1][2 * (i & 1)]), b = weight(s[r][i >> 1][2 * (i & 1) + 1]);
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
            add_block(even, odd, b, p);
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

// Waves of a SIMD that the registers are kept few enough for: a row tile's
// sums and queries, a step's codes and scales, and about 70 more.  An estimate:
// rows_kernel keeps 11 registers of a lane in memory for bf16 heads of 32 and
// 160 and f32 heads of 96, 3 for f32 heads of 192, line_kernel one for f32 heads
// of 32 in items of 32 that are cut.
template <typename T, int NB, int R>
constexpr int kRegisters = R * NB * (8 + 4 * Parts<T>::q) + 6 * NB + 60 + 10 * R;
template <typename T, int NB, int R>
constexpr int kOccupancy = kRegisters<T, NB, R> <= 110   ? 4
                           : kRegisters<T, NB, R> <= 150 ? 3
                           : kRegisters<T, NB, R> <= 235 ? 2
                                                         : 1;

// The keys that rows of a sequence see, from the first's first to the last's last.
struct Keys {
    int lo, hi;
};
__device__ inline Keys keys_of(const AttendArgs &a, const Span &s, int query0, int query1) {
    const int past = s.length - s.n;  // keys before the first query's own
    return {a.window > 0 ? max(max(past + query0 + 1, 0) - a.window, 0) : 0,
            min(max(past + query1 + 1, 0), s.length)};
}

// A wave's rows from `row0`: its queries, and the keys that each sees.
template <typename T, int NB, int R>
__device__ inline void load_rows(const AttendArgs &a, const Span &seq, int kh, int group, int rows, int row0, int lane,
                                 Rows<T, NB, R> &st, Place (&at)[R], bool (&real)[R]) {
    st.clear(a.scale * kLog2e);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + 16 * r + (lane & 15);
        real[r] = row < rows;
        const int i = real[r] ? row / group : 0;
        at[r].token = seq.first + i;
        at[r].head = kh * group + (real[r] ? row - i * group : 0);
        const Keys k = keys_of(a, seq, i, i);
        st.lo[r] = k.lo;
        st.hi[r] = real[r] ? k.hi : 0;
        st.load_query(r,
                      static_cast<const T *>(a.q.p) + at[r].token * a.q.token_stride + at[r].head * a.q.head_stride,
                      lane, real[r]);
    }
}

// Where groups of 16 keys lie, asked for in ascending order.  A group outside
// of what the rows see is not read, but the nearest in its place; a bad page
// is not read either.  A lane holds where one of 64 pages begins, and the
// number of one of the 64 after them, so that a step waits for no table and
// finds its place with a few scalar instructions (4 x 512 queries: 49 us of 340
// with a page's number read, checked and multiplied for each group).
template <int NB>
struct Groups {
    const int32_t *table;
    int first, last, shift;  // groups that hold keys which some row sees; groups of a page
    int lane;
    bool bad;
    int at, next;            // which 64 pages; the numbers of the next ones
    int64_t here, head, unit, pages;

    __device__ Groups(const AttendArgs &a, const Span &seq, int b, const Keys &any, int kh, int lane)
        : table(a.tables + b * a.table_stride), first(any.lo / kCacheGroup), last((any.hi - 1) / kCacheGroup),
          shift(a.cache.page_shift - 4), lane(lane), bad(seq.bad), at(-1), next(0), here(0),
          head(a.cache.group(0, kh, 0)), unit(a.cache.group(1, 0, 0)), pages(a.cache.pages) {}
    // Of groups first .. last (there is one).
    __device__ int load(int block) const {
        return table[min(max(block * 64 + lane, first >> shift), last >> shift)];
    }
    __device__ int64_t begin_of(int page) {
        const bool real = page >= 0 && page < pages;
        bad |= __any(!real);
        return (real ? page : 0) * unit + head;
    }
    __device__ void begin(int g) {
        at = (min(max(g, first), last) >> shift) >> 6;
        here = begin_of(load(at));
        next = load(at + 1);
    }
    __device__ int64_t aim(int g) {
        g = min(max(g, first), last);
        const int i = g >> shift;
        if (i >> 6 != at) {
            if (i >> 6 == at + 1)
                at = i >> 6, here = begin_of(next), next = load(at + 1);
            else
                begin(g);
        }
        const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(here), i & 63),
                       hi = __builtin_amdgcn_readlane(static_cast<int>(here >> 32), i & 63);
        return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo) + (g & ((1 << shift) - 1)) * (544 * NB);
    }
};

// The sequence of the rank-th greatest length, of 64 at most (the first of equal ones first).
__device__ inline int of_rank(const int32_t *lengths, int sequences, int rank, int lane) {
    const int mine = lane < sequences ? lengths[lane] : INT32_MIN;
    int before = 0;
    for (int i = 0; i < sequences; ++i) {
        const int other = __builtin_amdgcn_readlane(mine, i);
        before += other > mine || (other == mine && i < lane);
    }
    const uint64_t found = __ballot(lane < sequences && before == rank);
    return found ? __builtin_ctzll(found) : 0;
}

// Steps' keys and values as the products' left operands, in LDS, with the
// values' scales: what a block of rows_kernel works from.
template <int NB>
struct Operands {
    u32x4 k[2][2][NB][64];     // step, group, piece of 8 elements, lane
    u32x4 v[2][NB][2][64];     // step, block, even or odd elements, lane
    uint32_t vs[2][2][4][NB];  // step, group, four tokens, block
};

// What a wave converts of a step: of one group the first or the second half
// of the pieces and of the blocks (where NB is odd the first has one less).
template <int N>
struct __attribute__((packed, aligned(4))) Run {
    uint32_t w[N];
};
template <int NB>
struct Share {
    static constexpr int kMost = NB - NB / 2, kScales = NB % 4 == 0 ? 1 : kMost;
    Run<kMost> k, v, vs;
    uint8_t ks[kScales];

    // Where a half begins: of an odd number of pieces they share one.
    static __device__ int first_of(int wave) { return wave & 1 ? NB / 2 : 0; }

    __device__ void load_keys(const uint8_t *g, int lane, int first) {
        k = *reinterpret_cast<const Run<kMost> *>(g + lane * 4 * NB + 4 * first);
#pragma unroll
        for (int i = 0; i < kScales; ++i)
            ks[i] = g[16 * 32 * NB + (lane & 15) * NB + ((lane >> 4) * NB + first + i) / 4];
    }
    __device__ void load_values(const uint8_t *g, int lane, int first) {
        constexpr int D = 32 * NB;
        v = *reinterpret_cast<const Run<kMost> *>(g + 8 * D + lane * 4 * NB + 4 * first);
        vs = *reinterpret_cast<const Run<kMost> *>(g + 16 * D + D / 2 + (lane >> 4) * 4 * NB + 4 * first);
    }
    __device__ void convert_keys(Operands<NB> &to, int step, int u, int lane, int first) const {
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const float scale = __uint_as_float(static_cast<uint32_t>(ks[i % kScales]) << 23);
            to.k[step & 1][u][first + i][lane] = u32x4{fp4_pair<0>(k.w[i], scale), fp4_pair<1>(k.w[i], scale),
                                                       fp4_pair<2>(k.w[i], scale), fp4_pair<3>(k.w[i], scale)};
        }
    }
    // In a masked step the values' scales are kept, and those that no weight
    // of 0 would take away become zeros.  Apart from the conversion, which has
    // no branch: products and other instructions then stand in one stretch of
    // code, and the scheduler puts them beside each other.
    __device__ void clean_values(Operands<NB> &to, int step, int u, int lane, int first) {
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            if ((lane & 15) == 0) to.vs[step & 1][u][lane >> 4][first + i] = vs.w[i];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if ((vs.w[i] >> (8 * j) & 255) > 252) vs.w[i] &= ~(255u << (8 * j));
        }
    }
    __device__ void convert_values(Operands<NB> &to, int step, int u, int lane, int first) const {
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
            const uint32_t by = vs.w[i];
            const uint32_t w[4] = {fp4_pair<0>(v.w[i], scale_of(by, 0)), fp4_pair<1>(v.w[i], scale_of(by, 1)),
                                   fp4_pair<2>(v.w[i], scale_of(by, 2)), fp4_pair<3>(v.w[i], scale_of(by, 3))};
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            reinterpret_cast<u32x2 *>(&to.v[step & 1][first + i][0][lane])[u] =
                u32x2{__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u)};
            reinterpret_cast<u32x2 *>(&to.v[step & 1][first + i][1][lane])[u] =
                u32x2{__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)};
        }
    }
};

// Rows of their own for each wave; a block's four waves go through the keys
// together and share the conversion of a step to bf16, a quarter each, through
// LDS.  The scores of a step are computed beside the weights of the one
// before, and the next operands converted beside the second product; what is
// converted was read two steps before.  4 x 512 queries, 32 heads of 128 over
// 8 of up to 8192 keys in 276 us, 706 TFLOP/s (before later steps, 345: every
// wave converting for itself: 428; in the sequences' order: 393).  Bound by
// the instructions of weights, conversion and products, of which two waves on
// a SIMD hide little of each other's.
template <typename T, int NB, int R>
__global__ __launch_bounds__(256, (kOccupancy<T, NB, R>)) void rows_kernel(AttendArgs a, int tiles_at_once) {
    using State = Rows<T, NB, R>;
    constexpr int kRows = 16 * R * kWaves;
    __shared__ Operands<NB> ops;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = a.q_heads / a.cache.heads;
    const float c = a.scale * kLog2e;
    const int64_t each = static_cast<int64_t>(tiles_at_once) * a.cache.heads, all = each * a.sequences;
    for (int64_t id = blockIdx.x; id < all; id += gridDim.x) {
        // Neighbouring blocks take the heads of keys, which then stay in one
        // die's cache.  The longest sequences come first; where all blocks run
        // at once, every second 256 of them, which join the 256 before on
        // their compute units, stand in reverse.
        int64_t place = id;
        if (a.sequences <= 64 && all <= 256 * kOccupancy<T, NB, R> && (id >> 8 & 1)) {
            const int64_t layer = id & ~255, last = min(layer + 256, all) - 1;
            place = layer + (last - id);
        }
        const int rank = static_cast<int>(place / each), in = static_cast<int>(place - rank * each);
        const int kh = in % a.cache.heads;
        const int b = a.sequences <= 64 ? of_rank(a.lengths, a.sequences, rank, lane) : rank;
        const Span seq = span_of(a, b);
        const int rows = seq.n * group;  // the launcher holds tokens x q_heads below 2^31
        const int tiles = (rows - 1) / kRows + (rows > 0);
        // The last rows, which see the most keys, first.
        for (int tile = tiles - 1 - in / a.cache.heads; tile >= 0; tile -= tiles_at_once) {
            const int row0 = tile * kRows, row1 = min(rows - row0, kRows) + row0 - 1;
            const Keys any = keys_of(a, seq, row0 / group, row1 / group);
            const int lo_all = keys_of(a, seq, row1 / group, row1 / group).lo,
                      hi_all = keys_of(a, seq, row0 / group, row0 / group).hi;
            State st;
            Place at[R];
            bool real[R];
            load_rows(a, seq, kh, group, rows, row0 + wave * 16 * R, lane, st, at, real);
            const int t0 = any.lo / kTile, t1 = (any.hi + kTile - 1) / kTile;
            Groups<NB> groups(a, seq, b, any, kh, lane);
            auto masked = [&](int t) { return t * kTile < lo_all || t * kTile + kTile > hi_all; };
            if (any.lo < any.hi) {
                const int u = wave >> 1, half = Share<NB>::first_of(wave);
                groups.begin(2 * t0 + u);
                // The group of a step that this wave converts; past the last step that one again.
                auto group_of = [&](int t) { return a.cache.data + groups.aim(2 * min(t, t1 - 1) + u); };
                auto scores = [&](int t, f32x4 (&s)[R][2]) {
#pragma unroll
                    for (int r = 0; r < R; ++r) s[r][0] = s[r][1] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int g = 0; g < 2; ++g) st.score(ops.k[t & 1][g][i][lane], i, s, g);
                };
                // On their way: the keys of two steps and the values of two,
                // those one step behind.
                Share<NB> now, then;
                const uint8_t *g0 = group_of(t0), *g1 = group_of(t0 + 1), *g2 = group_of(t0 + 2), *g3 = group_of(t0 + 3);
                now.load_keys(g0, lane, half);
                now.load_values(g0, lane, half);
                then.load_keys(g1, lane, half);
                now.convert_keys(ops, t0, u, lane, half);
                if (masked(t0)) now.clean_values(ops, t0, u, lane, half);
                now.convert_values(ops, t0, u, lane, half);
                then.convert_keys(ops, t0 + 1, u, lane, half);
                now.load_keys(g2, lane, half);
                now.load_values(g1, lane, half);
                then.load_keys(g3, lane, half);
                then.load_values(g2, lane, half);
                __syncthreads();
                f32x4 s[R][2];
                scores(t0, s);
                __syncthreads();  // step t0's keys are read
                for (int t = t0; t < t1; ++t) {
                    // Here: scores of t; in LDS the keys of t + 1 and the
                    // values of t; on their way the keys of t + 2 and the
                    // values of t + 1 (now), and those of the step after.
                    const uint8_t *g4 = group_of(t + 4);
                    if (masked(t)) {
                        uint32_t vs[2][NB];
#pragma unroll
                        for (int g = 0; g < 2; ++g)
#pragma unroll
                            for (int i = 0; i < NB; ++i) vs[g][i] = ops.vs[t & 1][g][lane >> 4][i];
                        st.mask(vs, t * kTile, lane, s);
                    }
                    if (masked(t + 1)) now.clean_values(ops, t + 1, u, lane, half);
                    st.raise(s, c);
                    f32x4 next[R][2];
                    u32x4 p[R][State::kP];
                    scores(t + 1, next);
                    st.weights(s, c, p);
                    u32x4 even = ops.v[t & 1][0][0][lane], odd = ops.v[t & 1][0][1][lane];
                    now.convert_keys(ops, t + 2, u, lane, half);
                    now.convert_values(ops, t + 1, u, lane, half);
                    now = then;
                    then.load_keys(g4, lane, half);
                    then.load_values(g3, lane, half);
                    g3 = g4;
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        const int n = i + 1 < NB ? i + 1 : i;
                        const u32x4 e = ops.v[t & 1][n][0][lane], o = ops.v[t & 1][n][1][lane];
                        st.add_block(even, odd, i, p);
                        even = e, odd = o;
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) s[r][0] = next[r][0], s[r][1] = next[r][1];
                    __syncthreads();
                }
            }
            const bool bad = __syncthreads_or(groups.bad);  // of pages that a wave alone went to
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float total = bad ? NAN : st.sum[r];
                total += __shfl_xor(total, 16);
                total += __shfl_xor(total, 32);
                st.poison[r] |= __shfl_xor(st.poison[r], 16);
                st.poison[r] |= __shfl_xor(st.poison[r], 32);
                if (!real[r]) continue;
                const float inv = total == 0 ? 0.0f : 1.0f / total;
                T *dst = static_cast<T *>(a.out.p) + at[r].token * a.out.token_stride + at[r].head * a.out.head_stride +
                         8 * (lane >> 4);
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = st.poison[r] >> n & 1 ? NAN : st.o[r][n][i & 1][i >> 1] * inv;
                    store_eight(dst + 32 * n, v);
                }
            }
        }
    }
}

// A step's two groups as they lie in the cache, in LDS, and how many steps
// are on their way there: what fits beside the waves that the registers allow.
template <int NB>
constexpr int kStage = 2 * 544 * NB;
template <int NB>
constexpr int kSlots = NB <= 2 ? 4 : NB <= 4 ? 3 : 2;

// LDS of a block: its waves' rings, or their parts of the output, and maxima and sums.
template <int NB, int R>
constexpr int kLineLds = 768 * R + kWaves * std::max(kStage<NB> * kSlots<NB>, 16 * R * (32 * NB + 4) * 4);

// Waits until at most N of this wave's loads are on their way.
template <int N>
__device__ inline void outstanding() {
    static_assert(N < 64, "the counter's range");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
    asm volatile("" ::: "memory");
}

// All steps of a call in one line: sequence after sequence, its row tiles and
// heads of keys one after the other (an item each), and an item's steps of 32
// keys.  Each of `count` blocks takes an equal stretch of it, whatever the
// sequences' lengths.  Beginning an item and joining its waves takes a block
// about as long as kItemCost steps, which stand before its first one in the
// line (without them, in an earlier state, 64 sequences of 500 to 8192 keys:
// blocks done after 55 to 106 us).
struct Line {
    int64_t total;  // steps
    int count;      // blocks
    __device__ int64_t from(int i) const { return total * i / count; }
    __device__ int block_of(int64_t w) const { return static_cast<int>(((w + 1) * count - 1) / total); }
};
// 64 sequences of 500 to 8192 keys: 73.7 us (8: 77.1, 12: 74.0, 24: 72.8, 40:
// 75.0); one of 65 536: 28.5 (24 and 40: 29.3).
constexpr int kItemCost = 16;
// The least stretch of a block: short calls have fewer blocks, each of which
// costs the rest a part to join (17 sequences of up to 3001 keys, 5 queries
// and a window of 1000: 15.0 us; 4: 15.9, 16: 16.6, 40: 24.2).
constexpr int kLeast = 8;

// A number that is one for the wave, in a scalar register.
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline int64_t uniform(int64_t v) {
    const uint32_t lo = uniform(static_cast<int>(v)), hi = uniform(static_cast<int>(v >> 32));
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// An item's length for sequence s (a step where its rows see no key: they are
// written as well), and its items.  All items of a sequence run the steps that
// any of its rows sees, so that an item's place in the line is a product: a
// prompt from its first token runs twice the steps that its rows see, 512
// queries with a window of 128 four times.
__device__ inline int length_of(const AttendArgs &a, const Span &s) {
    const Keys k = keys_of(a, s, 0, s.n - 1);
    return kItemCost + (k.lo < k.hi ? (k.hi + kTile - 1) / kTile - k.lo / kTile : 1);
}
template <int R>
__device__ inline int items_of(const AttendArgs &a, const Span &s, int group) {
    return (s.n * group + 16 * R - 1) / (16 * R) * a.cache.heads;
}

// Which blocks hold the parts of a row's output: `parts` of them from `first`
// on (none: the output is written), as row `row` of their tiles.
struct Parts16 {
    int first, parts, row, pad;
};

// What a part's weights refer to, and their sum.
struct Stats {
    double m;
    float sum, pad;
};

// Waves of a SIMD of it: few values of it are not the wave's.
template <typename T, int NB, int R>
constexpr int kLineOccupancy = kRegisters<T, NB, R> <= 126 ? 4 : kOccupancy<T, NB, R>;

// An item is 16 R rows of a head of keys, shared by a block's four waves, which
// split its keys.  kWhole: a block takes items as they are, `tiles` row tiles of
// a sequence at once, and nothing is left to join; else its stretch of the line.
template <typename T, int NB, int R, bool kWhole>
__global__ __launch_bounds__(256, (kLineOccupancy<T, NB, R>)) void line_kernel(AttendArgs a, int tiles, float *parts,
                                                                              Stats *stats, Parts16 *where) {
    constexpr int D = 32 * NB, kRows = 16 * R;
    using State = Rows<T, NB, R>;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kLineLds<NB, R> - 768 * R];
    __shared__ double all_m[kWaves][kRows];
    __shared__ float all_sum[kWaves][kRows];
    auto all_o = reinterpret_cast<float(*)[kRows][D + 4]>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), block = blockIdx.x;
    const int group = a.q_heads / a.cache.heads;
    const float c = a.scale * kLog2e;

    // Steps [n0, n1) of the item of rows from row0; `share` of them (0: the
    // item is whole) will be joined.
    auto work = [&](const Span &seq, int b, int kh, int row0, int n0, int n1, int share) {
        const int rows = seq.n * group, row1 = min(rows - row0, kRows) + row0 - 1;
        const Keys all = keys_of(a, seq, 0, seq.n - 1), any = keys_of(a, seq, row0 / group, row1 / group);
        const int lo_all = keys_of(a, seq, row1 / group, row1 / group).lo,
                  hi_all = keys_of(a, seq, row0 / group, row0 / group).hi;
        // This wave's steps: every fourth of the block's.
        const int t0 = all.lo / kTile + n0 + wave, t1 = all.lo / kTile + n1;
        Groups<NB> groups(a, seq, b, any, kh, lane);
        // Copies a step straight to LDS, 16 bytes a lane, as it lies.  Past
        // the last step that one is copied again (a branch around the loads
        // would cost more).
        constexpr int kGroupChunks = 34 * NB, kLoads = (2 * kGroupChunks + 63) / 64;
        uint8_t *ring = lds + wave * kStage<NB> * kSlots<NB>;
        int64_t base[2];
        // Past the last step that one again.
        auto aim = [&](int t) {
            t = min(t, t1 - 1);
            base[0] = groups.aim(2 * t);
            base[1] = groups.aim(2 * t + 1);
        };
        auto fetch = [&](int slot) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int chunk = i * 64 + lane;
                const bool second = chunk >= kGroupChunks;
                const uint8_t *src = a.cache.data + (second ? base[1] : base[0]) +
                                     (chunk - (second ? kGroupChunks : 0)) * 16;
                if (chunk < 2 * kGroupChunks)
                    __builtin_amdgcn_global_load_lds(
                        (const __attribute__((address_space(1))) void *)src,
                        (__attribute__((address_space(3))) void *)(ring + slot * kStage<NB> + i * 1024), 16, 0, 0);
            }
        };
        const bool steps = any.lo < any.hi && t0 < t1;
        if (steps) {
            groups.begin(2 * t0);
#pragma unroll
            for (int i = 0; i < kSlots<NB>; ++i) {
                aim(t0 + i * kWaves);
                fetch(i);
            }
            aim(t0 + kSlots<NB> * kWaves);
        }
        State st;
        Place at[R];
        bool real[R];
        load_rows(a, seq, kh, group, rows, row0, lane, st, at, real);
        if (steps) {
            outstanding<0>();  // the queries are not counted below
            int slot = 0;
            for (int t = t0; t < t1; t += kWaves) {
                outstanding<(kSlots<NB> - 1) * kLoads>();
                const uint8_t *stage = ring + slot * kStage<NB>;
                Raw<NB> x;
                f32x4 s[R][2];
                u32x4 p[R][State::kP];
#pragma unroll
                for (int u = 0; u < 2; ++u) load_keys<NB>(stage + u * 544 * NB, lane, u, x);
                st.scores(x, lane, s);
#pragma unroll
                for (int u = 0; u < 2; ++u) load_values<NB>(stage + u * 544 * NB, lane, u, x);
                const int first = t * kTile;
                if (first < lo_all || first + kTile > hi_all) st.mask(x.vs, first, lane, s);
                st.raise(s, c);
                st.weights(s, c, p);
                // The step is in registers: its slot is free.
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                fetch(slot);
                aim(t + (kSlots<NB> + 1) * kWaves);
                st.add(x, p);
                slot = slot == kSlots<NB> - 1 ? 0 : slot + 1;
            }
            outstanding<0>();  // the ring's memory is used again
        }
        // The waves' parts are brought to one maximum and added.
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float total = groups.bad ? NAN : st.sum[r];
            total += __shfl_xor(total, 16);
            total += __shfl_xor(total, 32);
            st.poison[r] |= __shfl_xor(st.poison[r], 16);
            st.poison[r] |= __shfl_xor(st.poison[r], 32);
            if (lane < 16) all_m[wave][16 * r + lane] = st.reference(st.raw, st.m[r], c), all_sum[wave][16 * r + lane] = total;
        }
        __syncthreads();  // all waves are through with their rings
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!real[r]) continue;
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float4 *dst = reinterpret_cast<float4 *>(&all_o[wave][16 * r + (lane & 15)][32 * n + 8 * (lane >> 4)]);
                const bool nan = st.poison[r] >> n & 1;
                const f32x4 e = st.o[r][n][0], o = st.o[r][n][1];
                dst[0] = nan ? make_float4(NAN, NAN, NAN, NAN) : make_float4(e[0], o[0], e[1], o[1]);
                dst[1] = nan ? make_float4(NAN, NAN, NAN, NAN) : make_float4(e[2], o[2], e[3], o[3]);
            }
        }
        __syncthreads();
        // A thread takes some of a row's elements.
        constexpr int kPer = D / 16;
        const int e0 = (threadIdx.x & 15) * kPer;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int rr = 16 * r + (threadIdx.x >> 4), rw = row0 + rr;
            if (rw >= rows) break;
            double m = all_m[0][rr];
            float f[kWaves], sum = 0;
#pragma unroll
            for (int v = 1; v < kWaves; ++v) m = fmax(m, all_m[v][rr]);
#pragma unroll
            for (int v = 0; v < kWaves; ++v) {
                f[v] = factor(all_m[v][rr], m);
                sum += f[v] * all_sum[v][rr];
            }
            const int i = rw / group;
            const int64_t token = seq.first + i;
            const int head = kh * group + rw - i * group;
            const int64_t slot = (2 * block + (n0 == 0)) * kRows + rr;  // where a part goes
            if (!kWhole && (threadIdx.x & 15) == 0) {
                if (share) stats[slot] = Stats{m, sum, 0};
                if (n0 == 0) where[token * a.q_heads + head] = Parts16{block, share, rr, 0};
            }
            const float inv = share ? 1.0f : sum == 0 ? 0.0f : 1.0f / sum;
            T *dst = static_cast<T *>(a.out.p) + token * a.out.token_stride + head * a.out.head_stride + e0;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                float v = 0;
#pragma unroll
                for (int u = 0; u < kWaves; ++u) v += f[u] * all_o[u][rr][e0 + j];
                v *= inv;
                if (share)
                    parts[slot * D + e0 + j] = v;
                else if constexpr (sizeof(T) == 4)
                    dst[j] = v;
                else
                    dst[j] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
            }
        }
        __syncthreads();
    };

    if constexpr (kWhole) {
        const int64_t each = static_cast<int64_t>(tiles) * a.cache.heads, all = each * a.sequences;
        for (int64_t id = block; id < all; id += gridDim.x) {
            const int b = static_cast<int>(id / each), in = static_cast<int>(id - b * each), kh = in % a.cache.heads;
            const Span seq = span_of(a, b);
            // Counted in tiles: rows end near 2^31.
            const int of_rows = (seq.n * group + kRows - 1) / kRows;
            for (int tile = in / a.cache.heads; tile < of_rows; tile += tiles)
                work(seq, b, kh, tile * kRows, 0, length_of(a, seq) - kItemCost, 0);
        }
        return;
    }
    // The line's length, 64 sequences at a time (the last 64 stay in registers).
    Line line = {0, 0};
    int64_t mine = 0;
    for (int b = lane; b < (a.sequences + 63) / 64 * 64; b += 64) {
        mine = 0;
        if (b < a.sequences) {
            const Span s = span_of(a, b);
            mine = static_cast<int64_t>(items_of<R>(a, s, group)) * length_of(a, s);
        }
        line.total += mine;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) line.total += __shfl_xor(static_cast<long long>(line.total), o);
    line.total = uniform(line.total);
    if (line.total == 0) return;
    line.count = static_cast<int>(min(max(line.total / kLeast, INT64_C(1)), static_cast<int64_t>(gridDim.x)));
    if (block >= line.count) return;
    int64_t w = line.from(block);
    const int64_t w_end = line.from(block + 1);
    // The sequence that w is in, and where that begins.
    int b = 0;
    int64_t begin = 0;
    for (int b0 = 0; b0 < a.sequences; b0 += 64) {
        if (a.sequences > 64) {
            mine = 0;
            if (b0 + lane < a.sequences) {
                const Span s = span_of(a, b0 + lane);
                mine = static_cast<int64_t>(items_of<R>(a, s, group)) * length_of(a, s);
            }
        }
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t v = __shfl_up(static_cast<long long>(upto), o);
            if (lane >= o) upto += v;
        }
        const uint64_t past = __ballot(begin + upto > w);
        if (past) {
            const int l = __builtin_ctzll(past);
            b = b0 + l;
            begin += __shfl(static_cast<long long>(upto - mine), l);
            break;
        }
        begin += __shfl(static_cast<long long>(upto), 63);
    }
    b = uniform(b);
    begin = uniform(begin);
    while (w < w_end) {
        const Span seq = span_of(a, b);
        const int length = length_of(a, seq);
        const int64_t of_sequence = static_cast<int64_t>(items_of<R>(a, seq, group)) * length;
        if (w >= begin + of_sequence) {  // its rows are through, or it has none
            begin += of_sequence;
            ++b;
            continue;
        }
        const int item = static_cast<int>((w - begin) / length);
        const int64_t item_begin = begin + static_cast<int64_t>(item) * length;
        // The block's steps of the item.
        const int n0 = max(static_cast<int>(w - item_begin) - kItemCost, 0),
                  n1 = static_cast<int>(min(w_end - item_begin, static_cast<int64_t>(length))) - kItemCost;
        w = min(w_end, item_begin + length);
        if (n0 >= n1) continue;
        const bool whole = n0 == 0 && n1 == length - kItemCost;
        const int share = whole ? 0 : n0 > 0 ? 1 : line.block_of(item_begin + length - 1) - block + 1;
        work(seq, b, item % a.cache.heads, item / a.cache.heads * kRows, n0, n1, share);
    }
}

// Rows whose items several blocks share, joined: a block per row, its threads
// four elements of every (256 / (D / 4))th part each, so that the parts are
// read at once (a wave per row, part after part: 51 us for 64 parts of 32 rows
// of 128).
template <typename T, int NB>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a, int item_rows, const float *__restrict__ parts,
                                                   const Stats *__restrict__ stats,
                                                   const Parts16 *__restrict__ where) {
    constexpr int D = 32 * NB, kQuads = D / 4, kJoinSlots = 256 / kQuads;
    __shared__ float4 sums[kJoinSlots][kQuads];
    __shared__ float totals[kJoinSlots];
    const int quad = threadIdx.x % kQuads, slot = threadIdx.x / kQuads, lane = threadIdx.x & 63;
    int64_t first = 0, end = a.tokens;
    if (a.starts) {  // rows behind the last sequence stay as they are
        first = min(max(static_cast<int64_t>(a.starts[0]), INT64_C(0)), a.tokens);
        end = min(max(static_cast<int64_t>(a.starts[a.sequences]), first), a.tokens);
    }
    for (int64_t row = first * a.q_heads + blockIdx.x; row < end * a.q_heads; row += gridDim.x) {
        const Parts16 at = where[row];
        if (at.parts == 0) continue;
        auto part = [&](int i) { return (2 * static_cast<int64_t>(at.first + i) + (i == 0)) * item_rows + at.row; };
        double m = -INFINITY;
        for (int i = lane; i < at.parts; i += 64) m = fmax(m, stats[part(i)].m);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) m = fmax(m, __shfl_xor(m, o));
        float4 v = make_float4(0, 0, 0, 0);
        float sum = 0;
        if (slot < kJoinSlots) {
#pragma unroll 4
            for (int i = slot; i < at.parts; i += kJoinSlots) {
                const int64_t p = part(i);
                const Stats x = stats[p];
                const float4 y = *reinterpret_cast<const float4 *>(parts + p * D + 4 * quad);
                // A part that saw no key has the lowest maximum, and zeros.
                const float f = factor(x.m, m);
                sum += f * x.sum;
                v.x += f * y.x, v.y += f * y.y, v.z += f * y.z, v.w += f * y.w;
            }
            sums[slot][quad] = v;
            if (quad == 0) totals[slot] = sum;
        }
        __syncthreads();
        if (slot == 0) {
#pragma unroll
            for (int i = 1; i < kJoinSlots; ++i) {
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
    bool own;       // waves have rows of their own
    bool wide;      // else: items of 32 rows
    bool whole;     // that are not cut
    int64_t tiles;  // row tiles of a sequence that the grid covers at once
    int blocks;
    int64_t parts_bytes, stats_bytes, where_bytes;
};

constexpr int kOwnTiles = 2;  // R of waves with rows of their own

// Items of 32 rows convert a step once for twice the rows; the heads for which
// two blocks still fit a compute unit.
template <typename T, int NB>
constexpr bool kWide = kRegisters<T, NB, 2> <= 235 && 2 * kLineLds<NB, 2> <= 163840;

// Blocks of a line that the card holds at once, by their registers and LDS.
template <typename T, int NB, int R>
constexpr int kLineBlocks = 256 * std::min(kLineOccupancy<T, NB, R>, 163840 / kLineLds<NB, R>);

template <typename T, int NB>
Plan plan_of(const AttendArgs &a) {
    Plan p{};
    const int64_t group = a.q_heads / a.cache.heads;
    const int64_t rows = std::max<int64_t>(1, a.most_queries) * group;
    const int64_t seqs = std::max(1, a.sequences), heads = a.cache.heads;
    const int64_t own = (rows + 16 * kOwnTiles - 1) / (16 * kOwnTiles);
    // Rows of their own for two waves of every SIMD; for fewer the line spreads
    // the keys (2 x 512 queries over up to 8000 keys: 139 us for 330, as a line; 4 x 512
    // over 4096 to 8192: 282 for 459; 32 heads of 128 over 8, bf16).
    p.own = rows > 16 && own * heads * seqs >= 2048;
    if (p.own) {
        p.tiles = std::min<int64_t>(own, 1 << 20);
        return p;
    }
    // Few items keep 16 rows, for more blocks: 17 of up to 40 rows over 1000
    // keys in 16 us (20); 512 of 20 rows over up to 4000 take 65 us for 70.
    p.wide = kWide<T, NB> && rows > 16 && (rows + 31) / 32 * heads * seqs >= 128;
    const int64_t item_rows = p.wide ? 32 : 16, items_of = (rows + item_rows - 1) / item_rows;
    p.tiles = items_of;
    p.blocks = kLineBlocks<T, NB, 1>;
    if constexpr (kWide<T, NB>)
        if (p.wide) p.blocks = kLineBlocks<T, NB, 2>;
    // Where an item is short it is not cut, which spares the line's prologue
    // and the launch that joins: one query of 200 keys in 7.5 us (12.8), 16
    // of up to 1000 in 13.1 (15.1), 100 of up to 2000 in 34 (42); but 16 of up
    // to 2000 in 20 (18), one of 4000 in 34 (13) and 64 of up to 8192 in 101
    // (79), 8 heads of keys of 128 in bf16 each.
    const int64_t items = p.tiles * heads * seqs, keys = static_cast<int64_t>(a.width) << a.cache.page_shift;
    p.whole = keys <= 1152 || (keys <= 2304 && 2 * items >= p.blocks) || items >= 8 * p.blocks;
    if (p.whole) {
        p.blocks = static_cast<int>(std::min<int64_t>(items, 1 << 22));
        return p;
    }
    p.parts_bytes = static_cast<int64_t>(p.blocks) * 2 * item_rows * a.cache.dim * 4;
    p.stats_bytes = static_cast<int64_t>(p.blocks) * 2 * item_rows * static_cast<int64_t>(sizeof(Stats));
    p.where_bytes = a.tokens * a.q_heads * static_cast<int64_t>(sizeof(Parts16));
    return p;
}

template <typename T, int NB, int R>
void launch_line(const AttendArgs &a, const Plan &p, char *workspace, hipStream_t stream) {
    const int tiles = static_cast<int>(p.tiles);
    if (p.whole) {
        line_kernel<T, NB, R, true><<<p.blocks, 256, 0, stream>>>(a, tiles, nullptr, nullptr, nullptr);
        return;
    }
    auto *parts = reinterpret_cast<float *>(workspace);
    auto *stats = reinterpret_cast<Stats *>(workspace + p.parts_bytes);
    auto *where = reinterpret_cast<Parts16 *>(workspace + p.parts_bytes + p.stats_bytes);
    line_kernel<T, NB, R, false><<<p.blocks, 256, 0, stream>>>(a, tiles, parts, stats, where);
    const int64_t rows = a.tokens * a.q_heads;
    join_kernel<T, NB>
        <<<static_cast<unsigned>(std::min<int64_t>(rows, 1 << 20)), 256, 0, stream>>>(a, 16 * R, parts, stats, where);
}

template <typename T, int NB>
void launch(const AttendArgs &a, const Plan &p, char *workspace, hipStream_t stream) {
    if (p.own) {
        constexpr int R = sizeof(T) == 4 ? 1 : kOwnTiles;
        const int64_t tiles = (p.tiles * (kOwnTiles / R) + kWaves - 1) / kWaves;  // of 64 R rows
        const int64_t blocks = std::min<int64_t>(tiles * a.cache.heads * a.sequences, 1 << 22);
        rows_kernel<T, NB, R><<<static_cast<unsigned>(blocks), 256, 0, stream>>>(a, static_cast<int>(tiles));
        return;
    }
    if constexpr (kWide<T, NB>)
        if (p.wide) return launch_line<T, NB, 2>(a, p, workspace, stream);
    launch_line<T, NB, 1>(a, p, workspace, stream);
}

// f(type, blocks of a head) of a call.
template <typename F>
auto for_kind(const AttendArgs &a, F f) {
    auto with = [&](auto t) {
        switch (a.cache.dim / 32) {
            case 1: return f(t, std::integral_constant<int, 1>());
            case 2: return f(t, std::integral_constant<int, 2>());
            case 3: return f(t, std::integral_constant<int, 3>());
            case 4: return f(t, std::integral_constant<int, 4>());
            case 5: return f(t, std::integral_constant<int, 5>());
            case 6: return f(t, std::integral_constant<int, 6>());
            case 7: return f(t, std::integral_constant<int, 7>());
            default: return f(t, std::integral_constant<int, 8>());
        }
    };
    return a.bf16 ? with(uint16_t()) : with(float());
}

}  // namespace

int64_t attend_workspace_bytes(const AttendArgs &a) {
    if (a.sequences == 0 || a.tokens == 0) return 0;
    const Plan p = for_kind(a, [&](auto t, auto nb) { return plan_of<decltype(t), nb.value>(a); });
    return p.parts_bytes + p.stats_bytes + p.where_bytes;
}

bool attend_launch(const AttendArgs &a, void *workspace, hipStream_t stream) {
    if (a.sequences == 0 || a.tokens == 0) return true;
    for_kind(a, [&](auto t, auto nb) {
        using T = decltype(t);
        launch<T, nb.value>(a, plan_of<T, nb.value>(a), static_cast<char *>(workspace), stream);
    });
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
