// heads.hip -- queries and keys normed head by head and rotated by their
// positions, and the gradients.
//
// y = R(p) (x r w), r = 1 / sqrt(mean x^2 + eps), R turning the pairs (x_i,
// x_j) of a head's first `rot` elements by p f_i.  Backwards, with g = R(-p)
// dy: dw = sum over tokens and heads of g x r, and dx = r (g w - n mean(g w n)),
// n = x r.  Without w there is no norm: y = R x, dx = g.
//
// Every element is read once and written once.  A head lies in a group of lanes (a power of two), four pairs to a lane, so that a
// rotation stays in a lane and a norm's sum crosses the group alone; a
// block's tokens share their angles, which one thread each works out in
// float64 (a position of 10^6 has 4 digits left of a float32 angle).
// 4 x 2048 tokens of 32 + 8 heads of 128 in bf16: 46 us, 3.6 TB/s of a copy's
// 5.35; without a rotation, and so without angles and their barrier, 45.  The
// gradients take 78 us, 3.5 TB/s, and 5 for the weights' sums.  They keep
// weights and sums in registers over a block's tokens, which at four waves on a
// SIMD leaves 10 of a lane's registers (f32: 14) in memory: 95 MB are written
// for 84 of outputs (weights read anew for each side of queries and keys, which
// spilled as well: 53 and 87 us).  Heads or rotated parts that are no multiples
// of 8 go element by element: 8192 tokens of 40 heads of 80, 20 of them rotated,
// take 64 us, all 80 rotated 34.  A call of 64 tokens takes 8 us (without a
// rotation 7), its latency: angles, then elements, then sums across a group.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "heads.hpp"
#include "mx4_block.hpp"

namespace fgd {
namespace {

constexpr int kThreads = 256;

template <typename T>
struct __attribute__((aligned(4 * sizeof(T)))) Four {
    T e[4];
};

template <typename T>
__device__ inline T rounded(float v) {
    if constexpr (sizeof(T) == 4)
        return v;
    else
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// The elements of pair p of a head.
struct Pairs {
    int half, interleaved;
    __device__ int first(int p) const { return p < half && !interleaved ? p : 2 * p; }
    __device__ int second(int p) const { return p < half && !interleaved ? p + half : 2 * p + 1; }
};

// A lane's four pairs as they lie in memory.  kVec: in vectors of four (the
// launcher checked sizes and alignment).
template <typename T>
struct Raw {
    T u[4], v[4];
};

template <typename T, bool kVec>
__device__ inline void read_pairs(const T *src, int p0, int pairs, const Pairs &at, Raw<T> &r) {
    if constexpr (kVec) {
        const bool apart = p0 < at.half && !at.interleaved;
        const Four<T> u = *reinterpret_cast<const Four<T> *>(src + (apart ? p0 : 2 * p0)),
                      v = *reinterpret_cast<const Four<T> *>(src + (apart ? p0 + at.half : 2 * p0 + 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) r.u[i] = u.e[i], r.v[i] = v.e[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool real = p0 + i < pairs;
            r.u[i] = real ? src[at.first(p0 + i)] : T(0);
            r.v[i] = real ? src[at.second(p0 + i)] : T(0);
        }
    }
}

// a, b: the pairs' first and second elements.
template <typename T, bool kVec>
__device__ inline void to_pairs(const Raw<T> &r, int p0, const Pairs &at, float (&a)[4], float (&b)[4]) {
    const bool apart = !kVec || (p0 < at.half && !at.interleaved);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = widen(apart ? r.u[i] : (i < 2 ? r.u : r.v)[2 * (i & 1)]);
        b[i] = widen(apart ? r.v[i] : (i < 2 ? r.u : r.v)[2 * (i & 1) + 1]);
    }
}

template <typename T, bool kVec>
__device__ inline void store_pairs(T *dst, int p0, int pairs, const Pairs &at, const float (&a)[4],
                                   const float (&b)[4]) {
    if constexpr (kVec) {
        const bool apart = p0 < at.half && !at.interleaved;
        Four<T> u, v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u.e[i] = rounded<T>(apart ? a[i] : i & 1 ? b[i >> 1] : a[i >> 1]);
            v.e[i] = rounded<T>(apart ? b[i] : i & 1 ? b[2 + (i >> 1)] : a[2 + (i >> 1)]);
        }
        *reinterpret_cast<Four<T> *>(dst + (apart ? p0 : 2 * p0)) = u;
        *reinterpret_cast<Four<T> *>(dst + (apart ? p0 + at.half : 2 * p0 + 4)) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p0 + i >= pairs) continue;
            dst[at.first(p0 + i)] = rounded<T>(a[i]);
            dst[at.second(p0 + i)] = rounded<T>(b[i]);
        }
    }
}

__device__ inline float weight_at(const HeadsArgs &g, const HeadSide &s, int64_t m, int d) {
    if (!s.weight) return 1.0f;
    const int64_t i = m * g.weight_stride + d;
    return g.weight_bf16 ? widen(static_cast<const uint16_t *>(s.weight)[i]) : static_cast<const float *>(s.weight)[i];
}

// kGrad: the gradients; a block's part of the weights' gradients goes to
// parts [batch][gridDim.x][2][dim].  A group of lanes reads kAtOnce heads
// before it works on the first (one: 67 us forwards and 166 us backwards at 4
// x 2048 tokens of 40 heads of 128 in bf16).
template <typename T, bool kVec, bool kGrad>
__global__ __launch_bounds__(kThreads, 4) void heads_kernel(HeadsArgs g, int chunk, int lanes_log2, float *parts) {
    constexpr int kAtOnce = kGrad ? 2 : 4;
    extern __shared__ float table[];  // cos, sin of the chunk's tokens and frequencies
    const int lanes = 1 << lanes_log2, groups = kThreads >> lanes_log2;
    const int group = threadIdx.x >> lanes_log2, p0 = 4 * (threadIdx.x & (lanes - 1));
    const int pairs = g.dim / 2;
    const Pairs at = {g.rot / 2, g.interleaved};
    const bool here = p0 < pairs;
    const float per = 1.0f / g.dim;
    for (int64_t m = blockIdx.y; m < g.batch; m += gridDim.y) {
        float wa[2][4], wb[2][4], ga[2][4] = {}, gb[2][4] = {};
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool real = p0 + i < pairs;
                wa[s][i] = real ? weight_at(g, g.side[s], m, at.first(p0 + i)) : 0.0f;
                wb[s][i] = real ? weight_at(g, g.side[s], m, at.second(p0 + i)) : 0.0f;
            }
        for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * chunk; t0 < g.tokens;
             t0 += static_cast<int64_t>(gridDim.x) * chunk) {
            const int n = static_cast<int>(min(static_cast<int64_t>(chunk), g.tokens - t0));
            for (int i = threadIdx.x; i < n * at.half; i += kThreads) {
                const int t = i / at.half;
                // The angle over pi, less whole turns, with the rest of the
                // product: far positions keep the angle's own digits.
                constexpr double kInv = 0.31830988618379067154, kInvRest = -1.9678676675182486e-17;
                const double angle = g.positions[m * g.position_stride + t0 + t] * g.freqs[i - t * at.half];
                const double halves = angle * kInv;
                const double rest = __builtin_fma(angle, kInv, -halves) + angle * kInvRest;
                double sine, cosine;
                sincospi(halves - 2 * rint(0.5 * halves) + rest, &sine, &cosine);
                table[2 * i] = static_cast<float>(cosine);
                table[2 * i + 1] = static_cast<float>(kGrad ? -sine : sine);
            }
            __syncthreads();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const HeadSide &side = g.side[s];
                const int heads = side.heads;
                if (heads == 0) continue;
                const bool norm = side.weight != nullptr;
                auto row = [&](const HeadArray &x, int t, int h) {
                    return static_cast<T *>(x.p) + m * x.batch_stride + (t0 + t) * x.token_stride + h * x.head_stride;
                };
                for (int i = group; i < n * heads; i += kAtOnce * groups) {
                    Raw<T> x[kAtOnce], dy[kGrad ? kAtOnce : 1];
                    int ts[kAtOnce], hs[kAtOnce];
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u) {
                        const int j = i + u * groups;
                        ts[u] = j / heads, hs[u] = j - ts[u] * heads;
                        x[u] = {};
                        if (kGrad) dy[kGrad ? u : 0] = {};
                        if (!here || j >= n * heads) continue;
                        if (norm || !kGrad) read_pairs<T, kVec>(row(side.x, ts[u], hs[u]), p0, pairs, at, x[u]);
                        if constexpr (kGrad) read_pairs<T, kVec>(row(side.dy, ts[u], hs[u]), p0, pairs, at, dy[u]);
                    }
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u) {
                        const int t = ts[u];
                        if (i + u * groups >= n * heads) break;
                        float a[4], b[4];
                        to_pairs<T, kVec>(x[u], p0, at, a, b);
                        float r = 1.0f;
                        if (norm) {
                            float sum = 0;
#pragma unroll
                            for (int j = 0; j < 4; ++j) sum += a[j] * a[j] + b[j] * b[j];
                            for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor(sum, o);
                            r = rsqrtf(sum * per + g.eps);
                        }
                        float c[4], z[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const bool turned = p0 + j < at.half;
                            c[j] = turned ? table[2 * (t * at.half + p0 + j)] : 1.0f;
                            z[j] = turned ? table[2 * (t * at.half + p0 + j) + 1] : 0.0f;
                        }
                        if constexpr (!kGrad) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float v = norm ? a[j] * r * wa[s][j] : a[j],
                                            w = norm ? b[j] * r * wb[s][j] : b[j];
                                a[j] = v * c[j] - w * z[j];
                                b[j] = v * z[j] + w * c[j];
                            }
                        } else {
                            float da[4], db[4], dot = 0;
                            to_pairs<T, kVec>(dy[u], p0, at, da, db);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float v = da[j] * c[j] - db[j] * z[j], w = da[j] * z[j] + db[j] * c[j];
                                da[j] = v, db[j] = w;
                                if (norm) {
                                    a[j] *= r, b[j] *= r;
                                    const float pa = v * a[j], pb = w * b[j];
                                    ga[s][j] += pa;
                                    gb[s][j] += pb;
                                    dot += pa * wa[s][j] + pb * wb[s][j];
                                }
                            }
                            if (norm) {
                                for (int o = 1; o < lanes; o <<= 1) dot += __shfl_xor(dot, o);
                                dot *= per;
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                a[j] = norm ? r * (da[j] * wa[s][j] - a[j] * dot) : da[j];
                                b[j] = norm ? r * (db[j] * wb[s][j] - b[j] * dot) : db[j];
                            }
                        }
                        if (here) store_pairs<T, kVec>(row(side.out, t, hs[u]), p0, pairs, at, a, b);
                    }
                }
            }
            __syncthreads();
        }
        if constexpr (kGrad) {
            if (!parts) continue;
            __shared__ float sums[kThreads][9];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
#pragma unroll
                for (int j = 0; j < 4; ++j) sums[threadIdx.x][j] = ga[w][j], sums[threadIdx.x][4 + j] = gb[w][j];
                __syncthreads();
                float *dst = parts + ((m * gridDim.x + blockIdx.x) * 2 + w) * g.dim;
                for (int i = threadIdx.x; i < 8 * lanes; i += kThreads) {
                    const int lane = i >> 3, j = i & 7, p = 4 * lane + (j & 3);
                    if (p >= pairs) continue;
                    float v = 0;
                    for (int q = 0; q < groups; ++q) v += sums[q * lanes + lane][j];
                    dst[j < 4 ? at.first(p) : at.second(p)] = v;
                }
                __syncthreads();
            }
        }
    }
}

// The sums of the blocks' parts, in their order: 32 elements of one weight a
// block, 32 threads to an element.
__global__ __launch_bounds__(1024) void weights_kernel(HeadsArgs g, const float *__restrict__ parts, int64_t count) {
    __shared__ double sums[32][33];
    const int col = threadIdx.x & 31, slot = threadIdx.x >> 5, d = blockIdx.x * 32 + col, s = blockIdx.y;
    float *out = g.side[s].weight_grad;
    if (!out) return;
    const int64_t of = blockIdx.z;  // which batch entry's weight
    double v = 0;
    if (d < g.dim) {
        const float *src = parts + (of * count * 2 + s) * g.dim + d;
#pragma unroll 8
        for (int64_t i = slot; i < count; i += 32) v += src[i * 2 * g.dim];
    }
    sums[slot][col] = v;
    __syncthreads();
    if (slot == 0 && d < g.dim) {
        for (int i = 1; i < 32; ++i) v += sums[i][col];
        out[of * g.dim + d] = static_cast<float>(v);
    }
}

int lanes_log2_of(int dim) {
    int n = 0;
    while ((8 << n) < dim) ++n;
    return n;
}

bool four_aligned(const HeadArray &x, size_t es) {
    return reinterpret_cast<uintptr_t>(x.p) % (4 * es) == 0 && x.batch_stride % 4 == 0 && x.token_stride % 4 == 0 &&
           x.head_stride % 4 == 0;
}

bool vectors_of(const HeadsArgs &a, bool grad) {
    if (a.dim % 8 || a.rot % 8) return false;
    const size_t es = a.bf16 ? 2 : 4;
    for (const HeadSide &s : a.side) {
        if (s.heads == 0) continue;
        if (!four_aligned(s.out, es) || ((s.weight || !grad) && !four_aligned(s.x, es)) ||
            (grad && !four_aligned(s.dy, es)))
            return false;
    }
    return true;
}

// Tokens of a block at a time: eight, whose angles are then worked out
// together, where that leaves four blocks for a compute unit; of shorter calls
// as many as fill its lanes once, where that leaves one; angles of 32 KB.
int chunk_of(const HeadsArgs &a) {
    const int64_t heads = std::max(1, a.side[0].heads + a.side[1].heads), all = a.tokens * a.batch;
    const int64_t fill = (2 * (kThreads >> lanes_log2_of(a.dim)) + heads - 1) / heads;
    const int64_t most = a.rot ? 4096 / (a.rot / 2) : 8;
    return static_cast<int>(
        std::clamp<int64_t>(std::max(all / 1024, std::min(fill, all / 256)), 1, std::min<int64_t>(most, 8)));
}

// Blocks per batch entry of the gradients: their parts are few enough to sum at once.
int64_t grad_blocks(const HeadsArgs &a) {
    const int64_t chunk = chunk_of(a);
    return std::max<int64_t>(1, std::min((a.tokens + chunk - 1) / chunk, std::max<int64_t>(1, 1024 / std::max<int64_t>(1, a.batch))));
}

template <typename T, bool kGrad>
void launch(const HeadsArgs &a, dim3 grid, int chunk, float *parts, hipStream_t stream) {
    const size_t lds = static_cast<size_t>(chunk) * (a.rot / 2) * 8;
    const int lanes = lanes_log2_of(a.dim);
    if (vectors_of(a, kGrad))
        heads_kernel<T, true, kGrad><<<grid, kThreads, lds, stream>>>(a, chunk, lanes, parts);
    else
        heads_kernel<T, false, kGrad><<<grid, kThreads, lds, stream>>>(a, chunk, lanes, parts);
}

}  // namespace

bool rotate_heads_launch(const HeadsArgs &a, hipStream_t stream) {
    if (a.batch == 0 || a.tokens == 0 || a.side[0].heads + a.side[1].heads == 0) return true;
    const int chunk = chunk_of(a);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((a.tokens + chunk - 1) / chunk, 1 << 22)),
                    static_cast<unsigned>(std::min<int64_t>(a.batch, 65535)));
    if (a.bf16)
        launch<uint16_t, false>(a, grid, chunk, nullptr, stream);
    else
        launch<float, false>(a, grid, chunk, nullptr, stream);
    return hipGetLastError() == hipSuccess;
}

int64_t rotate_heads_grads_workspace_bytes(const HeadsArgs &a) {
    if (!a.side[0].weight && !a.side[1].weight) return 0;
    return a.batch * grad_blocks(a) * 2 * a.dim * 4;
}

bool rotate_heads_grads_launch(const HeadsArgs &a, float *workspace, hipStream_t stream) {
    const bool weights = a.side[0].weight || a.side[1].weight;
    const int64_t blocks = grad_blocks(a);
    if (a.batch > 0 && a.tokens > 0 && a.side[0].heads + a.side[1].heads > 0) {
        const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(std::min<int64_t>(a.batch, 65535)));
        float *parts = weights ? workspace : nullptr;
        if (a.bf16)
            launch<uint16_t, true>(a, grid, chunk_of(a), parts, stream);
        else
            launch<float, true>(a, grid, chunk_of(a), parts, stream);
        if (hipGetLastError() != hipSuccess) return false;
    }
    if (!weights) return true;
    // Weights of their own: a batch entry's blocks; shared ones: all blocks.
    const int64_t outs = a.weight_stride ? a.batch : 1;
    const bool empty = a.tokens == 0 || a.batch == 0 || a.side[0].heads + a.side[1].heads == 0;
    const int64_t count = empty ? 0 : a.weight_stride ? blocks : blocks * a.batch;
    for (int64_t z = 0; z < outs; z += 65535) {
        HeadsArgs part = a;
        for (HeadSide &s : part.side)
            if (s.weight_grad) s.weight_grad += z * a.dim;
        weights_kernel<<<dim3((a.dim + 31) / 32, 2, static_cast<unsigned>(std::min<int64_t>(outs - z, 65535))), 1024, 0,
                         stream>>>(part, workspace + (empty ? 0 : z * count * 2 * a.dim), count);
    }
    return hipGetLastError() == hipSuccess;
}

}  // namespace fgd
