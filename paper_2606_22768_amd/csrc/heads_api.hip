// heads_api.hip -- the C ABI of norming and rotating heads: argument checks
// and launches of the kernels in heads.hip.  No engine is involved; the calls
// run on the caller's current device.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "../../include/fgd.h"
#include "api_args.hpp"
#include "heads.hpp"

namespace {

using fgd::api_fail;

fgd_status check_sizes(const fgd_heads *s) {
    if (!s || s->struct_size != sizeof(fgd_heads))
        return api_fail(FGD_ERR_INVALID_ARG, "heads: NULL or of another size");
    if (fgd_status st = fgd::api_check_dtype(s->dtype)) return st;
    if (fgd_status st = fgd::api_check_dtype(s->weight_dtype)) return st;
    if (s->batch < 0 || s->tokens < 0 || s->q_heads < 0 || s->k_heads < 0)
        return api_fail(FGD_ERR_INVALID_ARG, "heads: negative size");
    if (s->head_dim < 2 || s->head_dim > FGD_MAX_HEAD_DIM || s->head_dim % 2)
        return api_fail(FGD_ERR_INVALID_ARG, "head_dim must be even and in [2, %d], got %d", FGD_MAX_HEAD_DIM,
                        s->head_dim);
    if (s->rot_dim < 0 || s->rot_dim > s->head_dim || s->rot_dim % 2)
        return api_fail(FGD_ERR_INVALID_ARG, "rot_dim must be even and in [0, head_dim], got %d", s->rot_dim);
    if (s->interleaved != 0 && s->interleaved != 1)
        return api_fail(FGD_ERR_INVALID_ARG, "interleaved must be 0 or 1");
    if (!(s->eps >= 0) || isinf(s->eps)) return api_fail(FGD_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (s->position_stride != 0 && s->position_stride < s->tokens)
        return api_fail(FGD_ERR_INVALID_ARG, "position_stride must be 0 or at least tokens");
    if (s->weight_stride != 0 && s->weight_stride < s->head_dim)
        return api_fail(FGD_ERR_INVALID_ARG, "weight_stride must be 0 or at least head_dim");
    const fgd::wide all = static_cast<fgd::wide>(s->batch) * s->tokens *
                          (static_cast<int64_t>(s->q_heads) + s->k_heads + 1) * s->head_dim;
    const fgd::wide strides = static_cast<fgd::wide>(s->batch) *
                              (static_cast<fgd::wide>(s->position_stride) + s->weight_stride);
    if (static_cast<int64_t>(s->q_heads) + s->k_heads > FGD_MAX_HEADS || all >= fgd::kMostBytes / 8 ||
        strides >= fgd::kMostBytes / 8)
        return api_fail(FGD_ERR_INVALID_ARG, "heads: sizes are too large");
    return FGD_OK;
}

struct Spans {
    const void *p[16];
    int64_t n[16];
    int count = 0;
    void add(const void *q, int64_t bytes) { p[count] = q, n[count++] = bytes; }
};

fgd::HeadArray array_of(const void *p, const int64_t *strides) {
    return p ? fgd::HeadArray{const_cast<void *>(p), strides[0], strides[1], strides[2]} : fgd::HeadArray{};
}

fgd_status check_one(const char *what, const fgd_heads *s, int heads, const void *p, const int64_t *strides, bool output,
                     int64_t *bytes) {
    *bytes = 0;
    if (s->batch == 0 || s->tokens == 0 || heads == 0) return FGD_OK;
    if (!strides) return api_fail(FGD_ERR_INVALID_ARG, "%s: NULL strides", what);
    return fgd::api_check_heads(what, p, s->dtype, s->batch, s->tokens, heads, s->head_dim, strides[0], strides[1],
                                strides[2], output, bytes);
}

// Whether an element of q is one of k, which differ in their heads only: views
// of one array, whose spans may overlap and whose elements lie between each
// other.  Arrays that do not step alike count as meeting where their spans do.
bool heads_meet(const fgd_heads *s, const void *q, const int64_t *x, int64_t qb, const void *k, const int64_t *y,
                int64_t kb) {
    if (!fgd::api_overlap(q, qb, k, kb)) return false;
    const int64_t D = s->head_dim, n[2] = {s->batch, s->tokens};
    if ((n[0] > 1 && x[0] != y[0]) || (n[1] > 1 && x[1] != y[1]) || (s->q_heads + s->k_heads > 2 && x[2] != y[2]))
        return true;
    const int big = n[0] > 1 && (n[1] == 1 || x[0] >= x[1]) ? 0 : 1;
    const int64_t from = (static_cast<const char *>(k) - static_cast<const char *>(q)) / fgd::api_elem_size(s->dtype);
    // v less a number of steps of an axis, the one that leaves 0 or more or the next.
    auto less = [&](int64_t v, int axis, int64_t up) {
        if (n[axis] <= 1 || x[axis] == 0) return v;
        const int64_t whole = v >= 0 ? v / x[axis] : -((-v + x[axis] - 1) / x[axis]);
        const int64_t steps = whole + up, most = n[axis] - 1;
        return v - (steps < -most ? -most : steps > most ? most : steps) * x[axis];
    };
    for (int64_t h = 1 - s->q_heads; h < s->k_heads; ++h)
        for (int i = 0; i < 4; ++i) {
            const int64_t v = less(less(from + h * x[2], big, i & 1), 1 - big, i >> 1);
            if (v < D && v > -D) return true;
        }
    return false;
}

// That no output overlaps an input or another output.  `pair`: the first two
// are those of q and k and have been compared by their elements.
fgd_status check_apart(const Spans &in, const Spans &out, bool pair) {
    for (int i = 0; i < out.count; ++i) {
        for (int j = 0; j < in.count; ++j)
            if (fgd::api_overlap(out.p[i], out.n[i], in.p[j], in.n[j]))
                return api_fail(FGD_ERR_INVALID_ARG, "outputs and the workspace must not overlap the inputs");
        for (int j = pair && i == 1 ? 1 : 0; j < i; ++j)
            if (fgd::api_overlap(out.p[i], out.n[i], out.p[j], out.n[j]))
                return api_fail(FGD_ERR_INVALID_ARG, "outputs and the workspace must not overlap each other");
    }
    return FGD_OK;
}

// The inputs that both calls have besides their heads.
fgd_status check_common(const fgd_heads *s, const int32_t *positions, const double *freqs, const void *q_weight,
                        const void *k_weight, Spans *in) {
    const bool work = s->batch > 0 && s->tokens > 0 && s->q_heads + s->k_heads > 0;
    const int ws = fgd::api_elem_size(s->weight_dtype);
    if (work && s->rot_dim > 0) {
        if (fgd_status st = fgd::api_check_array("positions", positions, s->tokens, 4)) return st;
        if (fgd_status st = fgd::api_check_array("freqs", freqs, s->rot_dim / 2, 8)) return st;
        in->add(positions, ((s->batch - 1) * s->position_stride + s->tokens) * 4);
        in->add(freqs, static_cast<int64_t>(s->rot_dim) * 4);
    }
    for (const void *w : {q_weight, k_weight})
        if (w && !fgd::api_aligned(w, ws))
            return api_fail(FGD_ERR_INVALID_ARG, "weights must be aligned to their element size");
    const int64_t span = (s->batch > 0 ? (s->batch - 1) * s->weight_stride + s->head_dim : 0) * ws;
    in->add(q_weight, span);
    in->add(k_weight, span);
    return FGD_OK;
}

fgd::HeadsArgs args_of(const fgd_heads *s, const int32_t *positions, const double *freqs, const void *q_weight,
                       const void *k_weight) {
    fgd::HeadsArgs a{};
    a.positions = positions;
    a.freqs = freqs;
    a.batch = s->batch;
    a.tokens = s->tokens;
    a.position_stride = s->position_stride;
    a.weight_stride = s->weight_stride;
    a.dim = s->head_dim;
    a.rot = s->rot_dim;
    a.eps = s->eps;
    a.interleaved = s->interleaved != 0;
    a.bf16 = s->dtype == FGD_BF16;
    a.weight_bf16 = s->weight_dtype == FGD_BF16;
    a.side[0].heads = s->q_heads;
    a.side[1].heads = s->k_heads;
    a.side[0].weight = q_weight;
    a.side[1].weight = k_weight;
    return a;
}

}  // namespace

extern "C" {

fgd_status fgd_rotate_heads(const fgd_heads *sizes, const void *q, const int64_t *q_strides, const void *k,
                            const int64_t *k_strides, const int32_t *positions, const double *freqs,
                            const void *q_weight, const void *k_weight, void *q_out, const int64_t *q_out_strides,
                            void *k_out, const int64_t *k_out_strides, void *stream) {
    fgd::api_clear();
    if (fgd_status st = check_sizes(sizes)) return st;
    int64_t qb, kb, qob, kob;
    if (fgd_status st = check_one("q", sizes, sizes->q_heads, q, q_strides, false, &qb)) return st;
    if (fgd_status st = check_one("k", sizes, sizes->k_heads, k, k_strides, false, &kb)) return st;
    if (fgd_status st = check_one("q_out", sizes, sizes->q_heads, q_out, q_out_strides, true, &qob)) return st;
    if (fgd_status st = check_one("k_out", sizes, sizes->k_heads, k_out, k_out_strides, true, &kob)) return st;
    Spans in, out;
    if (fgd_status st = check_common(sizes, positions, freqs, q_weight, k_weight, &in)) return st;
    auto same = [](const void *a, const int64_t *x, const void *b, const int64_t *y, int64_t n) {
        return n > 0 && a == b && x[0] == y[0] && x[1] == y[1] && x[2] == y[2];
    };
    // In place, views of one projection interleave: their spans overlap, their elements do not.
    const bool q_same = same(q, q_strides, q_out, q_out_strides, qb), k_same = same(k, k_strides, k_out, k_out_strides, kb);
    if ((q_same || k_same) && heads_meet(sizes, q, q_strides, qb, k, k_strides, kb))
        return api_fail(FGD_ERR_INVALID_ARG, "in place q and k must not share elements");
    const int common = in.count;
    if (!q_same) out.add(q_out, qob);
    if (!k_same) out.add(k_out, kob);
    if (!q_same || !k_same) {
        in.add(q, qb);
        in.add(k, kb);
    }
    const bool pair = out.count == 2 && !heads_meet(sizes, q_out, q_out_strides, qob, k_out, k_out_strides, kob);
    if (fgd_status st = check_apart(in, out, pair)) return st;
    if (q_same || k_same) {
        Spans written, rest;
        if (q_same) written.add(q_out, qob);
        if (k_same) written.add(k_out, kob);
        for (int i = 0; i < common; ++i) rest.add(in.p[i], in.n[i]);
        for (int i = 0; i < written.count; ++i)
            for (int j = 0; j < rest.count; ++j)
                if (fgd::api_overlap(written.p[i], written.n[i], rest.p[j], rest.n[j]))
                    return api_fail(FGD_ERR_INVALID_ARG, "outputs and the workspace must not overlap the inputs");
    }
    fgd::HeadsArgs a = args_of(sizes, positions, freqs, q_weight, k_weight);
    a.side[0].x = array_of(qb ? q : nullptr, q_strides);
    a.side[1].x = array_of(kb ? k : nullptr, k_strides);
    a.side[0].out = array_of(qob ? q_out : nullptr, q_out_strides);
    a.side[1].out = array_of(kob ? k_out : nullptr, k_out_strides);
    if (!fgd::rotate_heads_launch(a, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "head rotation launch failed");
    return FGD_OK;
}

fgd_status fgd_rotate_heads_grads_workspace_size(const fgd_heads *sizes, int64_t *bytes) {
    fgd::api_clear();
    if (!bytes) return api_fail(FGD_ERR_INVALID_ARG, "NULL bytes");
    if (fgd_status st = check_sizes(sizes)) return st;
    fgd::HeadsArgs a = args_of(sizes, nullptr, nullptr, sizes, sizes);
    *bytes = fgd::rotate_heads_grads_workspace_bytes(a);
    return FGD_OK;
}

fgd_status fgd_rotate_heads_grads(const fgd_heads *sizes, const void *dq, const int64_t *dq_strides, const void *dk,
                                  const int64_t *dk_strides, const void *q, const int64_t *q_strides, const void *k,
                                  const int64_t *k_strides, const int32_t *positions, const double *freqs,
                                  const void *q_weight, const void *k_weight, void *q_grad,
                                  const int64_t *q_grad_strides, void *k_grad, const int64_t *k_grad_strides,
                                  float *q_weight_grad, float *k_weight_grad, void *workspace,
                                  int64_t workspace_bytes, void *stream) {
    fgd::api_clear();
    if (fgd_status st = check_sizes(sizes)) return st;
    int64_t dqb, dkb, qb = 0, kb = 0, qob, kob;
    if (fgd_status st = check_one("dq", sizes, sizes->q_heads, dq, dq_strides, false, &dqb)) return st;
    if (fgd_status st = check_one("dk", sizes, sizes->k_heads, dk, dk_strides, false, &dkb)) return st;
    if (q_weight)  // without a norm nothing is needed of q but its gradient
        if (fgd_status st = check_one("q", sizes, sizes->q_heads, q, q_strides, false, &qb)) return st;
    if (k_weight)
        if (fgd_status st = check_one("k", sizes, sizes->k_heads, k, k_strides, false, &kb)) return st;
    if (fgd_status st = check_one("q_grad", sizes, sizes->q_heads, q_grad, q_grad_strides, true, &qob)) return st;
    if (fgd_status st = check_one("k_grad", sizes, sizes->k_heads, k_grad, k_grad_strides, true, &kob)) return st;
    Spans in, out;
    if (fgd_status st = check_common(sizes, positions, freqs, q_weight, k_weight, &in)) return st;
    if ((q_weight != nullptr) != (q_weight_grad != nullptr) || (k_weight != nullptr) != (k_weight_grad != nullptr))
        return api_fail(FGD_ERR_INVALID_ARG, "a weight and its gradient must be given together");
    if (!fgd::api_aligned(q_weight_grad, 4) || !fgd::api_aligned(k_weight_grad, 4) || !fgd::api_aligned(workspace, 16))
        return api_fail(FGD_ERR_INVALID_ARG,
                        "arrays must be aligned to their element size and the workspace to 16 bytes");
    fgd::HeadsArgs a = args_of(sizes, positions, freqs, q_weight, k_weight);
    const int64_t need = fgd::rotate_heads_grads_workspace_bytes(a);
    if (workspace_bytes < need || (need > 0 && !workspace))
        return api_fail(FGD_ERR_INVALID_ARG, "workspace of %lld bytes is below the %lld this call needs",
                        static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    const int64_t grads = (sizes->weight_stride ? static_cast<int64_t>(sizes->batch) : 1) * sizes->head_dim * 4;
    in.add(dq, dqb);
    in.add(dk, dkb);
    in.add(q, qb);
    in.add(k, kb);
    out.add(q_grad, qob);
    out.add(k_grad, kob);
    out.add(q_weight_grad, grads);
    out.add(k_weight_grad, grads);
    out.add(workspace, need);
    const bool pair = !heads_meet(sizes, q_grad, q_grad_strides, qob, k_grad, k_grad_strides, kob);
    if (fgd_status st = check_apart(in, out, pair)) return st;
    a.side[0].x = array_of(qb ? q : nullptr, q_strides);
    a.side[1].x = array_of(kb ? k : nullptr, k_strides);
    a.side[0].dy = array_of(dqb ? dq : nullptr, dq_strides);
    a.side[1].dy = array_of(dkb ? dk : nullptr, dk_strides);
    a.side[0].out = array_of(qob ? q_grad : nullptr, q_grad_strides);
    a.side[1].out = array_of(kob ? k_grad : nullptr, k_grad_strides);
    a.side[0].weight_grad = q_weight_grad;
    a.side[1].weight_grad = k_weight_grad;
    if (!fgd::rotate_heads_grads_launch(a, static_cast<float *>(workspace), static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "head rotation gradients launch failed");
    return FGD_OK;
}

}  // extern "C"
