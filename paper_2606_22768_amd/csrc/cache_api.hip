// cache_api.hip -- the C ABI of the paged 4-bit cache, of attention over it
// and of its pages: argument checks and launches of the kernels in cache.hip,
// attend.hip and pages.hip.  No engine is involved; the calls run on the
// caller's current device.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "../../include/fgd.h"
#include "api_args.hpp"
#include "cache.hpp"
#include "pages.hpp"

namespace {

using fgd::api_fail;

fgd_status check_cache(const fgd_mx4_cache *c, fgd::CacheView *view, int64_t *bytes, bool data) {
    if (!c || c->struct_size != sizeof(fgd_mx4_cache))
        return api_fail(FGD_ERR_INVALID_ARG, "cache: NULL or of another size");
    if (c->pages < 0 || c->heads < 1 || c->heads > FGD_MAX_HEADS)
        return api_fail(FGD_ERR_INVALID_ARG, "cache: pages must not be negative and heads must be in [1, %d]",
                        FGD_MAX_HEADS);
    if (c->page < 16 || c->page > 65536 || (c->page & (c->page - 1)))
        return api_fail(FGD_ERR_INVALID_ARG, "cache: page must be a power of two in [16, 65536], got %d", c->page);
    if (c->head_dim < 32 || c->head_dim > 256 || c->head_dim % 32)
        return api_fail(FGD_ERR_INVALID_ARG, "cache: head_dim must be a multiple of 32 in [32, 256], got %d",
                        c->head_dim);
    if (c->reserved != 0) return api_fail(FGD_ERR_INVALID_ARG, "cache: reserved must be 0");
    if (c->pages > INT32_MAX ||
        static_cast<fgd::wide>(c->pages) * c->page * c->heads * c->head_dim >= fgd::kMostBytes / 2)
        return api_fail(FGD_ERR_INVALID_ARG, "cache: sizes are too large");
    int shift = 0;
    while ((1 << shift) < c->page) ++shift;
    *view = {static_cast<uint8_t *>(c->data), c->pages, c->heads, c->head_dim, shift};
    *bytes = view->group(c->pages, 0, 0);
    if (!data || *bytes == 0) return FGD_OK;
    if (!c->data) return api_fail(FGD_ERR_INVALID_ARG, "cache: NULL array");
    if (!fgd::api_aligned(c->data, 16)) return api_fail(FGD_ERR_INVALID_ARG, "cache: data must be 16-byte aligned");
    return FGD_OK;
}

fgd_status check_tokens(int32_t dtype, int64_t tokens) {
    if (fgd_status st = fgd::api_check_dtype(dtype)) return st;
    if (tokens < 0 || tokens > INT32_MAX) return api_fail(FGD_ERR_INVALID_ARG, "tokens must be in [0, 2^31)");
    return FGD_OK;
}

fgd_status check_apart(const char *what, const void *out, int64_t n, const void *in, int64_t m) {
    if (fgd::api_overlap(out, n, in, m)) return api_fail(FGD_ERR_INVALID_ARG, "%s must not overlap", what);
    return FGD_OK;
}

// Keys and values of a write (into the cache) or a read (out of it).
fgd_status check_rows(const fgd_mx4_cache *cache, const void *k, int64_t kt, int64_t kh, const void *v, int64_t vt,
                      int64_t vh, int32_t dtype, int64_t tokens, const int64_t *slots, bool output,
                      fgd::CacheView *view) {
    int64_t bytes, kb, vb;
    if (fgd_status st = check_cache(cache, view, &bytes, true)) return st;
    if (fgd_status st = check_tokens(dtype, tokens)) return st;
    const int H = view->heads, D = view->dim;
    if (fgd_status st = fgd::api_check_heads("k", k, dtype, 1, tokens, H, D, 0, kt, kh, output, &kb)) return st;
    if (fgd_status st = fgd::api_check_heads("v", v, dtype, 1, tokens, H, D, 0, vt, vh, output, &vb)) return st;
    if (fgd_status st = fgd::api_check_array("slots", slots, tokens, 8)) return st;
    if (fgd_status st = check_apart("the cache and k, v and slots", cache->data, bytes, k, kb)) return st;
    if (fgd_status st = check_apart("the cache and k, v and slots", cache->data, bytes, v, vb)) return st;
    if (fgd_status st = check_apart("the cache and k, v and slots", cache->data, bytes, slots, tokens * 8)) return st;
    if (output) {
        if (fgd_status st = check_apart("k and v", k, kb, v, vb)) return st;
        if (fgd_status st = check_apart("k and slots", k, kb, slots, tokens * 8)) return st;
        if (fgd_status st = check_apart("v and slots", v, vb, slots, tokens * 8)) return st;
    }
    return FGD_OK;
}

fgd_status check_attention(const fgd_mx4_cache *cache, const fgd_attention *s, bool data, fgd::AttendArgs *a,
                           int64_t *cache_bytes) {
    if (!s || s->struct_size != sizeof(fgd_attention))
        return api_fail(FGD_ERR_INVALID_ARG, "attention: NULL or of another size");
    *a = {};
    if (fgd_status st = check_cache(cache, &a->cache, cache_bytes, data)) return st;
    if (fgd_status st = check_tokens(s->dtype, s->tokens)) return st;
    if (s->sequences < 0 || s->table_width < 0) return api_fail(FGD_ERR_INVALID_ARG, "attention: negative size");
    if (s->q_heads < 1 || s->q_heads > FGD_MAX_HEADS || s->q_heads % cache->heads)
        return api_fail(FGD_ERR_INVALID_ARG, "q_heads must be a multiple of the cache's %d heads in [1, %d], got %d",
                        cache->heads, FGD_MAX_HEADS, s->q_heads);
    if (s->reserved != 0) return api_fail(FGD_ERR_INVALID_ARG, "attention: reserved must be 0");
    if (s->most_queries < 0) return api_fail(FGD_ERR_INVALID_ARG, "most_queries must not be negative");
    if (s->window < 0) return api_fail(FGD_ERR_INVALID_ARG, "window must not be negative");
    if (!(s->scale > 0) || isinf(s->scale))
        return api_fail(FGD_ERR_INVALID_ARG, "scale must be finite and above 0");
    if (static_cast<int64_t>(s->table_width) * cache->page > INT32_MAX - 63)
        return api_fail(FGD_ERR_INVALID_ARG, "table_width times page must be at most 2^31 - 64");
    if (cache->pages == 0 && s->table_width > 0)
        return api_fail(FGD_ERR_INVALID_ARG, "a cache without pages has tables of width 0 only");
    if (s->tokens * s->q_heads > INT32_MAX - 4095)
        return api_fail(FGD_ERR_INVALID_ARG, "attention: tokens times q_heads must be at most 2^31 - 4096");
    a->tokens = s->tokens;
    a->sequences = s->sequences;
    a->width = s->table_width;
    a->q_heads = s->q_heads;
    a->most_queries = static_cast<int32_t>(s->most_queries < s->tokens ? s->most_queries : s->tokens);
    a->window = s->window;
    a->scale = s->scale;
    a->bf16 = s->dtype == FGD_BF16;
    return FGD_OK;
}

fgd_status check_pages(const fgd_pages *s, fgd::PagesView *p) {
    if (!s || s->struct_size != sizeof(fgd_pages))
        return api_fail(FGD_ERR_INVALID_ARG, "pages: NULL or of another size");
    if (s->requests < 0 || s->table_width < 0 || s->capacity < 0)
        return api_fail(FGD_ERR_INVALID_ARG, "pages: negative size");
    if (s->reserved != 0) return api_fail(FGD_ERR_INVALID_ARG, "pages: reserved must be 0");
    if (s->page < 1 || s->page > 65536)
        return api_fail(FGD_ERR_INVALID_ARG, "page must be in [1, 65536], got %d", s->page);
    if (s->table_stride < s->table_width && s->requests > 1)
        return api_fail(FGD_ERR_INVALID_ARG, "table_stride is below table_width");
    if (static_cast<fgd::wide>(s->table_stride) * s->requests >= fgd::kMostBytes / 8 ||
        static_cast<int64_t>(s->table_width) * s->requests > INT32_MAX)
        return api_fail(FGD_ERR_INVALID_ARG, "pages: sizes are too large");
    const bool table = s->requests > 0 && s->table_width > 0;
    if (fgd_status st = fgd::api_check_array("tables", s->tables, table, 4)) return st;
    if (fgd_status st = fgd::api_check_array("lengths", s->lengths, s->requests, 4)) return st;
    if (fgd_status st = fgd::api_check_array("free", s->free, s->capacity, 4)) return st;
    if (fgd_status st = fgd::api_check_array("free_count", s->free_count, 1, 4)) return st;
    *p = {s->tables,   s->lengths,     s->free, s->free_count, s->table_stride,
          s->requests, s->table_width, s->page, s->capacity};
    return FGD_OK;
}

struct Span {
    const void *p;
    int64_t n;
};

// The state's arrays, and further ones, none of which may overlap another.
template <int N>
fgd_status check_state_apart(const fgd_pages *s, const Span (&more)[N]) {
    const int64_t table = s->requests > 0 && s->table_width > 0
                              ? (s->table_stride * (s->requests - 1) + s->table_width) * 4
                              : 0;
    const Span own[] = {{s->tables, table},
                        {s->lengths, s->requests * INT64_C(4)},
                        {s->free, s->capacity * INT64_C(4)},
                        {s->free_count, 4}};
    Span all[4 + N];
    for (int i = 0; i < 4 + N; ++i) {
        all[i] = i < 4 ? own[i] : more[i - 4];
        for (int j = 0; j < i; ++j)
            if (fgd::api_overlap(all[i].p, all[i].n, all[j].p, all[j].n))
                return api_fail(FGD_ERR_INVALID_ARG, "pages: arrays must not overlap");
    }
    return FGD_OK;
}

}  // namespace

extern "C" {

fgd_status fgd_mx4_cache_size(const fgd_mx4_cache *cache, int64_t *bytes) {
    fgd::api_clear();
    if (!bytes) return api_fail(FGD_ERR_INVALID_ARG, "NULL bytes");
    fgd::CacheView view;
    return check_cache(cache, &view, bytes, false);
}

fgd_status fgd_mx4_cache_write(const fgd_mx4_cache *cache, const void *k, int64_t k_token_stride,
                               int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride,
                               int32_t dtype, int64_t tokens, const int64_t *slots, void *stream) {
    fgd::api_clear();
    fgd::CacheView view;
    if (fgd_status st = check_rows(cache, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, dtype,
                                   tokens, slots, false, &view))
        return st;
    if (view.pages == 0) return FGD_OK;
    if (!fgd::cache_write_launch(view, {const_cast<void *>(k), k_token_stride, k_head_stride},
                                 {const_cast<void *>(v), v_token_stride, v_head_stride}, dtype == FGD_BF16, tokens,
                                 slots, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "cache write launch failed");
    return FGD_OK;
}

fgd_status fgd_mx4_cache_read(const fgd_mx4_cache *cache, const int64_t *slots, int64_t tokens, void *k,
                              int64_t k_token_stride, int64_t k_head_stride, void *v, int64_t v_token_stride,
                              int64_t v_head_stride, int32_t dtype, void *stream) {
    fgd::api_clear();
    fgd::CacheView view;
    if (fgd_status st = check_rows(cache, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, dtype,
                                   tokens, slots, true, &view))
        return st;
    if (!fgd::cache_read_launch(view, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride},
                                dtype == FGD_BF16, tokens, slots, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "cache read launch failed");
    return FGD_OK;
}

fgd_status fgd_mx4_attend_workspace_size(const fgd_mx4_cache *cache, const fgd_attention *sizes, int64_t *bytes) {
    fgd::api_clear();
    if (!bytes) return api_fail(FGD_ERR_INVALID_ARG, "NULL bytes");
    fgd::AttendArgs a;
    int64_t cache_bytes;
    if (fgd_status st = check_attention(cache, sizes, false, &a, &cache_bytes)) return st;
    *bytes = fgd::attend_workspace_bytes(a);
    return FGD_OK;
}

fgd_status fgd_mx4_attend(const fgd_mx4_cache *cache, const fgd_attention *sizes, const void *q,
                          int64_t q_token_stride, int64_t q_head_stride, const int32_t *tables, int64_t table_stride,
                          const int32_t *lengths, const int32_t *starts, void *out, int64_t out_token_stride,
                          int64_t out_head_stride, void *workspace, int64_t workspace_bytes, void *stream) {
    fgd::api_clear();
    fgd::AttendArgs a;
    int64_t cache_bytes, qb, ob;
    if (fgd_status st = check_attention(cache, sizes, true, &a, &cache_bytes)) return st;
    if (!starts && sizes->tokens != sizes->sequences)
        return api_fail(FGD_ERR_INVALID_ARG, "without starts there is one query per sequence");
    const int D = a.cache.dim, B = sizes->sequences;
    if (fgd_status st = fgd::api_check_heads("q", q, sizes->dtype, 1, sizes->tokens, sizes->q_heads, D, 0,
                                             q_token_stride, q_head_stride, false, &qb))
        return st;
    if (fgd_status st = fgd::api_check_heads("out", out, sizes->dtype, 1, sizes->tokens, sizes->q_heads, D, 0,
                                             out_token_stride, out_head_stride, true, &ob))
        return st;
    if (B > 1 && table_stride < sizes->table_width)
        return api_fail(FGD_ERR_INVALID_ARG, "table_stride is below table_width");
    if (B > 0 && static_cast<fgd::wide>(table_stride) * B >= fgd::kMostBytes / 8)
        return api_fail(FGD_ERR_INVALID_ARG, "tables: strides are too large");
    const int64_t table_bytes =
        B > 0 && sizes->table_width > 0 ? (table_stride * (B - 1) + sizes->table_width) * 4 : 0;
    if (fgd_status st = fgd::api_check_array("tables", tables, table_bytes, 4)) return st;
    if (fgd_status st = fgd::api_check_array("lengths", lengths, B, 4)) return st;
    if (starts)
        if (fgd_status st = fgd::api_check_array("starts", starts, B + INT64_C(1), 4)) return st;
    const int64_t need = fgd::attend_workspace_bytes(a);
    if (!fgd::api_aligned(workspace, 16))
        return api_fail(FGD_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
    if (workspace_bytes < need || (need > 0 && !workspace))
        return api_fail(FGD_ERR_INVALID_ARG, "workspace of %lld bytes is below the %lld this call needs",
                        static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    const Span in[] = {{cache->data, cache_bytes}, {q, qb},
                       {tables, table_bytes},      {lengths, B * INT64_C(4)},
                       {starts, starts ? (B + INT64_C(1)) * 4 : 0}};
    for (const Span &s : in) {
        if (fgd_status st = check_apart("the output and the inputs", out, ob, s.p, s.n)) return st;
        if (fgd_status st = check_apart("the workspace and the inputs", workspace, need, s.p, s.n)) return st;
    }
    if (fgd_status st = check_apart("the output and the workspace", out, ob, workspace, need)) return st;
    a.q = {const_cast<void *>(q), q_token_stride, q_head_stride};
    a.out = {out, out_token_stride, out_head_stride};
    a.tables = tables;
    a.table_stride = table_stride;
    a.lengths = lengths;
    a.starts = starts;
    if (!fgd::attend_launch(a, workspace, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "attention launch failed");
    return FGD_OK;
}

fgd_status fgd_extend_pages(const fgd_pages *pages, const int32_t *counts, int64_t tokens, int32_t *starts,
                            int32_t *positions, int64_t *slots, void *stream) {
    fgd::api_clear();
    fgd::PagesView p;
    if (fgd_status st = check_pages(pages, &p)) return st;
    if (tokens < 0 || tokens > INT32_MAX) return api_fail(FGD_ERR_INVALID_ARG, "tokens must be in [0, 2^31)");
    if (fgd_status st = fgd::api_check_array("counts", counts, p.requests, 4)) return st;
    if (fgd_status st = fgd::api_check_array("starts", starts, p.requests + INT64_C(1), 4)) return st;
    if (fgd_status st = fgd::api_check_array("positions", positions, tokens, 4)) return st;
    if (fgd_status st = fgd::api_check_array("slots", slots, tokens, 8)) return st;
    if (fgd_status st = check_state_apart<4>(pages, {{counts, p.requests * INT64_C(4)},
                                                     {starts, (p.requests + INT64_C(1)) * 4},
                                                     {positions, tokens * 4},
                                                     {slots, tokens * 8}}))
        return st;
    if (!fgd::pages_extend_launch(p, counts, tokens, starts, positions, slots, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "block table launch failed");
    return FGD_OK;
}

fgd_status fgd_truncate_pages(const fgd_pages *pages, const int32_t *keep, void *stream) {
    fgd::api_clear();
    fgd::PagesView p;
    if (fgd_status st = check_pages(pages, &p)) return st;
    if (fgd_status st = fgd::api_check_array("keep", keep, p.requests, 4)) return st;
    if (fgd_status st = check_state_apart<1>(pages, {{keep, p.requests * INT64_C(4)}})) return st;
    if (!fgd::pages_truncate_launch(p, keep, static_cast<hipStream_t>(stream)))
        return api_fail(FGD_ERR_HIP, "block table launch failed");
    return FGD_OK;
}

}  // extern "C"
