// C ABI of the reader's calls: argument validation and dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "kv.h"
#include "status.h"
#include "tq_internal.h"

using namespace tq;

namespace {

constexpr int64_t kMost = INT32_MAX;
// HIP takes fewer than 2^32 threads along a grid's side: workgroups of 256
constexpr int64_t kMostGroups = (int64_t)1 << 24;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// A tensor whose 8-element pieces can be loaded 16 bytes at a time.
bool wide_rows(const tq_rows *t) {
    return aligned16(t->data_dev) && t->token_stride % 8 == 0 && t->head_stride % 8 == 0;
}

tq_status check_dim(int32_t d) {
    if (d != 64 && d != 128 && d != 256)
        return fail(TQ_EUNSUPPORTED, "head_dim must be 64, 128 or 256, got " + std::to_string(d));
    return TQ_OK;
}

tq_status check_float(int32_t dtype) {
    if (dtype != TQ_F16 && dtype != TQ_BF16) return fail(TQ_EINVAL, "dtype must be TQ_F16 or TQ_BF16");
    return TQ_OK;
}

tq_status check_rows(const tq_rows *t, int64_t n, const char *name) {
    if (!t) return fail(TQ_EINVAL, std::string(name) + " is NULL");
    if (n > 0 && !t->data_dev) return fail(TQ_EINVAL, std::string(name) + ": NULL device pointer");
    if (t->token_stride < 0 || t->head_stride < 0) return fail(TQ_EINVAL, std::string(name) + ": negative stride");
    if (reinterpret_cast<uintptr_t>(t->data_dev) & 1) return fail(TQ_EINVAL, std::string(name) + " is not aligned to its elements");
    return TQ_OK;
}

tq_status check_cache(const tq_kv_cache *c) {
    if (!c) return fail(TQ_EINVAL, "NULL cache");
    if (!c->k_dev || !c->v_dev || !c->k_scale_dev || !c->v_scale_dev) return fail(TQ_EINVAL, "cache: NULL device pointer");
    if (!aligned16(c->k_dev) || !aligned16(c->v_dev)) return fail(TQ_EINVAL, "cache: codes must be 16-byte aligned");
    if (c->layers < 1 || c->kv_heads < 1 || c->pages < 1 || c->pages > kMost) return fail(TQ_EINVAL, "cache: sizes must be positive");
    if (c->kv_heads > 4096) return fail(TQ_EUNSUPPORTED, "cache: more than 4096 key heads");
    if (c->type != TQ_KV_INT8 && c->type != TQ_KV_FP8) return fail(TQ_EINVAL, "cache: type must be TQ_KV_INT8 or TQ_KV_FP8");
    return check_dim(c->head_dim);
}

KvLayer layer_of(const tq_kv_cache *c, int32_t layer) {
    const int64_t tiles = (int64_t)layer * c->pages * c->kv_heads;
    KvLayer l;
    l.k = static_cast<char *>(c->k_dev) + tiles * kPage * c->head_dim;
    l.v = static_cast<char *>(c->v_dev) + tiles * kPage * c->head_dim;
    l.ks = c->k_scale_dev + tiles * 4;
    l.vs = c->v_scale_dev + tiles * 4;
    l.status = c->status_dev;
    l.pages = (int)c->pages;
    l.heads = c->kv_heads;
    return l;
}

// What append and attend share: the layer, the rows and the packed tokens.
tq_status check_call(const tq_kv_cache *c, int32_t layer, int32_t dtype, int64_t n, const int32_t *tables,
                     int32_t width, const int32_t *lens, const int32_t *starts, int32_t rows) {
    tq_status st = check_cache(c);
    if (st != TQ_OK) return st;
    if (layer < 0 || layer >= c->layers) return fail(TQ_EINVAL, "layer out of range");
    if ((st = check_float(dtype)) != TQ_OK) return st;
    if (n < 0 || n > kMost || rows < 0 || width < 0) return fail(TQ_EINVAL, "negative or oversized n, rows or width");
    if ((int64_t)rows * width > kMost) return fail(TQ_EUNSUPPORTED, "tables of 2^31 or more entries");
    if ((int64_t)width * kPage > kMost) return fail(TQ_EUNSUPPORTED, "rows of 2^31 or more tokens");
    if (n == 0 || rows == 0) return n > 0 ? fail(TQ_EINVAL, "tokens but no rows") : TQ_OK;
    if (!lens || (!tables && width > 0)) return fail(TQ_EINVAL, "NULL tables or lens");
    if (!starts && n != rows) return fail(TQ_EINVAL, "without starts there is one token per row");
    return TQ_OK;
}

tq_status heads_of(int32_t heads, int32_t kv_heads) {
    if (heads < 1 || kv_heads < 1 || heads % kv_heads)
        return fail(TQ_EINVAL, "heads must be a positive multiple of kv_heads");
    if (heads > 4096) return fail(TQ_EUNSUPPORTED, "more than 4096 heads");
    return TQ_OK;
}

tq_status check_pool(const tq_kv_rows *r) {
    if (!r) return fail(TQ_EINVAL, "NULL rows");
    if (r->pages < 1 || r->pages > kMost / 4 || r->rows < 0 || r->width < 0) return fail(TQ_EINVAL, "rows: sizes out of range");
    if ((int64_t)r->rows * r->width > kMost || (int64_t)r->width * kPage > kMost)
        return fail(TQ_EUNSUPPORTED, "rows: tables of 2^31 or more entries or tokens");
    return TQ_OK;
}

tq_status pool_args(const tq_kv_rows *r, const tq_kv_cache *c, int64_t n, void *ws, size_t bytes, PagesArgs *a) {
    tq_status st = check_pool(r);
    if (st != TQ_OK) return st;
    if ((st = check_cache(c)) != TQ_OK) return st;
    if (c->pages != r->pages) return fail(TQ_EINVAL, "the cache and the rows disagree on the number of pages");
    if (!r->refs_dev || (r->rows > 0 && (!r->lens_dev || (r->width > 0 && !r->tables_dev))))
        return fail(TQ_EINVAL, "rows: NULL device pointer");
    if (n < 0 || n > kMost || (n > 0 && n * r->width > kMost)) return fail(TQ_EINVAL, "n out of range");
    // the copies' grid: pieces of 16 KiB of two stores along y
    if (2 * (int64_t)c->layers * (((int64_t)c->kv_heads * kPage * c->head_dim + 16383) / 16384) > 65535)
        return fail(TQ_EUNSUPPORTED, "a page of all layers is over 512 MiB");
    if (!ws || bytes < kv_rows_bytes(r->pages, r->rows, r->width, n)) return fail(TQ_EINVAL, "workspace too small");
    if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(TQ_EINVAL, "workspace not aligned");
    a->tables = r->tables_dev;
    a->lens = r->lens_dev;
    a->refs = r->refs_dev;
    a->pages = (int)r->pages;
    a->rows = r->rows;
    a->width = r->width;
    a->cache = layer_of(c, 0);
    a->layers = c->layers;
    a->D = c->head_dim;
    a->ws = ws;
    return TQ_OK;
}

// Entry points do not let host allocation failures (message strings) out.
template <class F>
tq_status guarded(F f) {
    try {
        return f();
    } catch (...) {
        return TQ_ENOMEM;
    }
}

}  // namespace

tq_status tq_kv_append(const tq_kv_cache *cache, int32_t layer, const tq_rows *k, const tq_rows *v, int32_t dtype,
                       int64_t n, const int32_t *tables, int32_t width, const int32_t *lens, const int32_t *starts,
                       int32_t rows, void *stream) {
    return guarded([&]() -> tq_status {
        tq_status st = check_call(cache, layer, dtype, n, tables, width, lens, starts, rows);
        if (st != TQ_OK) return st;
        if ((st = check_rows(k, n, "k")) != TQ_OK || (st = check_rows(v, n, "v")) != TQ_OK) return st;
        if (n == 0 || width == 0) return TQ_OK;
        if ((starts ? n / kBlock + 2 * (int64_t)rows : rows) >= kMostGroups)
            return fail(TQ_EUNSUPPORTED, "too many tokens or rows for one append");
        if ((st = device_ready()) != TQ_OK) return st;
        AppendArgs a;
        a.layer = layer_of(cache, layer);
        a.set = {tables, lens, starts, rows, width, (int)n};
        a.k = k->data_dev;
        a.v = v->data_dev;
        a.kt = k->token_stride, a.kh = k->head_stride, a.vt = v->token_stride, a.vh = v->head_stride;
        a.bf16 = dtype == TQ_BF16;
        a.wide = wide_rows(k) && wide_rows(v);
        const hipError_t e = kv_append(a, cache->head_dim, cache->type, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? TQ_OK : hip_fail(e, "append");
    });
}

tq_status tq_kv_attend_workspace(const tq_kv_cache *cache, int64_t n, int32_t heads, int32_t width, int32_t rows,
                                 int32_t longest, size_t *bytes_out) {
    return guarded([&]() -> tq_status {
        if (!bytes_out) return fail(TQ_EINVAL, "bytes_out is NULL");
        *bytes_out = 0;
        tq_status st = check_cache(cache);
        if (st != TQ_OK) return st;
        if ((st = heads_of(heads, cache->kv_heads)) != TQ_OK) return st;
        if (n < 0 || n > kMost || rows < 0 || width < 0 || longest < 0) return fail(TQ_EINVAL, "negative size");
        if (n == 0 || rows == 0) return TQ_OK;
        // rows of single tokens and rows of several (starts) may be cut differently
        const int group = heads / cache->kv_heads;
        for (const bool starts : {false, true}) {
            const AttendPlan p = attend_plan(n, rows, group, cache->kv_heads, width, longest, cache->head_dim, starts);
            *bytes_out = std::max(*bytes_out, attend_bytes(p, cache->head_dim));
        }
        return TQ_OK;
    });
}

tq_status tq_kv_attend(const tq_kv_cache *cache, int32_t layer, const tq_rows *q, int32_t dtype, int64_t n,
                       int32_t heads, const int32_t *tables, int32_t width, const int32_t *lens,
                       const int32_t *starts, int32_t rows, int32_t longest, float scale, void *out, float *lse,
                       void *ws, size_t ws_bytes, void *stream) {
    return guarded([&]() -> tq_status {
        tq_status st = check_call(cache, layer, dtype, n, tables, width, lens, starts, rows);
        if (st != TQ_OK) return st;
        if ((st = heads_of(heads, cache->kv_heads)) != TQ_OK) return st;
        if ((st = check_rows(q, n, "q")) != TQ_OK) return st;
        if (longest < 0) return fail(TQ_EINVAL, "longest < 0");
        if (!std::isfinite(scale)) return fail(TQ_EINVAL, "scale is not finite");
        if (n == 0) return TQ_OK;
        if (!out || (reinterpret_cast<uintptr_t>(out) & 7)) return fail(TQ_EINVAL, "out is NULL or not 8-byte aligned");
        const int group = heads / cache->kv_heads;
        const AttendPlan p = attend_plan(n, rows, group, cache->kv_heads, width, longest, cache->head_dim, starts != nullptr);
        const size_t need = attend_bytes(p, cache->head_dim);
        if (need && (!ws || ws_bytes < need || !aligned16(ws)))
            return fail(TQ_EINVAL, "workspace too small or not aligned");
        if (p.line >= (int64_t)1 << 30 || p.units >= kMostGroups / 2 || n * heads >= kMostGroups || n * group > kMost)
            return fail(TQ_EUNSUPPORTED, "too many queries or tokens for one call");
        if ((st = device_ready()) != TQ_OK) return st;
        AttendArgs a;
        a.layer = layer_of(cache, layer);
        a.set = {tables, lens, starts, rows, width, (int)n};
        a.q = q->data_dev;
        a.qt = q->token_stride, a.qh = q->head_stride;
        a.out = out;
        a.lse = lse;
        a.info = static_cast<int *>(ws);
        a.parts = reinterpret_cast<float *>(static_cast<char *>(ws) + attend_info_bytes(p));
        a.scale2 = scale * 1.44269504089f;
        a.heads = heads;
        a.group = group;
        a.bf16 = dtype == TQ_BF16;
        a.wide = wide_rows(q);
        a.shares = p.shares;
        a.limit = longest > 0 && longest < width * kPage ? longest : width * kPage;
        const hipError_t e = kv_attend(a, p, cache->head_dim, cache->type, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? TQ_OK : hip_fail(e, "attention over the cache");
    });
}

tq_status tq_kv_rows_workspace(const tq_kv_rows *rows, int64_t n, size_t *bytes_out) {
    return guarded([&]() -> tq_status {
        if (!bytes_out) return fail(TQ_EINVAL, "bytes_out is NULL");
        *bytes_out = 0;
        const tq_status st = check_pool(rows);
        if (st != TQ_OK) return st;
        if (n < 0 || n > kMost) return fail(TQ_EINVAL, "n out of range");
        *bytes_out = kv_rows_bytes(rows->pages, rows->rows, rows->width, n);
        return TQ_OK;
    });
}

tq_status tq_kv_resize(const tq_kv_rows *rows, const int32_t *goals, const tq_kv_cache *cache, void *ws, size_t bytes,
                       void *stream) {
    return guarded([&]() -> tq_status {
        PagesArgs a;
        tq_status st = pool_args(rows, cache, 0, ws, bytes, &a);
        if (st != TQ_OK) return st;
        if (rows->rows == 0) return TQ_OK;
        if (!goals) return fail(TQ_EINVAL, "goals is NULL");
        if ((st = device_ready()) != TQ_OK) return st;
        const hipError_t e = kv_resize(a, goals, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? TQ_OK : hip_fail(e, "resize");
    });
}

tq_status tq_kv_fork(const tq_kv_rows *rows, const int32_t *src, const int32_t *dst, int64_t n,
                     const tq_kv_cache *cache, void *ws, size_t bytes, void *stream) {
    return guarded([&]() -> tq_status {
        PagesArgs a;
        tq_status st = pool_args(rows, cache, n, ws, bytes, &a);
        if (st != TQ_OK) return st;
        if (n == 0) return TQ_OK;
        if (!src || !dst) return fail(TQ_EINVAL, "src or dst is NULL");
        if ((st = device_ready()) != TQ_OK) return st;
        const hipError_t e = kv_fork(a, src, dst, (int)n, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? TQ_OK : hip_fail(e, "fork");
    });
}

tq_status tq_kv_compact(const tq_kv_rows *rows, const tq_kv_cache *cache, int32_t *live, void *ws, size_t bytes,
                        void *stream) {
    return guarded([&]() -> tq_status {
        PagesArgs a;
        tq_status st = pool_args(rows, cache, 0, ws, bytes, &a);
        if (st != TQ_OK) return st;
        if (!live) return fail(TQ_EINVAL, "live_dev is NULL");
        if ((st = device_ready()) != TQ_OK) return st;
        const hipError_t e = kv_compact(a, live, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? TQ_OK : hip_fail(e, "compact");
    });
}

tq_status tq_attention(const tq_rows *q, const tq_rows *k, const tq_rows *v, int32_t dtype, int64_t n, int64_t n_keys,
                       int32_t heads, int32_t kv_heads, int32_t head_dim, const int32_t *starts,
                       const int32_t *key_starts, int32_t rows, int32_t longest, int32_t causal, float scale,
                       void *out, float *lse, void *stream) {
    return guarded([&]() -> tq_status {
        tq_status st = check_dim(head_dim);
        if (st != TQ_OK) return st;
        if ((st = check_float(dtype)) != TQ_OK || (st = heads_of(heads, kv_heads)) != TQ_OK) return st;
        if (n < 0 || n > kMost || n_keys < 0 || n_keys > kMost || rows < 0 || longest < 0)
            return fail(TQ_EINVAL, "negative or oversized n, n_keys, rows or longest");
        if ((st = check_rows(q, n, "q")) != TQ_OK || (st = check_rows(k, n_keys, "k")) != TQ_OK ||
            (st = check_rows(v, n_keys, "v")) != TQ_OK)
            return st;
        if (!std::isfinite(scale)) return fail(TQ_EINVAL, "scale is not finite");
        if (!key_starts && n_keys != n) return fail(TQ_EINVAL, "without key_starts there are as many keys as queries");
        if (n == 0) return TQ_OK;
        if (rows == 0 || !starts) return fail(TQ_EINVAL, "queries but no rows, or starts is NULL");
        if (!out || (reinterpret_cast<uintptr_t>(out) & 7)) return fail(TQ_EINVAL, "out is NULL or not 8-byte aligned");
        const int group = heads / kv_heads;
        if ((n * group / 32 + 4 * (int64_t)rows) * kv_heads >= kMostGroups || n * group > kMost)
            return fail(TQ_EUNSUPPORTED, "too many queries for one call");
        if ((st = device_ready()) != TQ_OK) return st;
        PromptArgs a;
        a.q = q->data_dev, a.k = k->data_dev, a.v = v->data_dev;
        a.qt = q->token_stride, a.qh = q->head_stride;
        a.kt = k->token_stride, a.kh = k->head_stride;
        a.vt = v->token_stride, a.vh = v->head_stride;
        a.starts = starts;
        a.key_starts = key_starts;
        a.rows = rows;
        a.total = (int)n;
        a.keys = (int)n_keys;
        a.heads = heads;
        a.group = group;
        a.kv_heads = kv_heads;
        a.levels = prompt_levels(group, longest);
        a.causal = causal;
        // a step's 64 rows lie within 32-bit distances
        a.wide = wide_rows(q) && wide_rows(k) && wide_rows(v) && k->token_stride < 1 << 24 && v->token_stride < 1 << 24;
        a.scale2 = scale * 1.44269504089f;
        a.out = out;
        a.lse = lse;
        const hipError_t e = prompt_attention(a, head_dim, dtype == TQ_BF16, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? TQ_OK : hip_fail(e, "prompt attention");
    });
}
