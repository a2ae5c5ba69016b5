// api_multi.cpp -- the extern "C" entry points of include/dsim_multi_ops.h.
//
// Host side only: argument validation and the launches.  Nothing here may
// throw: no allocation, no C++ library call that can.
#include <cmath>

#include "checks.h"
#include "multi_ops.h"

namespace dsim {

constexpr int kMaxCaches = 1024;
constexpr int64_t kMaxRows = INT32_MAX - 255;   // blocks of up to 256 rows end in 32 bits

static dsim_status check_queries(const dsim_kv_cache *c, const dsim_queries *q)
{
    dsim_status st = check_cache(c, false);
    if (st) return st;
    if (!q) return fail(DSIM_EINVAL, "queries is NULL");
    if ((st = check_dtype(q->dtype, c))) return st;
    if (q->n_q_heads < 1 || q->n_q_heads > kMaxHeads || q->n_q_heads % c->n_heads)
        return fail(DSIM_ERANGE, "n_q_heads must be a multiple of n_heads (%d) and at most %d", c->n_heads, kMaxHeads);
    if (q->n_tok < 0 || q->n_tok > kMaxRows || q->n_tok * q->n_q_heads > kMaxRows)
        return fail(DSIM_ERANGE, "n_tok must be >= 0 and n_tok * n_q_heads at most 2^31 - 256");
    if (!(std::fabs(q->scale) <= 0x1p126f)) return fail(DSIM_EINVAL, "scale must be in [-2^126, 2^126]");
    if (q->cap != 0.0f && !(q->cap >= 0x1p-60f && q->cap <= 0x1p60f)) return fail(DSIM_EINVAL, "cap must be 0 or in [2^-60, 2^60]");
    // (a capped score is taken times their quotient: infinite it would make NaN of a
    // score of 0, and 0 of every other where it has no bits left)
    const float quotient = std::fabs(q->scale) / q->cap;
    if (q->cap != 0.0f && q->scale != 0.0f && !(quotient >= 0x1p-126f && quotient <= 0x1p126f))
        return fail(DSIM_EINVAL, "scale / cap must be 0 or in [2^-126, 2^126]");
    if (q->window < 0) return fail(DSIM_EINVAL, "window must be >= 0");
    if (c->n_seq == 0) return DSIM_OK;
    if (q->n_tok > 0) {
        const int es = elem_size(q->dtype);
        if ((st = check_rows("q", &q->q, q->n_tok, q->n_q_heads, es)) || (st = check_rows("out", &q->out, q->n_tok, q->n_q_heads, es)) ||
            (st = check_apart("out", &q->out, q->n_tok, q->n_q_heads, c->head_dim)) ||
            (st = check_in_place("out", &q->q, &q->out, q->n_tok, q->n_q_heads)))
            return st;
    }
    if (!q->start || !q->len) return fail(DSIM_EINVAL, "start and len must not be NULL");
    const size_t need = rows_workspace(q->n_tok, c->n_seq, q->n_q_heads, c->n_heads, c->head_dim);
    if (!q->workspace || q->ws_bytes < need) return fail(DSIM_ENOSPC, "workspace needs %zu bytes", need);
    if (!aligned16(q->workspace)) return fail(DSIM_EINVAL, "workspace must be 16-byte aligned");
    return DSIM_OK;
}

static dsim_status check_pool(const dsim_page_pool *p)
{
    if (!p) return fail(DSIM_EINVAL, "pool is NULL");
    if (p->page_size < 1 || p->page_size > (1 << 20)) return fail(DSIM_ERANGE, "page_size must be 1..2^20");
    if (p->n_pages < 0 || p->n_pages > INT32_MAX) return fail(DSIM_ERANGE, "n_pages must be 0..2^31 - 1");
    if (p->n_seq < 0 || p->n_seq > (1 << 20)) return fail(DSIM_ERANGE, "n_seq must be 0..2^20");
    if (p->table_width < 0 || p->table_stride < 0 || !product_ok(p->table_stride, 4 * (int64_t)(1 << 20)) ||
        (p->n_seq > 1 && p->table_stride < p->table_width))
        return fail(DSIM_EINVAL, "table_width and table_stride must be >= 0, rows of the table must not overlap");
    if ((int64_t)p->table_width * p->page_size > INT32_MAX)
        return fail(DSIM_ERANGE, "table_width * page_size must be below 2^31");
    if ((p->n_pages > 0 && (!p->refs || !p->free)) || (p->n_seq > 0 && !p->held) ||
        (p->n_seq > 0 && p->table_width > 0 && !p->block_table))
        return fail(DSIM_EINVAL, "refs, free, held and block_table must not be NULL");
    return DSIM_OK;
}

// Caches of one shape, in launches of kLayersAtOnce; their block tables count
// only with `tables` (the first's).
static dsim_status check_layers(const dsim_kv_cache *c, int32_t n, bool tables, Layers *out)
{
    if (!c) return fail(DSIM_EINVAL, "layers is NULL");
    if (n < 1 || n > kMaxCaches) return fail(DSIM_ERANGE, "n_layers must be 1..%d", kMaxCaches);
    for (int32_t i = 0; i < n; ++i) {
        dsim_kv_cache x = c[i];
        if (!tables || i > 0) {
            x.block_table = nullptr;
            x.n_seq = x.table_width = 0;
            x.table_stride = 0;
        }
        const dsim_status st = check_cache(&x, true);
        if (st) return st;
        const dsim_kv_cache &a = c[0];
        const auto differ = [](int64_t n, int64_t s, int64_t t) { return n > 1 && s != t; };
        if (x.dtype != a.dtype || x.n_heads != a.n_heads || x.head_dim != a.head_dim || x.page_size != a.page_size ||
            x.n_pages != a.n_pages || differ(a.n_pages, x.page_stride, a.page_stride) ||
            differ(a.page_size, x.slot_stride, a.slot_stride) || differ(a.n_heads, x.head_stride, a.head_stride))
            return fail(DSIM_EINVAL, "layers must have the same shape, strides and type");
        Layers &l = out[i / kLayersAtOnce];
        const int es = elem_size(a.dtype);
        if (i % kLayersAtOnce == 0) {
            l.n_pages = a.n_pages;
            l.page_stride = a.n_pages > 1 ? a.page_stride * es / 16 : 0;
            l.slot_stride = a.page_size > 1 ? a.slot_stride * es / 16 : 0;
            l.head_stride = a.n_heads > 1 ? a.head_stride * es / 16 : 0;
            l.n = 0;
            l.n_heads = a.n_heads;
            l.page_size = a.page_size;
            l.chunks = a.head_dim * es / 16;
        }
        l.p[2 * l.n] = x.k;
        l.p[2 * l.n + 1] = x.v;
        ++l.n;
    }
    return DSIM_OK;
}

static int launches_of(int32_t n_layers) { return (n_layers + kLayersAtOnce - 1) / kLayersAtOnce; }

}  // namespace dsim

using namespace dsim;

extern "C" {

dsim_status dsim_kv_append_axes(const dsim_kv_cache *cache, int64_t n_tok, int32_t dtype, const dsim_rows *k,
                                const dsim_rows *v, const dsim_rows *q, const dsim_rows *q_out, int32_t n_q_heads,
                                const int32_t *seq, const int32_t *slot, const int32_t *pos, int32_t n_axes,
                                const int32_t *sections, const float *rope, int64_t n_rope, int32_t rot_dim,
                                int32_t interleaved, int32_t *status, void *hip_stream)
{
    AppendArgs a{};
    dsim_status st = check_append(cache, n_tok, dtype, k, v, q, q_out, n_q_heads, seq, slot, rope, n_rope, rot_dim,
                                  interleaved, status, a);
    if (st) return st;
    AxesArgs x{};
    if (rope) {
        if (n_axes < 1 || n_axes > DSIM_MAX_AXES) return fail(DSIM_ERANGE, "n_axes must be 1..%d", DSIM_MAX_AXES);
        if (!sections) return fail(DSIM_EINVAL, "sections is NULL");
        int64_t sum = 0;
        for (int i = 0; i < DSIM_MAX_AXES; ++i) {
            if (i < n_axes && sections[i] < 0) return fail(DSIM_EINVAL, "sections must be >= 0");
            sum += i < n_axes ? sections[i] : 0;
            x.end[i] = (int32_t)(sum > rot_dim ? rot_dim : sum);
        }
        if (sum != rot_dim / 2) return fail(DSIM_EINVAL, "sections must sum to rot_dim / 2");
        if (n_tok > 0 && !pos) return fail(DSIM_EINVAL, "pos is NULL");
        x.pos = pos;
        x.n_axes = n_axes;
    }
    if (n_tok == 0) return DSIM_OK;
    return launch_append_axes(a, x, (hipStream_t)hip_stream);
}

size_t dsim_prompt_attention_workspace(int64_t n_tok, int32_t n_seq, int32_t n_q_heads, int32_t n_heads, int32_t head_dim)
{
    if (n_heads < 1 || n_q_heads < n_heads || n_q_heads > kMaxHeads || n_q_heads % n_heads || head_dim < 16 ||
        head_dim > kMaxHeadDim || head_dim % 16 || n_tok < 0 || n_tok > kMaxRows || n_tok * n_q_heads > kMaxRows ||
        n_seq < 0 || n_seq > (1 << 20))
        return 0;
    return rows_workspace(n_tok, n_seq, n_q_heads, n_heads, head_dim);
}

dsim_status dsim_prompt_attention(const dsim_kv_cache *cache, const dsim_queries *queries, const int32_t *prefix_len,
                                  const int32_t *first_key, void *hip_stream)
{
    const dsim_status st = check_queries(cache, queries);
    if (st || cache->n_seq == 0) return st;
    RowsArgs a{};
    a.c = *cache;
    a.q = *queries;
    a.prefix_len = prefix_len;
    a.first_key = first_key;
    return launch_rows(a, (hipStream_t)hip_stream);
}

dsim_status dsim_tree_attention(const dsim_kv_cache *cache, const dsim_queries *queries, const uint32_t *mask,
                                int64_t mask_stride, int32_t mask_words, const int32_t *depth, void *hip_stream)
{
    const dsim_status st = check_queries(cache, queries);
    if (st) return st;
    if (mask_words < 1 || mask_words > (1 << 26)) return fail(DSIM_ERANGE, "mask_words must be 1..2^26");
    if (mask_stride < 0 || !product_ok(mask_stride, 4 * (queries->n_tok + 1)) || (queries->n_tok > 1 && mask_stride < mask_words))
        return fail(DSIM_EINVAL, "rows of the mask must hold mask_words words");
    if (queries->n_tok > 0 && !mask) return fail(DSIM_EINVAL, "mask is NULL");
    if (queries->n_tok > 0 && !depth && (queries->window > 0 || queries->slopes))
        return fail(DSIM_EINVAL, "a window and slopes need depth");
    if (cache->n_seq == 0) return DSIM_OK;
    RowsArgs a{};
    a.c = *cache;
    a.q = *queries;
    a.mask = mask;
    a.mask_stride = mask_stride;
    a.mask_words = mask_words;
    a.depth = depth;
    a.tree = true;
    return launch_rows(a, (hipStream_t)hip_stream);
}

dsim_status dsim_kv_reserve(const dsim_page_pool *pool, const int32_t *seq_len, const int32_t *new_len, int32_t *status,
                            void *hip_stream)
{
    const dsim_status st = check_pool(pool);
    if (st || pool->n_seq == 0) return st;
    if (!seq_len || !new_len || !status) return fail(DSIM_EINVAL, "seq_len, new_len and status must not be NULL");
    return launch_reserve(*pool, seq_len, new_len, status, (hipStream_t)hip_stream);
}

dsim_status dsim_kv_release(const dsim_page_pool *pool, int64_t n, const int32_t *row, const int32_t *keep_len,
                            int32_t *status, void *hip_stream)
{
    const dsim_status st = check_pool(pool);
    if (st) return st;
    if (n < 0 || n > (1 << 30)) return fail(DSIM_ERANGE, "n must be 0..2^30");
    if (n == 0) return DSIM_OK;
    if (!row || !keep_len) return fail(DSIM_EINVAL, "row and keep_len must not be NULL");
    return launch_release(*pool, n, row, keep_len, status, (hipStream_t)hip_stream);
}

dsim_status dsim_kv_fork(const dsim_kv_cache *layers, int32_t n_layers, const dsim_page_pool *pool, int32_t *seq_len,
                         int64_t n, const int32_t *src, const int32_t *dst, int32_t *status, void *hip_stream)
{
    Layers l[launches_of(kMaxCaches)];
    dsim_status st = check_layers(layers, n_layers, false, l);
    if (st || (st = check_pool(pool))) return st;
    if (layers->n_pages != pool->n_pages || layers->page_size != pool->page_size)
        return fail(DSIM_EINVAL, "pool and layers must have the same pages");
    if (n < 0 || n > (1 << 30)) return fail(DSIM_ERANGE, "n must be 0..2^30");
    if (n == 0) return DSIM_OK;
    if (!seq_len || !src || !dst || !status) return fail(DSIM_EINVAL, "seq_len, src, dst and status must not be NULL");
    return launch_fork(l, launches_of(n_layers), *pool, seq_len, n, src, dst, status, (hipStream_t)hip_stream);
}

dsim_status dsim_kv_copy_pages(const dsim_kv_cache *layers, int32_t n_layers, int64_t n, const int32_t *src,
                               const int32_t *dst, void *hip_stream)
{
    Layers l[launches_of(kMaxCaches)];
    dsim_status st = check_layers(layers, n_layers, false, l);
    if (st) return st;
    if (n < 0 || n > (1 << 30)) return fail(DSIM_ERANGE, "n must be 0..2^30");
    if (n == 0) return DSIM_OK;
    if (!src || !dst) return fail(DSIM_EINVAL, "src and dst must not be NULL");
    for (int i = 0; i < launches_of(n_layers) && !st; ++i) st = launch_copy_pages(l[i], n, src, dst, (hipStream_t)hip_stream);
    return st;
}

dsim_status dsim_kv_compact(const dsim_kv_cache *layers, int32_t n_layers, const int32_t *start, const int32_t *keep,
                            int64_t keep_stride, int32_t keep_width, const int32_t *n_keep, int32_t *status,
                            void *hip_stream)
{
    Layers l[launches_of(kMaxCaches)];
    dsim_status st = check_layers(layers, n_layers, true, l);
    if (st) return st;
    if (keep_width > (1 << 30)) return fail(DSIM_ERANGE, "keep_width must be at most 2^30");
    if (keep_width < 0 || keep_stride < 0 || !product_ok(keep_stride, 4 * (int64_t)(1 << 20)) ||
        (layers->n_seq > 1 && keep_stride < keep_width))
        return fail(DSIM_EINVAL, "rows of keep must hold keep_width entries");
    if (layers->n_seq == 0) return DSIM_OK;
    if (!start || !n_keep || (keep_width > 0 && !keep)) return fail(DSIM_EINVAL, "start, keep and n_keep must not be NULL");
    CompactArgs a{};
    a.table = layers->block_table;
    a.table_stride = layers->table_stride;
    a.n_seq = layers->n_seq;
    a.table_width = layers->table_width;
    a.start = start;
    a.keep = keep;
    a.keep_stride = keep_stride;
    a.keep_width = keep_width;
    a.n_keep = n_keep;
    for (int i = 0; i < launches_of(n_layers) && !st; ++i) {
        a.status = i == 0 ? status : nullptr;   // (told once)
        st = launch_compact(l[i], a, (hipStream_t)hip_stream);
    }
    return st;
}

}  // extern "C"
