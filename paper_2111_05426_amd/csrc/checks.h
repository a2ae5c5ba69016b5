// checks.h -- what the operators' entry points check of their arguments on the
// host.  Nothing here may throw.
#pragma once

#include "ops.h"

namespace dsim {

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// |a * b| < 2^62, for sizes of memory
inline bool product_ok(int64_t a, int64_t b)
{
    int64_t r;
    return !__builtin_mul_overflow(a, b, &r) && r > -((int64_t)1 << 62) && r < ((int64_t)1 << 62);
}

// the stride of `n` elements of `size` bytes, 16 bytes aligned (that of a
// single one is never used)
inline bool stride_ok(int64_t stride, int64_t n, int size)
{
    return n <= 1 || (stride >= 0 && product_ok(stride, size) && product_ok(stride * size, n) && stride * size % 16 == 0);
}

// Whether rows of d elements, n[i] of them stride[i] apart in dimension i of
// m, lie apart: each stride spans what the smaller ones reach.
inline bool apart(int64_t d, int m, const int64_t *n, const int64_t *stride)
{
    int64_t reach = d, last = -1;
    for (int k = 0; k < m; ++k) {
        int at = -1;   // the next larger stride
        for (int i = 0; i < m; ++i)
            if (n[i] > 1 && stride[i] > last && (at < 0 || stride[i] < stride[at])) at = i;
        if (at < 0) break;
        int same = 0;
        for (int i = 0; i < m; ++i) same += n[i] > 1 && stride[i] == stride[at];
        if (same > 1 || stride[at] < reach) return false;
        reach += stride[at] * (n[at] - 1);
        last = stride[at];
    }
    return true;
}

// written: the rows must lie apart
inline dsim_status check_cache(const dsim_kv_cache *c, bool written)
{
    if (!c) return fail(DSIM_EINVAL, "cache is NULL");
    if (c->dtype < DSIM_F32 || c->dtype > DSIM_E4M3) return fail(DSIM_EINVAL, "unknown cache dtype %d", c->dtype);
    if (c->n_heads < 1 || c->n_heads > kMaxHeads) return fail(DSIM_ERANGE, "n_heads must be 1..%d", kMaxHeads);
    if (c->head_dim < 16 || c->head_dim > kMaxHeadDim || c->head_dim % 16)
        return fail(DSIM_ERANGE, "head_dim must be a multiple of 16 in 16..%d, not %d", kMaxHeadDim, c->head_dim);
    if (c->page_size < 1 || c->page_size > (1 << 20)) return fail(DSIM_ERANGE, "page_size must be 1..2^20");
    if (c->n_pages < 0 || c->n_pages > INT32_MAX) return fail(DSIM_ERANGE, "n_pages must be 0..2^31 - 1");
    if (c->n_seq < 0 || c->n_seq > (1 << 20)) return fail(DSIM_ERANGE, "n_seq must be 0..2^20");
    if (c->table_width < 0 || c->table_stride < 0 || !product_ok(c->table_stride, 4 * (int64_t)(1 << 20)) ||
        (c->n_seq > 1 && c->table_stride < c->table_width))
        return fail(DSIM_EINVAL, "table_width and table_stride must be >= 0, rows of the table must not overlap");
    if ((int64_t)c->table_width * c->page_size > INT32_MAX)
        return fail(DSIM_ERANGE, "table_width * page_size must be below 2^31");
    const int es = elem_size(c->dtype);
    if (!stride_ok(c->page_stride, c->n_pages, es) || !stride_ok(c->slot_stride, c->page_size, es) ||
        !stride_ok(c->head_stride, c->n_heads, es))
        return fail(DSIM_EINVAL, "cache strides must be >= 0 and multiples of 16 bytes");
    const int64_t n[3] = {c->n_pages, c->page_size, c->n_heads}, strides[3] = {c->page_stride, c->slot_stride, c->head_stride};
    if (written && !apart(c->head_dim, 3, n, strides)) return fail(DSIM_EINVAL, "rows of the cache overlap");
    if ((c->n_pages > 0 && (!c->k || !c->v)) || !aligned16(c->k) || !aligned16(c->v))
        return fail(DSIM_EINVAL, "k and v must not be NULL and must be 16-byte aligned");
    if ((c->k_scale || c->v_scale) && c->dtype != DSIM_E4M3)
        return fail(DSIM_EINVAL, "scales need an e4m3 cache");
    if (c->n_seq > 0 && c->table_width > 0 && !c->block_table) return fail(DSIM_EINVAL, "block_table is NULL");
    return DSIM_OK;
}

inline dsim_status check_rows(const char *name, const dsim_rows *r, int64_t n, int32_t heads, int size)
{
    if (!r || !r->data) return fail(DSIM_EINVAL, "%s must not be NULL", name);
    if (!aligned16(r->data) || !stride_ok(r->row_stride, n, size) || !stride_ok(r->head_stride, heads, size))
        return fail(DSIM_EINVAL, "%s: pointer and strides must be multiples of 16 bytes, strides >= 0", name);
    return DSIM_OK;
}

inline dsim_status check_apart(const char *name, const dsim_rows *r, int64_t n, int32_t heads, int32_t d)
{
    const int64_t size[2] = {n, heads}, stride[2] = {r->row_stride, r->head_stride};
    return apart(d, 2, size, stride) ? DSIM_OK : fail(DSIM_EINVAL, "rows of %s overlap", name);
}

// `out` that begins where `in` does must be the same rows
inline dsim_status check_in_place(const char *out_name, const dsim_rows *in, const dsim_rows *out, int64_t n, int32_t heads)
{
    if (in->data == out->data && ((n > 1 && in->row_stride != out->row_stride) ||
                                  (heads > 1 && in->head_stride != out->head_stride)))
        return fail(DSIM_EINVAL, "in place, %s must have the strides of q", out_name);
    return DSIM_OK;
}

inline dsim_status check_dtype(int32_t dtype, const dsim_kv_cache *c)
{
    if (dtype != DSIM_F32 && dtype != DSIM_F16 && dtype != DSIM_BF16) return fail(DSIM_EINVAL, "unknown dtype %d", dtype);
    if (c->dtype == DSIM_E4M3 ? dtype == DSIM_F32 : dtype != c->dtype)
        return fail(DSIM_EINVAL, "dtype must be the cache's, or fp16 / bf16 with an e4m3 cache");
    return DSIM_OK;
}

// The arguments of an append; pos: its tokens' places in the cache.
inline dsim_status check_append(const dsim_kv_cache *cache, int64_t n_tok, int32_t dtype, const dsim_rows *k,
                                const dsim_rows *v, const dsim_rows *q, const dsim_rows *q_out, int32_t n_q_heads,
                                const int32_t *seq, const int32_t *pos, const float *rope, int64_t n_rope,
                                int32_t rot_dim, int32_t interleaved, int32_t *status, AppendArgs &a)
{
    dsim_status st = check_cache(cache, true);
    if (st) return st;
    if ((st = check_dtype(dtype, cache))) return st;
    if (n_tok < 0 || n_tok > INT32_MAX) return fail(DSIM_ERANGE, "n_tok must be 0..2^31 - 1");
    if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 8)
        return fail(DSIM_EINVAL, "rot_dim must be a multiple of 8 in 0..head_dim");
    if (interleaved != 0 && interleaved != 1) return fail(DSIM_EINVAL, "interleaved must be 0 or 1");
    if ((rot_dim > 0) != (rope != nullptr)) return fail(DSIM_EINVAL, "rope and rot_dim > 0 come together");
    if (rope && (n_rope < 0 || !product_ok(n_rope, 4 * (int64_t)rot_dim) || !aligned16(rope)))
        return fail(DSIM_EINVAL, "n_rope must be >= 0 and rope 16-byte aligned");
    if (!q != !q_out) return fail(DSIM_EINVAL, "q and q_out come together");
    if (q && (n_q_heads < 1 || n_q_heads > kMaxHeads)) return fail(DSIM_ERANGE, "n_q_heads must be 1..%d", kMaxHeads);
    if (n_tok == 0) return DSIM_OK;
    const int es = elem_size(dtype);
    if ((st = check_rows("k", k, n_tok, cache->n_heads, es)) || (st = check_rows("v", v, n_tok, cache->n_heads, es)))
        return st;
    if (q && ((st = check_rows("q", q, n_tok, n_q_heads, es)) || (st = check_rows("q_out", q_out, n_tok, n_q_heads, es)) ||
              (st = check_apart("q_out", q_out, n_tok, n_q_heads, cache->head_dim)) ||
              (st = check_in_place("q_out", q, q_out, n_tok, n_q_heads))))
        return st;
    if (!seq || !pos) return fail(DSIM_EINVAL, "seq and pos must not be NULL");
    a.c = *cache;
    a.k = *k;
    a.v = *v;
    if (q) {
        a.q = *q;
        a.q_out = *q_out;
        a.n_q_heads = n_q_heads;
    }
    a.seq = seq;
    a.pos = pos;
    a.rope = rope;
    a.status = status;
    a.n_tok = n_tok;
    a.n_rope = n_rope;
    a.dtype = dtype;
    a.rot_dim = rot_dim;
    a.interleaved = interleaved;
    return DSIM_OK;
}

}  // namespace dsim
