// api_ops.cpp -- the extern "C" entry points of include/dsim_ops.h.
//
// Host side only: argument validation and the launches.  Nothing here may
// throw: no allocation, no C++ library call that can.
#include <cmath>

#include "checks.h"

using namespace dsim;

extern "C" {

dsim_status dsim_kv_append(const dsim_kv_cache *cache, int64_t n_tok, int32_t dtype, const dsim_rows *k,
                           const dsim_rows *v, const dsim_rows *q, const dsim_rows *q_out, int32_t n_q_heads,
                           const int32_t *seq, const int32_t *pos, const float *rope, int64_t n_rope, int32_t rot_dim,
                           int32_t interleaved, int32_t *status, void *hip_stream)
{
    AppendArgs a{};
    const dsim_status st = check_append(cache, n_tok, dtype, k, v, q, q_out, n_q_heads, seq, pos, rope, n_rope, rot_dim,
                                        interleaved, status, a);
    if (st || n_tok == 0) return st;
    return launch_append(a, (hipStream_t)hip_stream);
}

size_t dsim_paged_attention_workspace(int32_t n_q_heads, int32_t n_heads, int32_t head_dim)
{
    if (n_heads < 1 || n_q_heads < n_heads || n_q_heads > kMaxHeads || n_q_heads % n_heads || head_dim < 16 ||
        head_dim > kMaxHeadDim || head_dim % 16)
        return 0;
    return attend_workspace(n_q_heads, n_heads, head_dim);
}

dsim_status dsim_paged_attention(const dsim_kv_cache *cache, int32_t dtype, const dsim_rows *q, const dsim_rows *out,
                                 int32_t n_q_heads, const int32_t *seq_len, float scale, int32_t window, float *lse,
                                 int32_t *status, void *workspace, size_t ws_bytes, void *hip_stream)
{
    dsim_status st = check_cache(cache, false);
    if (st) return st;
    if ((st = check_dtype(dtype, cache))) return st;
    if (n_q_heads < 1 || n_q_heads > kMaxHeads || n_q_heads % cache->n_heads)
        return fail(DSIM_ERANGE, "n_q_heads must be a multiple of n_heads (%d) and at most %d", cache->n_heads, kMaxHeads);
    // (times log2 e it has to be finite too)
    if (!(std::fabs(scale) <= 0x1p126f)) return fail(DSIM_EINVAL, "scale must be in [-2^126, 2^126]");
    if (window < 0) return fail(DSIM_EINVAL, "window must be >= 0");
    if (cache->n_seq == 0) return DSIM_OK;
    const int es = elem_size(dtype);
    if ((st = check_rows("q", q, cache->n_seq, n_q_heads, es)) || (st = check_rows("out", out, cache->n_seq, n_q_heads, es)) ||
        (st = check_apart("out", out, cache->n_seq, n_q_heads, cache->head_dim)) ||
        (st = check_in_place("out", q, out, cache->n_seq, n_q_heads)))
        return st;
    if (!seq_len) return fail(DSIM_EINVAL, "seq_len is NULL");
    const size_t need = attend_workspace(n_q_heads, cache->n_heads, cache->head_dim);
    if (!workspace || ws_bytes < need) return fail(DSIM_ENOSPC, "workspace needs %zu bytes", need);
    if (!aligned16(workspace)) return fail(DSIM_EINVAL, "workspace must be 16-byte aligned");
    AttendArgs a{};
    a.c = *cache;
    a.q = *q;
    a.out = *out;
    a.seq_len = seq_len;
    a.lse = lse;
    a.status = status;
    a.ws = workspace;
    a.scale = scale;
    a.dtype = dtype;
    a.n_q_heads = n_q_heads;
    a.window = window;
    return launch_attend(a, (hipStream_t)hip_stream);
}

dsim_status dsim_logit_adjust(const dsim_logits *args, void *hip_stream)
{
    if (!args) return fail(DSIM_EINVAL, "args is NULL");
    const dsim_logits &a = *args;
    if (a.dtype != DSIM_F32 && a.dtype != DSIM_F16 && a.dtype != DSIM_BF16)
        return fail(DSIM_EINVAL, "unknown dtype %d", a.dtype);
    if (a.vocab < 1 || a.vocab > (1 << 30)) return fail(DSIM_ERANGE, "vocab must be 1..2^30");
    if (a.n_rows < 0 || a.n_rows > (1 << 20)) return fail(DSIM_ERANGE, "n_rows must be 0..2^20");
    if (a.n_bias < 0 || a.n_bias > kMaxBias) return fail(DSIM_ERANGE, "n_bias must be 0..%d", kMaxBias);
    if (a.history_width < 0 || a.history_width >= (1 << 30)) return fail(DSIM_ERANGE, "history_width must be in [0, 2^30)");
    if (a.n_rows == 0) return DSIM_OK;
    const int64_t rows = a.n_rows;
    if (!a.logits || !a.out) return fail(DSIM_EINVAL, "logits and out must not be NULL");
    if (rows > 1 && (a.logits_stride < a.vocab || a.out_stride < a.vocab))
        return fail(DSIM_EINVAL, "logits and out rows must not overlap (stride >= vocab)");
    if (!product_ok(a.logits_stride, rows * 4) || !product_ok(a.out_stride, rows * 4))
        return fail(DSIM_ERANGE, "logits are too large");
    const uintptr_t es = (uintptr_t)elem_size(a.dtype);
    if ((uintptr_t)a.logits % es || (uintptr_t)a.out % es) return fail(DSIM_EINVAL, "logits and out must be aligned to their type");
    if (a.logits == a.out && rows > 1 && a.logits_stride != a.out_stride)
        return fail(DSIM_EINVAL, "in place, out_stride must be logits_stride");
    if (a.history ? (!a.history_len || !product_ok(a.history_stride, rows * 4) ||
                     (rows > 1 && a.history_stride < a.history_width))
                  : (a.repetition || a.frequency || a.presence || a.prompt_len || a.history_len))
        return fail(DSIM_EINVAL, "penalties need history and history_len, and rows of the history must not overlap");
    if (a.n_bias > 0 && (!a.bias_id || !a.bias)) return fail(DSIM_EINVAL, "bias_id and bias must not be NULL");
    if (a.mask && (a.mask_stride < 0 || !product_ok(a.mask_stride, rows * 4) ||
                   (rows > 1 && a.mask_stride < (a.vocab + 31) / 32)))
        return fail(DSIM_EINVAL, "mask rows must hold ceil(vocab / 32) words");
    return launch_logits(a, (hipStream_t)hip_stream);
}

}  // extern "C"
