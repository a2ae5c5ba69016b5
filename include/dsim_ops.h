/*
 * dsim_ops.h -- C ABI of the operators of a single-token step.
 *
 * A transformer that answers one token at a time runs, beside its matrix
 * products, three operators bound by memory: the new token's key and value
 * are rotated by its position and written into a paged cache, its queries
 * attend to that cache, and the logits the step ends with are adjusted
 * before a token is chosen.  The simulator prices such ops by the device
 * model's launch overhead and memory bandwidth (dsim_device_model.launch_s,
 * mem_bytes_per_s); the calibration measures both on these kernels.
 *
 * The conventions of dsim.h hold for every call: dsim_status returned and
 * dsim_last_error() set, device buffers owned by the caller, everything
 * enqueued on `hip_stream`, arguments validated on the host before any
 * launch, deterministic results.  Calls allocate nothing, keep nothing
 * between calls, clear nothing with a memset and may be captured into a HIP
 * graph; the stream's device must be the current one.  Errors that only
 * device data shows (a page outside the cache, a position outside the
 * table) never abort: they set bits of the token's or sequence's status
 * word and no memory outside the buffers is touched.
 */
#ifndef DSIM_OPS_H
#define DSIM_OPS_H

#include "dsim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define DSIM_F32 0
#define DSIM_F16 1
#define DSIM_BF16 2
#define DSIM_E4M3 3   /* OCP 8-bit float: 4 exponent bits, 3 mantissa bits, largest value 448, no infinity; caches only */

/* status bits of a token or sequence */
#define DSIM_ST_BAD_PAGE 128       /* a page number outside [0, n_pages)                        */
#define DSIM_ST_BAD_POSITION 256   /* a position or length outside the block table or rope      */
#define DSIM_ST_BAD_SEQUENCE 512   /* a sequence number >= n_seq                                */

/*
 * A paged key-value cache.  Key and value of slot i of page p for head h are
 * rows of head_dim elements at  p * page_stride + i * slot_stride +
 * h * head_stride  (strides in elements; the same for k and v).  Position t
 * of sequence s lies in page block_table[s * table_stride + t / page_size],
 * slot t % page_size.  Entries of the table behind a sequence's last page
 * are never read.  Rows that are written must lie apart, nested in some
 * order of the three strides; the stride of a dimension of one is ignored.
 *   dtype:     DSIM_F32, DSIM_F16, DSIM_BF16 or DSIM_E4M3
 *   k_scale, v_scale: device arrays of n_heads or NULL (1): an e4m3 element
 *              of head h stands for scale[h] times its value.  Only with
 *              DSIM_E4M3; values must be > 0.
 *   head_dim:  a multiple of 16, 16..256
 *   page_size: 1..2^20;  n_pages: 0..2^31 - 1;  n_heads: 1..1024
 *   k, v and every stride in bytes: multiples of 16
 */
typedef struct {
    void *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *block_table;
    int64_t n_pages, page_stride, slot_stride, head_stride, table_stride;
    int32_t dtype, n_heads, head_dim, page_size, n_seq, table_width;
} dsim_kv_cache;

/* Rows of head_dim elements: row r, head h at r * row_stride + h *
 * head_stride (elements).  The pointer and both strides in bytes must be
 * multiples of 16; rows that are written must lie apart. */
typedef struct {
    void *data;
    int64_t row_stride, head_stride;
} dsim_rows;

/*
 * dsim_kv_append -- write n_tok new keys and values into the cache, rotated
 * by position on the way, and rotate their queries.
 * Token t belongs to sequence seq[t] at position pos[t]; its key and value
 * go to that position's page and slot.  Rotation of a row x by row p =
 * pos[t] of rope ([n_rope][rot_dim], rot_dim / 2 cosines, then as many
 * sines), with R = rot_dim, for i < R / 2:
 *   interleaved = 0: a = i,     b = i + R / 2
 *   interleaved = 1: a = 2 * i, b = 2 * i + 1
 *   y_a = x_a cos_i - x_b sin_i,   y_b = x_b cos_i + x_a sin_i
 * in fp32 (each product and sum rounded), elements from R on unchanged.
 * Keys and queries are rotated, values are not.  What is stored is y
 * rounded once to the type; in an e4m3 cache y / scale[h], values beyond
 * +-448 stored as +-448 (infinities too) and NaN as NaN.
 *   dtype:  type of k, v, q and q_out: that of the cache, or DSIM_F16 /
 *           DSIM_BF16 with an e4m3 cache
 *   q, q_out: both NULL, or rows of n_q_heads heads; q_out may be q (with
 *           its strides)
 *   rope:   NULL with rot_dim = 0 (nothing is rotated); rot_dim a multiple
 *           of 8, at most head_dim
 *   status: device array [n_tok] or NULL: 0 or DSIM_ST_* bits.  A flagged
 *           token writes nothing to the cache and NaN to its row of q_out.
 * A token with seq[t] < 0 is padding: nothing of it is written, and its
 * status is 0.  Two tokens of one call must not have the same place: each
 * element there is then one of theirs, which one is open.  No input or
 * output may overlap another, but q_out may be q.  n_tok < 2^31.
 */
DSIM_API dsim_status dsim_kv_append(const dsim_kv_cache *cache, int64_t n_tok, int32_t dtype, const dsim_rows *k,
                                    const dsim_rows *v, const dsim_rows *q, const dsim_rows *q_out,
                                    int32_t n_q_heads, const int32_t *seq, const int32_t *pos, const float *rope,
                                    int64_t n_rope, int32_t rot_dim, int32_t interleaved, int32_t *status,
                                    void *hip_stream);

/*
 * dsim_paged_attention -- attention of one query token per sequence over
 * its cached keys and values.  Query head h reads cache head h / (n_q_heads
 * / n_heads); n_heads divides n_q_heads (at most 1024).  With L =
 * seq_len[s] and the keys j in [max(0, L - window), L) (window = 0: [0, L)):
 *   s_j = scale * q . k_j,   o = sum_j exp(s_j) v_j / sum_j exp(s_j),
 *   lse = log sum_j exp(s_j)
 * computed with a running maximum, sums and exponentials in fp32; the
 * result is rounded once to out's type.
 *   q, out: one row per sequence of n_q_heads heads, both of `dtype`: the
 *           cache's type, or DSIM_F16 / DSIM_BF16 with an e4m3 cache;
 *           out may be q (with its strides); it must not overlap otherwise
 *   scale:  in [-2^126, 2^126]
 *   seq_len: device array [n_seq].  0: out is 0 and lse -inf.  Negative: the
 *           sequence's rows of out, lse and status are left as they were.
 *   lse:    device array [n_seq][n_q_heads] fp32, or NULL
 *   status: device array [n_seq] or NULL: 0 or DSIM_ST_* bits.  A sequence
 *           longer than table_width * page_size, or with a page of the keys it attends to
 *           outside the cache, gets NaN in out and lse.
 *   workspace: device buffer of at least dsim_paged_attention_workspace(...)
 *           bytes, 16-byte aligned, in use until hip_stream has passed the
 *           call; it needs no clearing and keeps nothing for later calls
 *           (0 is returned there for heads or a head_dim that the call
 *           refuses).
 * The work of all sequences is laid end to end and cut into equal parts, so
 * that one long context among short ones is spread over the GPU; contexts
 * that a cut goes through are joined by a second launch.  Where the block
 * table or the window keeps every context short (at most 1,024 keys, fewer
 * for long heads), each is one workgroup's and there is no second launch.
 * n_seq <= 2^20.
 */
DSIM_API size_t dsim_paged_attention_workspace(int32_t n_q_heads, int32_t n_heads, int32_t head_dim);
DSIM_API dsim_status dsim_paged_attention(const dsim_kv_cache *cache, int32_t dtype, const dsim_rows *q,
                                          const dsim_rows *out, int32_t n_q_heads, const int32_t *seq_len,
                                          float scale, int32_t window, float *lse, int32_t *status, void *workspace,
                                          size_t ws_bytes, void *hip_stream);

/*
 * dsim_logit_adjust -- penalties for repeated tokens, biases and grammar
 * masks on logits [n_rows][vocab].  For row b and token t, with x the logit
 * in fp32, c the count of t among the row's generated tokens and `seen`
 * whether t is among its prompt or generated ones:
 *   seen:  x = x > 0 ? x / repetition[b] : x * repetition[b]
 *   x = x - (frequency[b] * c + (c > 0 ? presence[b] : 0))
 *   x = x + bias of t, if the row has one
 *   x = -inf, if the row's mask bit of t is 0
 * (each step in fp32, without fused multiply-add), rounded once to the type.
 * Every part is optional:
 *   history:  device array [n_rows][history_stride] of token numbers:
 *             history_len[b] of them, the first prompt_len[b] the prompt;
 *             numbers outside [0, vocab) are ignored.  history_len is
 *             clamped to 0..history_width and prompt_len to
 *             0..history_len; prompt_len NULL: no prompt.
 *   repetition, frequency, presence: device arrays [n_rows], each NULL
 *             (1, 0, 0) or given; they need history.
 *   bias_id, bias: device arrays [n_rows][n_bias], n_bias <= 4096; entries
 *             whose id lies outside [0, vocab) are ignored, and of several
 *             entries of one id the last counts.
 *   mask:     device array [n_rows][mask_stride] of 32-bit words,
 *             mask_stride >= ceil(vocab / 32): bit t % 32 of word t / 32
 *             is 1 where t is allowed.
 *   dtype:    DSIM_F32, DSIM_F16 or DSIM_BF16, of logits and out; rows are
 *             logits_stride and out_stride elements apart (>= vocab, or any
 *             with n_rows = 1).  out may be logits (with the same stride);
 *             it must not overlap otherwise.
 * vocab 1..2^30, n_rows 0..2^20, history_width below 2^30; n_rows * vocab
 * below 2^35 (DSIM_ERANGE may be returned beyond: split the call).
 */
typedef struct {
    const void *logits;
    void *out;
    int64_t logits_stride, out_stride, n_rows;
    int32_t vocab, dtype;
    const int32_t *history, *prompt_len, *history_len;
    int64_t history_stride;
    int32_t history_width, n_bias;
    const float *repetition, *frequency, *presence;
    const int32_t *bias_id;
    const float *bias;
    const uint32_t *mask;
    int64_t mask_stride;
} dsim_logits;

DSIM_API dsim_status dsim_logit_adjust(const dsim_logits *args, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DSIM_OPS_H */
