/*
 * dsim_multi_ops.h -- C ABI of the operators of a step of several tokens.
 *
 * Next to the step that gives every sequence one token (dsim_ops.h) a program
 * that serves a transformer runs steps of many: prompts and chunks of them,
 * trees of drafted tokens that are checked at once, searches that fork a
 * sequence into several.  The operators here work on the same paged cache:
 * attention of prompts and of drafted trees, the append with positions apart
 * from the places in the cache and on several axes, the pages' counts, and
 * moving what stays of a sequence to its front.
 *
 * The conventions of dsim_ops.h hold for every call: arguments validated on
 * the host before any launch, everything enqueued on `hip_stream`, no
 * allocation, no memset, nothing kept between calls but what the caller's
 * buffers hold, calls may be captured into a HIP graph, results are
 * deterministic.  What only device data shows never aborts: it sets bits of a
 * status word and no memory outside the buffers is touched.
 */
#ifndef DSIM_MULTI_OPS_H
#define DSIM_MULTI_OPS_H

#include "dsim_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* more status bits */
#define DSIM_ST_NO_PAGE 1024      /* there are not enough free pages                                   */
#define DSIM_ST_SHARED_PAGE 2048  /* what would be written lies in a page that others hold too         */
#define DSIM_ST_IN_USE 4096       /* a row of the block table that should be empty holds pages         */

#define DSIM_MAX_AXES 4

/*
 * dsim_kv_append_axes -- dsim_kv_append with the place in the cache and the
 * rotation's positions apart, and with positions on several axes.  Token t
 * goes to place slot[t] of sequence seq[t].  The rot_dim / 2 rotated pairs are
 * cut into n_axes sections: the first sections[0] pairs turn by the angles of
 * row pos[t * n_axes + 0] of rope, the next sections[1] by those of row
 * pos[t * n_axes + 1], and so on.  Pair i uses column i of its row, on
 * whichever axis.  A drafted token's angle goes by its depth and its place by
 * its number (one axis); tokens of images and video have a time, a height and
 * a width.
 *   n_axes:   1..DSIM_MAX_AXES with rope; without, pos may be NULL
 *   sections: host array [n_axes], each >= 0, the sum rot_dim / 2
 * Everything else is dsim_kv_append's.  A slot outside the table or a
 * position outside rope (also one on an axis of no pairs) sets
 * DSIM_ST_BAD_POSITION.
 */
DSIM_API dsim_status dsim_kv_append_axes(const dsim_kv_cache *cache, int64_t n_tok, int32_t dtype, const dsim_rows *k,
                                         const dsim_rows *v, const dsim_rows *q, const dsim_rows *q_out,
                                         int32_t n_q_heads, const int32_t *seq, const int32_t *slot,
                                         const int32_t *pos, int32_t n_axes, const int32_t *sections,
                                         const float *rope, int64_t n_rope, int32_t rot_dim, int32_t interleaved,
                                         int32_t *status, void *hip_stream);

/*
 * The queries of a step: the tokens of all sequences, one sequence's behind
 * another's.  Tokens start[s] .. start[s + 1] - 1 belong to sequence s; start
 * has n_seq + 1 entries and must not descend.  Rows of q outside every
 * sequence (padding) leave their rows of out and lse as they were.  Query
 * head h reads cache head h / (n_q_heads / n_heads).  For a token at position
 * p and a key at position j that it attends to:
 *   x = scale * q . k_j;   x = cap * tanh(x / cap), if cap > 0;
 *   x = x - slopes[h] * |p - j|, if there are slopes;
 *   o = sum_j exp(x_j) v_j / sum_j exp(x_j),   lse = log sum_j exp(x_j)
 * A token that attends to nothing has o = 0 and lse = -inf; keys that it does
 * not attend to weigh nothing whatever they hold, and an attended value that is
 * not finite makes its element of o infinite or NaN.  Scores, statistics and
 * sums are fp32 (exponentials off by 2^-21, in 16 bits tanh by 2^-20 of itself or
 * 2^-21 of the cap); in 16 bits a weight enters the second sum as two numbers of
 * the type (off by 2^-16, fp16 2^-22, and fp16's below 2^-36 of the largest are
 * 0); the result is rounded once to out's type.
 *   q, out: n_tok rows of n_q_heads heads of `dtype`: the cache's type, or
 *           DSIM_F16 / DSIM_BF16 with an e4m3 cache; out may be q (with its
 *           strides), it must not overlap otherwise
 *   scale:  in [-2^126, 2^126];   cap: 0 (none) or in [2^-60, 2^60], and
 *           |scale| / cap 0 or in [2^-126, 2^126]; with a cap or slopes the
 *           scores themselves have to stay in fp32's range, and scale times
 *           k_scale in the ranges of scale
 *   slopes: device array [n_q_heads] or NULL
 *   lse:    device array [n_tok][n_q_heads] or NULL
 *   status: device array [n_seq] or NULL: 0 or DSIM_ST_* bits.  BAD_POSITION:
 *           tokens outside q (nothing is written for them), or more keys than
 *           the block table has places for (out and lse are NaN).  BAD_PAGE:
 *           a token attends to a key whose page lies outside the cache; out
 *           and lse of those tokens are NaN.
 *   workspace: device buffer of at least dsim_prompt_attention_workspace(...)
 *           bytes, 16-byte aligned, in use until hip_stream has passed the
 *           call; it needs no clearing and keeps nothing for later calls.
 * n_tok * n_q_heads <= 2^31 - 256, n_seq <= 2^20.
 */
typedef struct {
    dsim_rows q, out;
    int64_t n_tok;
    const int32_t *start;   /* [n_seq + 1] */
    const int32_t *len;     /* [n_seq], see the calls */
    const float *slopes;
    float *lse;
    int32_t *status;
    void *workspace;
    size_t ws_bytes;
    float scale, cap;
    int32_t dtype, n_q_heads, window;
} dsim_queries;

/* 0 for arguments that the calls refuse. */
DSIM_API size_t dsim_prompt_attention_workspace(int64_t n_tok, int32_t n_seq, int32_t n_q_heads, int32_t n_heads,
                                                int32_t head_dim);

/*
 * dsim_prompt_attention -- the new tokens of every sequence attend to its
 * cached keys and values, their own among them.  With L = queries.len[s] (all
 * keys of the sequence, the new tokens' included; negative: the sequence's
 * rows and status are left as they were) and n tokens, token i has position
 * p = L - n + i and attends to the keys
 *   max(p + 1 - window (if window > 0), first_key[t])  <=  j  <
 *   max(p + 1, min(prefix_len[s], L))
 *   prefix_len: device array [n_seq] or NULL: the first keys, which every
 *               token sees (a prefix that attends to itself in both
 *               directions)
 *   first_key:  device array [n_tok] or NULL: the first key of the token's
 *               document
 * n > L sets DSIM_ST_BAD_POSITION.
 */
DSIM_API dsim_status dsim_prompt_attention(const dsim_kv_cache *cache, const dsim_queries *queries,
                                           const int32_t *prefix_len, const int32_t *first_key, void *hip_stream);

/*
 * dsim_tree_attention -- drafted tokens attend to their sequence's context
 * and to one another as a mask says.  queries.len[s] is the length L of the
 * context (negative: the sequence's rows and status are left as they were);
 * the key and value of its node i lie behind it at place L + i.  Node i is at
 * position p = L + depth[t] and attends to the context's keys
 *   max(0, p + 1 - window (if window > 0))  <=  j  <  L
 * and to the nodes m whose bit m % 32 of word m / 32 of its row of the mask
 * is 1 (its ancestors and itself; the window does not cut them: where a tree is
 * as deep as the window, its caller clears the bits of ancestors that a
 * token on its own would not attend to).  A node's position is that of its key
 * too.
 *   mask:  device array [n_tok][mask_stride] of 32-bit words, mask_words
 *          that are read; a sequence of more than 32 * mask_words nodes sets
 *          DSIM_ST_BAD_POSITION
 *   depth: device array [n_tok], values >= 0 (others count as 0); NULL (all
 *          0) without window and slopes
 */
DSIM_API dsim_status dsim_tree_attention(const dsim_kv_cache *cache, const dsim_queries *queries, const uint32_t *mask,
                                         int64_t mask_stride, int32_t mask_words, const int32_t *depth,
                                         void *hip_stream);

/*
 * The pages of a cache and who holds them.  Row s of the block table holds
 * held[s] pages, its first ones; refs[p] counts the rows that hold page p; bit
 * p % 32 of word p / 32 of free is 1 where that is 0.  A pool begins with refs
 * and held 0 and the bits of all pages set (none behind the last).  All layers
 * of a model share a pool and a table.  Calls on one pool go one after another
 * (on one stream, or ordered).
 */
typedef struct {
    int32_t *refs;          /* [n_pages]                    */
    uint32_t *free;         /* [(n_pages + 31) / 32]        */
    int32_t *held;          /* [n_seq]                      */
    int32_t *block_table;   /* [n_seq][table_stride]        */
    int64_t n_pages, table_stride;
    int32_t n_seq, table_width, page_size;
} dsim_page_pool;

/*
 * dsim_kv_reserve -- pages for new_len[s] places in every row (negative: the
 * row and its status are left as they were; a row that holds enough already
 * stays as it is).  The lowest-numbered free pages are dealt out in order of
 * rows and places.  A row whose pages cannot all be had gets none, and neither
 * do the rows after it that need some.
 *   seq_len: device array [n_seq]: the places in use.  A row that is to grow
 *            beyond them writes to the pages that it holds already from place
 *            seq_len on, up to new_len: where other rows hold one of those too,
 *            writing would change theirs: DSIM_ST_SHARED_PAGE, no pages.
 *            (dsim_kv_release gives back those that lie behind seq_len,
 *            dsim_kv_fork makes a copy of the one in which it ends.)
 *   status:  device array [n_seq]: 0, DSIM_ST_NO_PAGE, DSIM_ST_SHARED_PAGE,
 *            DSIM_ST_BAD_POSITION (more places than the table has, or
 *            seq_len outside what the row holds) or DSIM_ST_BAD_PAGE (one of
 *            those pages lies outside the cache)
 */
DSIM_API dsim_status dsim_kv_reserve(const dsim_page_pool *pool, const int32_t *seq_len, const int32_t *new_len,
                                     int32_t *status, void *hip_stream);

/*
 * dsim_kv_release -- row row[i] gives back the pages behind its first
 * keep_len[i] places: their counts go down, those that nobody holds any more
 * are free, and the row's entries become -1.  row[i] < 0: nothing.  The same
 * row twice is released to the lesser length.
 *   status: device array [n] or NULL: 0, DSIM_ST_BAD_SEQUENCE, or
 *           DSIM_ST_BAD_PAGE (an entry outside the cache or without a count,
 *           which is left out; of the same row twice, either may have it)
 */
DSIM_API dsim_status dsim_kv_release(const dsim_page_pool *pool, int64_t n, const int32_t *row, const int32_t *keep_len,
                                     int32_t *status, void *hip_stream);

/*
 * dsim_kv_fork -- row dst[i] becomes a second holder of what row src[i] has
 * in its first seq_len[src[i]] places: whole pages are shared, the places of
 * a page in which that length ends are copied to a page of its own (the
 * lowest-numbered free ones, in order of i) in every layer.  seq_len[dst[i]]
 * becomes that length.
 *   layers: host array of n_layers caches of the same shape, strides and
 *           type, whose pages the pool counts (their block tables are not
 *           looked at)
 *   status: device array [n]: 0 or
 *           DSIM_ST_BAD_SEQUENCE  dst[i] or src[i] outside the table, or
 *                                 src[i] an empty row among the call's dst
 *           DSIM_ST_IN_USE        dst[i] holds pages, or an earlier fork of
 *                                 the call has it, also one that is refused
 *           DSIM_ST_BAD_POSITION  seq_len[src[i]] outside what the row holds
 *           DSIM_ST_NO_PAGE       no page is left for it (nor for later ones
 *                                 that need one)
 *           and then nothing of the fork is done; with DSIM_ST_BAD_PAGE
 *           (entries of src outside the cache) it is, without those.
 * dst[i] < 0 is padding: nothing is done, and its status is 0.  A row that
 * holds pages stays as it is though it is among the call's dst, and may be
 * another fork's src.
 */
DSIM_API dsim_status dsim_kv_fork(const dsim_kv_cache *layers, int32_t n_layers, const dsim_page_pool *pool,
                                  int32_t *seq_len, int64_t n, const int32_t *src, const int32_t *dst,
                                  int32_t *status, void *hip_stream);

/*
 * dsim_kv_copy_pages -- page dst[i] of every layer becomes what page src[i]
 * is.  A pair with a number below 0 is padding, one with a number outside the
 * cache does nothing.  No page may be dst twice, nor dst and another pair's
 * src: what such pages hold then is open.
 */
DSIM_API dsim_status dsim_kv_copy_pages(const dsim_kv_cache *layers, int32_t n_layers, int64_t n, const int32_t *src,
                                        const int32_t *dst, void *hip_stream);

/*
 * dsim_kv_compact -- of sequence s the places start[s] + keep[s][j], j <
 * n_keep[s], move to start[s] + j in every layer, as if all were read before
 * any is written.  The pages that are written to must be held by one row of
 * the table only, and once.  keep[s] must ascend (from 0 or more); it ends before the
 * first entry that does not.  What was behind the last of them stays as it is.
 *   layers:  as above, with layers[0]'s block table and n_seq
 *   keep:    device array [n_seq][keep_stride], keep_width entries that may
 *            be read, at most 2^30; n_keep is clamped to 0..keep_width
 *   status:  device array [n_seq] or NULL: 0, DSIM_ST_BAD_POSITION (entries
 *            that do not ascend, or places outside the block table: the
 *            list ends before them) or DSIM_ST_BAD_PAGE (of those that move a page
 *            outside the cache: that place is left out)
 * The accepted path of a drafted tree moves so to the end of its context, and
 * a context from which tokens are dropped closes up.
 */
DSIM_API dsim_status dsim_kv_compact(const dsim_kv_cache *layers, int32_t n_layers, const int32_t *start,
                                     const int32_t *keep, int64_t keep_stride, int32_t keep_width,
                                     const int32_t *n_keep, int32_t *status, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DSIM_MULTI_OPS_H */
