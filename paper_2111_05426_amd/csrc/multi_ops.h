// multi_ops.h -- declarations shared by the translation units of the operators
// of a step of several tokens (include/dsim_multi_ops.h).
#pragma once

#include "../../include/dsim_multi_ops.h"
#include "ops.h"

namespace dsim {

constexpr int kLayersAtOnce = 64;   // caches of one launch: their pointers are kernel arguments

// Positions on several axes beside a call of dsim_kv_append: pairs up to
// end[a] (from end[a - 1]) turn by axis a.
struct AxesArgs {
    const int32_t *pos;
    int32_t n_axes, end[DSIM_MAX_AXES];
};

// One call of dsim_prompt_attention or dsim_tree_attention.
struct RowsArgs {
    dsim_kv_cache c;
    dsim_queries q;
    const int32_t *prefix_len, *first_key;   // prompts
    const uint32_t *mask;                    // trees
    const int32_t *depth;
    int64_t mask_stride;
    int32_t mask_words;
    bool tree;
};

// The keys and values of up to kLayersAtOnce caches of one shape.
struct Layers {
    void *p[2 * kLayersAtOnce];
    int64_t n_pages, page_stride, slot_stride, head_stride;   // of 16-byte pieces
    int32_t n, n_heads, page_size, chunks;                    // chunks: 16-byte pieces of a row
};

struct CompactArgs {
    const int32_t *table, *start, *keep, *n_keep;
    int32_t *status;
    int64_t table_stride, keep_stride;
    int32_t n_seq, table_width, keep_width;
    uint32_t div_mul, div_shift;   // t / page_size = t * div_mul >> div_shift
};

// Kernel launchers (each returns DSIM_OK or DSIM_EHIP).
dsim_status launch_append_axes(const AppendArgs &a, const AxesArgs &x, hipStream_t s);
size_t rows_workspace(int64_t n_tok, int32_t n_seq, int32_t n_q_heads, int32_t n_heads, int32_t head_dim);
dsim_status launch_rows(const RowsArgs &a, hipStream_t s);
dsim_status launch_reserve(const dsim_page_pool &p, const int32_t *seq_len, const int32_t *new_len, int32_t *status,
                           hipStream_t s);
dsim_status launch_release(const dsim_page_pool &p, int64_t n, const int32_t *row, const int32_t *keep_len,
                           int32_t *status, hipStream_t s);
dsim_status launch_fork(const Layers *layers, int n_launches, const dsim_page_pool &p, int32_t *seq_len, int64_t n,
                        const int32_t *src, const int32_t *dst, int32_t *status, hipStream_t s);
dsim_status launch_copy_pages(const Layers &layers, int64_t n, const int32_t *src, const int32_t *dst, hipStream_t s);
dsim_status launch_compact(const Layers &layers, const CompactArgs &a, hipStream_t s);

}  // namespace dsim
