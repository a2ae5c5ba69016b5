// ops.h -- declarations shared by the translation units of the single-token
// step's operators (include/dsim_ops.h).
#pragma once

#include "../../include/dsim_ops.h"
#include "internal.h"

namespace dsim {

constexpr int kMaxHeadDim = 256;
constexpr int kMaxHeads = 1024;
constexpr int kMaxBias = 4096;
constexpr int kTileHeads = 16;   // query heads of one cache head that a workgroup takes at once

// One call of dsim_kv_append.
struct AppendArgs {
    dsim_kv_cache c;
    dsim_rows k, v, q, q_out;
    const int32_t *seq, *pos;
    const float *rope;
    int32_t *status;
    int64_t n_tok, n_rope;
    int32_t dtype, n_q_heads, rot_dim, interleaved;
};

// One call of dsim_paged_attention.
struct AttendArgs {
    dsim_kv_cache c;
    dsim_rows q, out;
    const int32_t *seq_len;
    float *lse;
    int32_t *status;
    void *ws;
    float scale;
    int32_t dtype, n_q_heads, window;
};

inline int elem_size(int32_t dtype) { return dtype == DSIM_F32 ? 4 : dtype == DSIM_E4M3 ? 1 : 2; }

// Kernel launchers (each returns DSIM_OK or DSIM_EHIP).
dsim_status launch_append(const AppendArgs &a, hipStream_t s);
size_t attend_workspace(int32_t n_q_heads, int32_t n_heads, int32_t head_dim);
dsim_status launch_attend(const AttendArgs &a, hipStream_t s);
dsim_status launch_logits(const dsim_logits &a, hipStream_t s);

}  // namespace dsim
