// paged_attention.hip -- dsim_paged_attention on the host: its workspace and
// its launch; the kernels are in paged_attention.h.
#include "paged_attention.h"

namespace dsim {

size_t attend_workspace(int32_t n_q_heads, int32_t n_heads, int32_t head_dim)
{
    using namespace attend;
    const int group = n_q_heads / n_heads, heads = group < kTileHeads ? group : kTileHeads;
    return (size_t)kMaxGrid * (sizeof(int4) + 2 * (size_t)part_size(heads, head_dim) * sizeof(float));
}

dsim_status launch_attend(const AttendArgs &a, hipStream_t s)
{
    using namespace attend;
    Params p{};
    p.k = a.c.k;
    p.v = a.c.v;
    p.q = a.q.data;
    p.out = a.out.data;
    p.k_scale = a.c.k_scale;
    p.v_scale = a.c.v_scale;
    p.table = a.c.block_table;
    p.seq_len = a.seq_len;
    p.lse = a.lse;
    p.status = a.status;
    p.cut = static_cast<int4 *>(a.ws);
    p.part = reinterpret_cast<float *>(p.cut + kMaxGrid);
    p.n_pages = a.c.n_pages;
    p.page_stride = a.c.page_stride;
    p.slot_stride = a.c.slot_stride;
    p.head_stride = a.c.head_stride;
    p.table_stride = a.c.table_stride;
    p.q_row = a.q.row_stride;
    p.q_head = a.q.head_stride;
    p.out_row = a.out.row_stride;
    p.out_head = a.out.head_stride;
    p.scale = a.scale * kLog2e;
    p.n_seq = a.c.n_seq;
    p.n_heads = a.c.n_heads;
    p.n_q_heads = a.n_q_heads;
    p.d = a.c.head_dim;
    p.page_size = a.c.page_size;
    p.table_width = a.c.table_width;
    // ceil(2^(31 + l) / n), l = ceil(log2 n): exact for t < 2^31
    int l = 0;
    while ((1 << l) < p.page_size) ++l;
    p.div_shift = 31 + l;
    p.div_mul = (uint32_t)((((uint64_t)1 << p.div_shift) + p.page_size - 1) / p.page_size);
    p.window = a.window;
    p.group = a.n_q_heads / a.c.n_heads;
    p.tiles_of_heads = (p.group + kTileHeads - 1) / kTileHeads;
    p.part_heads = p.group < kTileHeads ? p.group : kTileHeads;
    if (a.dtype == DSIM_F32) return attend::launch_f32(p, s);
    return (a.dtype == DSIM_F16 ? attend::launch_f16 : attend::launch_bf16)(p, a.c.dtype == DSIM_E4M3, s);
}

}  // namespace dsim
