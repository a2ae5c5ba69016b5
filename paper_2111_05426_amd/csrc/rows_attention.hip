// rows_attention.hip -- dsim_prompt_attention and dsim_tree_attention on the
// host: their workspace and their launch; the kernels are in
// rows_attention.h.
#include "rows_attention.h"

namespace dsim {
namespace rows {

// Rows of a block: about what the average sequence has (more are multiplied as
// padding, fewer read the keys again).  us with the size taken and another: 8
// rows a sequence, 32 9.6, 64 9.9; 60 rows, 64 9.0, 32 9.6, 128 9.7; 64 rows over
// 64 contexts, 64 153, 32 278, 128 178; 384 rows over an e4m3 cache, 128 865, 256 979; 32
// prompts of 1,200 rows, 128 116, 256 125; 64 of 2,200, 256 523, 128 575; one of 32,768,
// 256 797, 128 856.  (Against it: drafts of 32 rows over 64 and 256 contexts of some
// hundred tokens, heads of 128, 32 42 and 169, 128 36 and 126.)  fp32 has no registers
// for 256, and with blocks of 64 documents took 199 for 158.
static int rows_of(int64_t n_tok, int32_t n_seq, int32_t group, int32_t head_dim, bool f32)
{
    const int64_t average = n_seq > 0 ? (n_tok * group + n_seq - 1) / n_seq : 0;
    if (average <= 32 && head_dim <= 128) return 32;
    if (average <= 64) return 64;
    return average <= 1536 || head_dim > 128 || f32 ? 128 : 256;
}

static int64_t blocks(int64_t n_tok, int32_t n_seq, int32_t group, int rows)
{
    return (n_tok * group + rows - 1) / rows + n_seq;
}

struct Layout {
    size_t cost, span, first, base, cut, part, end;
    Layout(int64_t n_blocks, int32_t n_seq, int rows, int32_t d)
    {
        const auto up = [](size_t x) { return (x + 15) / 16 * 16; };
        cost = 0;
        span = up(cost + 8 * ((size_t)n_blocks + 1));
        first = up(span + 8 * (size_t)n_blocks);
        base = up(first + 4 * ((size_t)n_seq + 1));
        cut = up(base + 8 * ((size_t)n_seq + 1));
        part = cut + sizeof(int4) * kMaxGrid;
        end = part + (size_t)(rows == 256 ? kCus : kMaxGrid) * 2 * rows * (d + 2) * sizeof(float);
    }
};

}  // namespace rows

size_t rows_workspace(int64_t n_tok, int32_t n_seq, int32_t n_q_heads, int32_t n_heads, int32_t head_dim)
{
    const int32_t group = n_q_heads / n_heads;
    size_t most = 0;
    for (const bool f32 : {false, true}) {   // (whatever the type)
        const int rows = rows::rows_of(n_tok, n_seq, group, head_dim, f32);
        const size_t bytes = rows::Layout(rows::blocks(n_tok, n_seq, group, rows), n_seq, rows, head_dim).end;
        if (bytes > most) most = bytes;
    }
    return most;
}

dsim_status launch_rows(const RowsArgs &a, hipStream_t s)
{
    using namespace rows;
    Params p{};
    p.k = a.c.k;
    p.v = a.c.v;
    p.q = a.q.q.data;
    p.out = a.q.out.data;
    p.k_scale = a.c.k_scale;
    p.v_scale = a.c.v_scale;
    p.slopes = a.q.slopes;
    p.table = a.c.block_table;
    p.start = a.q.start;
    p.len = a.q.len;
    p.prefix_len = a.prefix_len;
    p.first_key = a.first_key;
    p.depth = a.depth;
    p.mask = a.mask;
    p.lse = a.q.lse;
    p.status = a.q.status;
    p.n_pages = a.c.n_pages;
    p.page_stride = a.c.page_stride;
    p.slot_stride = a.c.slot_stride;
    p.head_stride = a.c.head_stride;
    p.table_stride = a.c.table_stride;
    p.q_row = a.q.q.row_stride;
    p.q_head = a.q.q.head_stride;
    p.out_row = a.q.out.row_stride;
    p.out_head = a.q.out.head_stride;
    p.mask_stride = a.mask_stride;
    p.mask_words = a.mask_words;
    p.n_tok = a.q.n_tok;
    p.scale = a.q.scale;
    p.cap = a.q.cap;
    p.n_seq = a.c.n_seq;
    p.n_heads = a.c.n_heads;
    p.n_q_heads = a.q.n_q_heads;
    p.d = a.c.head_dim;
    p.page_size = a.c.page_size;
    p.table_width = a.c.table_width;
    p.window = a.q.window;
    p.group = a.q.n_q_heads / a.c.n_heads;
    p.rows = rows_of(p.n_tok, p.n_seq, p.group, p.d, a.q.dtype == DSIM_F32);
    // A cap of at most 128 takes tanh's short form over many rows of 16 bits: off
    // by 2^-21 of the cap, what the longer one is of a score half as large, and at
    // most 2^-14 of a weight.  Chunks of prompts 489 us, by the longer form 652; trees
    // over e4m3 866 and 1,107; 64 trees of 16 nodes over 1 to 4,096 tokens would take
    // 167 for 181, but few rows keep their scores' bits.
    p.short_cap = p.cap > 0.0f && p.cap <= 128.0f && !p.slopes && a.q.dtype != DSIM_F32 && p.rows >= 128;
    p.max_blocks = blocks(p.n_tok, p.n_seq, p.group, p.rows);
    p.tree = a.tree;
    const Layout at(p.max_blocks, p.n_seq, p.rows, p.d);
    char *ws = static_cast<char *>(a.q.workspace);
    p.cost = reinterpret_cast<int64_t *>(ws + at.cost);
    p.span = reinterpret_cast<int2 *>(ws + at.span);
    p.first = reinterpret_cast<int32_t *>(ws + at.first);
    p.base = reinterpret_cast<int64_t *>(ws + at.base);
    p.cut = reinterpret_cast<int4 *>(ws + at.cut);
    p.part = reinterpret_cast<float *>(ws + at.part);
    // ceil(2^(31 + l) / n), l = ceil(log2 n): exact for t < 2^31
    const auto divisor = [](int32_t n, uint32_t &mul, uint32_t &shift) {
        int l = 0;
        while ((1 << l) < n) ++l;
        shift = 31 + l;
        mul = (uint32_t)((((uint64_t)1 << shift) + n - 1) / n);
    };
    divisor(p.page_size, p.page_mul, p.page_shift);
    divisor(p.group, p.group_mul, p.group_shift);
    // A workgroup a block, without plan and join, where no block is long and
    // there are few: one request's prompt of 60 tokens 9.0 us, planned and joined
    // 16.4, its drafts 9.9 and 17.4; 128 prompts of 10 to 100 tokens of 32 / 8 heads
    // 75 and 83 (512 of them 305 and 272), 256 drafts over 10 to 500 keys of 12
    // heads of 64 94.6 and 100, of 32 / 8 heads of 128 169 and 163.  Each finds
    // its sequence among all, 64 at a time, so there are few of those too.  (By the
    // table's room, for lengths are on the device: under a table of more places a
    // short request is planned.)
    const int64_t most = (int64_t)p.table_width * p.page_size;
    p.direct = most <= 1024 && p.n_seq <= 256 && p.max_blocks * p.n_heads <= 8 * kMaxGrid;
    if (a.q.dtype == DSIM_F32) return rows::launch_f32(p, s);
    return (a.q.dtype == DSIM_F16 ? rows::launch_f16 : rows::launch_bf16)(p, a.c.dtype == DSIM_E4M3, s);
}

}  // namespace dsim
