// rows_attention.h -- the kernels of dsim_prompt_attention and
// dsim_tree_attention: attention of many rows (query tokens times the query
// heads of one cache head) over paged keys and values.
//
// Mathematics.  For a row i and the keys j it attends to, x_ij = score(q_i k_j),
// w_ij = exp2((x_ij - m_i) unit), o_i = sum_j w_ij v_j / sum_j w_ij, in one pass over
// the keys: m_i is a score at most SLACK base-2 units below the row's largest
// so far, and sums and outputs are scaled when one that is larger by more
// comes, which few tiles see.  Parts of a row with maxima m_a, m_b add up as sum
// exp2((m_a - m) unit) o_a + ....
//
// Layout.  A block is 32 WR rows (tokens times the query heads of a cache
// head) of one sequence.  Scores are taken transposed, S^T = K Q^T (32 keys x 32
// rows by 32x32x16 products, 32x32x2 in fp32): the lanes that hold a row's
// scores are then those that need its weights as the right operand of O^T =
// V^T P^T, whose left operand is read from shared memory transposed.  So
// weights never leave the registers, and a row's maximum and sum are 16 or 32
// elements of a lane and one exchange with lane + 32.  The order of keys that
// both products share is free, and is that of the score's elements.
//
// The blocks' tiles of all sequences and heads are laid end to end by one
// workgroup (k_plan: 6 to 8 us), cut into one equal run for each workgroup that
// is resident (neighbouring runs on one XCD, whose L2 then has a head's keys
// once), and what a cut goes through is joined (k_join: 11 to 16 us, tree_long's
// 25).  Short contexts take a workgroup a block and neither.
//
// What bounds it, on MI355X (bf16, heads of 128; the product of 8,192 cubed
// reaches 1,101 TFLOP/s here):
//   8,192 tokens of one prompt, 32 / 8 heads: 797 to 856 us, 642 to 690 TFLOP/s of
//     the formula's products, 963 to 1,035 of those that are made: the second is
//     made twice, for weights of two numbers.
//   16 chunks of 1 to 1,024 tokens behind 2,000, window 1,500, cap 50: 491 us, 410
//     TFLOP/s; a capped score takes two more transcendental instructions.
//   64 trees of 16 nodes over 1 to 4,096 tokens: 151 us, 3.7 TB/s of the cache,
//     of which plan and join 19.
//   4 trees of 48 nodes over 65,536 tokens in e4m3, 64 / 8 heads, cap 30: 885 us, 466
//     TFLOP/s: a tile is widened between two barriers.  (Widened a tile ahead
//     between the products, with two tiles in shared memory, and with weights of
//     one number 787 to 811 for 723; the compiler runs out of registers.)
//   fp32, 6 x 100 to 1,500 tokens of 3 documents, 12 heads of 80, a bias by
//     distance: 123 us, 27 TFLOP/s of 153; heads of 96 by their products, 1.7
//     times the pairs (documents end inside blocks of 128 rows), and 60 us to plan,
//     begin, end and join blocks of 9 tiles.
#pragma once

#include <type_traits>

#include "multi_ops.h"
#include "numeric.h"

namespace dsim {
namespace rows {

constexpr int kCus = 256;
constexpr int kMaxGrid = 2 * kCus;
constexpr int kJoin = 256;           // threads of the join
constexpr int kPlan = 1024;          // threads of the plan
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// What a block of rows costs beside its tiles, in tiles.  (Chunks of prompts, a
// long prompt, fp32 documents: 489, 797 and 123 us, with 4 493, 815 and 130, with
// 1 491, 840 and 118.  Trees, blocks of 64 rows: 150 us, with 2 158, with 8 more.)
constexpr int extra(int rows) { return rows >= 128 ? 2 : 4; }
constexpr int kMinTiles = 4;         // of a run at least: shorter ones only begin and end

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct Params {
    const void *k, *v, *q;
    void *out;
    const float *k_scale, *v_scale, *slopes;
    const int32_t *table, *start, *len, *prefix_len, *first_key, *depth;
    const uint32_t *mask;
    float *lse;
    int32_t *status;
    int64_t n_pages, page_stride, slot_stride, head_stride, table_stride, q_row, q_head, out_row, out_head, mask_stride;
    int64_t n_tok, max_blocks;
    // the plan, in the workspace
    int64_t *cost;        // [max_blocks + 1] sums of the blocks' costs, one head's
    int2 *span;           // [max_blocks] keys of a block
    int32_t *first;       // [n_seq + 1] sequences' first blocks
    int64_t *base;        // [n_seq + 1] the costs before them
    int4 *cut;            // [kMaxGrid]
    float *part;
    float scale, cap;     // scale: natural units
    int32_t n_seq, n_heads, d, page_size, table_width, window, mask_words;
    int32_t group, n_q_heads, rows;   // rows of a block
    bool tree, direct, short_cap;
    uint32_t page_mul, page_shift, group_mul, group_shift;   // t / n = t * mul >> shift, 0 <= t < 2^31
};

__device__ inline int32_t divide(int32_t t, uint32_t mul, uint32_t shift)
{
    return (int32_t)((uint64_t)(uint32_t)t * mul >> shift);
}

// A sequence of the call.
struct Seq {
    int32_t start, n, len;   // first token, tokens, length as given
    int32_t keys;            // all of them (none if bad)
    int32_t bad;             // its rows are NaN
    int32_t status;
};

__device__ inline Seq seq_of(const Params &p, int s)
{
    Seq x;
    x.start = p.start[s];
    x.len = p.len[s];
    const int32_t end = p.start[s + 1];
    x.n = 0;
    x.keys = 0;
    x.bad = x.status = 0;
    if (x.len < 0) return x;
    if (x.start < 0 || end < x.start || end > p.n_tok) {
        x.status = DSIM_ST_BAD_POSITION;
        return x;
    }
    x.n = end - x.start;
    const int64_t keys = p.tree ? (int64_t)x.len + x.n : x.len;
    if (keys > (int64_t)p.table_width * p.page_size || (p.tree ? x.n > 32 * (int64_t)p.mask_words : x.n > x.len))
        x.bad = x.status = DSIM_ST_BAD_POSITION;
    else
        x.keys = (int32_t)keys;
    return x;
}

__device__ inline int32_t blocks_of(const Params &p, const Seq &x)
{
    return (int32_t)(((int64_t)x.n * p.group + p.rows - 1) / p.rows);
}

// The keys that a token may attend to but for the mask of a tree: lo <= j <
// hi; position: that of the token.
struct Range {
    int32_t lo, hi, position;
};

__device__ inline Range range_of(const Params &p, const Seq &x, int32_t i, int32_t prefix, int32_t first_key, int32_t depth)
{
    Range r;
    if (p.tree) {
        r.position = (int32_t)min((int64_t)x.len + max(depth, 0), (int64_t)INT32_MAX);
        r.hi = x.len;
        r.lo = p.window > 0 ? max(r.position - p.window + 1, 0) : 0;
    } else {
        r.position = x.len - x.n + i;
        r.hi = min(max(r.position + 1, prefix), x.len);
        r.lo = max(p.window > 0 ? max(r.position - p.window + 1, 0) : 0, first_key);
    }
    if (x.bad || r.lo >= r.hi) r.lo = r.hi = 0;
    return r;
}

__device__ inline Range range_of(const Params &p, const Seq &x, int s, int32_t i)
{
    const int32_t t = x.start + i;
    return range_of(p, x, i, p.prefix_len ? p.prefix_len[s] : 0, p.first_key ? max(p.first_key[t], 0) : 0,
                    p.depth ? p.depth[t] : 0);
}

// Whether token i attends to a key.
__device__ inline bool attends(const Params &p, const Seq &x, int s, int32_t i, int32_t key)
{
    const Range r = range_of(p, x, s, i);
    if (key >= r.lo && key < r.hi) return true;
    if (!p.tree || key < x.len || key >= x.keys) return false;
    const int32_t node = key - x.len;
    return p.mask[(x.start + i) * p.mask_stride + node / 32] >> node % 32 & 1;
}

// The keys that some token of tokens i0 to i1 attends to lie in [x, y); with
// first keys, of every `lanes`-th of them.
__device__ inline int2 span_of(const Params &p, const Seq &x, int s, int32_t i0, int32_t i1, int lane, int lanes)
{
    if (x.bad) return make_int2(0, 0);
    if (p.tree) return make_int2(p.window > 0 ? min(max(x.len - p.window + 1, 0), x.len) : 0, x.keys);
    int lo = INT32_MAX, hi = 0;
    if (p.first_key) {
        for (int32_t i = i0 + lane; i <= i1; i += lanes) {
            const Range r = range_of(p, x, s, i);
            if (r.lo >= r.hi) continue;
            lo = min(lo, r.lo);
            hi = max(hi, r.hi);
        }
    } else {   // both grow with the token
        lo = range_of(p, x, s, i0).lo;
        hi = range_of(p, x, s, i1).hi;
    }
    return lo < hi ? make_int2(lo, hi) : make_int2(0, 0);
}

// (A last key may be 2^31 - 2: here and below nothing is added to a key that a tile
// further on might not fit.)
template <int KT> __device__ inline int32_t tiles_of(int2 span)
{
    return span.y > 0 ? (span.y - 1) / KT + 1 - span.x / KT : 1;
}

// Sum of x over the workgroup's threads before this one, and the total.
template <int THREADS> __device__ inline int64_t scan(int64_t x, int64_t *s, int64_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t incl = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 63) s[wave] = incl;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += s[w];
        total += s[w];
    }
    __syncthreads();
    return before + incl - x;
}

// Sum of x over the lanes up to this one.
__device__ inline int32_t prefix(int32_t x)
{
#define DSIM_STEP(control, rows) x += __builtin_amdgcn_update_dpp(0, x, control, rows, 0xf, true)
    DSIM_STEP(0x111, 0xf);   // within rows of 16, from 1, 2, 4 and 8 lanes before
    DSIM_STEP(0x112, 0xf);
    DSIM_STEP(0x114, 0xf);
    DSIM_STEP(0x118, 0xf);
    DSIM_STEP(0x142, 0xa);   // the last of a row to the next one
    DSIM_STEP(0x143, 0xc);   // the last of the first half to the second
#undef DSIM_STEP
    return x;
}

// The largest i < n with a(i) <= x, where a does not descend and a(0) <= x:
// 64 probes at a time, the same for all lanes.
template <class A> __device__ inline int32_t find(A a, int32_t n, int64_t x)
{
    const int lane = threadIdx.x & 63;
    int32_t lo = 0;
    while (n > 1) {
        const int32_t step = (n + 63) / 64, i = lo + lane * step;
        const bool le = lane * step < n && a(i) <= x;
        const int last = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(le));   // (lane 0's is)
        n = min(step, n - last * step);
        lo += last * step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Blocks of rows, their keys and what they cost, and the sequences' status.
constexpr int kLanes = 16;   // that look at the tokens of a block together
template <int KT> __global__ __launch_bounds__(kPlan) void k_plan(Params p)
{
    __shared__ int64_t s_sum[kPlan / 64];
    __shared__ int32_t s_first[kPlan + 1];   // what fits of first
    int64_t before = 0, total;
    for (int s0 = 0; s0 < p.n_seq; s0 += kPlan) {
        const int s = s0 + threadIdx.x;
        Seq x{};
        int64_t n = 0;
        if (s < p.n_seq) {
            x = seq_of(p, s);
            n = blocks_of(p, x);
        }
        const int64_t at = before + scan<kPlan>(n, s_sum, total);
        // (more rows than tokens: starts that descend; what does not fit is refused)
        if (s < p.n_seq) {
            p.first[s] = (int32_t)min(at, p.max_blocks);
            if (s < kPlan) s_first[s] = (int32_t)min(at, p.max_blocks);
            if (at + n > p.max_blocks) x.status = DSIM_ST_BAD_POSITION;
            if (p.status && x.len >= 0) p.status[s] = x.status;
        }
        before += total;
    }
    const int32_t n = (int32_t)min(before, p.max_blocks);
    if (threadIdx.x == 0) p.first[p.n_seq] = n;
    __syncthreads();
    // The blocks' keys, by several lanes where each token has its own.
    const int lanes = p.first_key ? kLanes : 1;
    for (int32_t at = threadIdx.x; at < n * lanes; at += kPlan) {
        const int32_t b = at / lanes;
        int s = 0, end = p.n_seq;   // the last sequence that begins at the block or before
        const int32_t *const first = p.n_seq <= kPlan ? s_first : p.first;
        while (end - s > 1) {
            const int mid = (s + end) / 2;
            (first[mid] <= b ? s : end) = mid;
        }
        const Seq x = seq_of(p, s);
        const int32_t r0 = (b - first[s]) * p.rows, r1 = min(r0 + p.rows, x.n * p.group);
        int2 span = span_of(p, x, s, r0 / p.group, (r1 - 1) / p.group, at % lanes, lanes);
        if (lanes > 1) {
            if (span.y == 0) span.x = INT32_MAX;
#pragma unroll
            for (int o = 1; o < kLanes; o <<= 1) {
                span.x = min(span.x, __shfl_xor(span.x, o));
                span.y = max(span.y, __shfl_xor(span.y, o));
            }
            if (span.y == 0) span.x = 0;
        }
        if (at % lanes == 0) p.span[b] = span;
    }
    __syncthreads();
    before = 0;
    for (int32_t b0 = 0; b0 < n; b0 += kPlan) {
        const int32_t b = b0 + threadIdx.x;
        const int64_t cost = b < n ? tiles_of<KT>(p.span[b]) + extra(p.rows) : 0;
        const int64_t at = before + scan<kPlan>(cost, s_sum, total);
        if (b < n) p.cost[b] = at;
        before += total;
    }
    if (threadIdx.x == 0) p.cost[n] = before;
    __syncthreads();
    for (int s = threadIdx.x; s <= p.n_seq; s += kPlan) {
        const int32_t first = s == p.n_seq ? n : p.first[s];
        p.base[s] = first == n ? before : p.cost[first];
    }
}

// What is not finite of 16 bytes of T becomes 0; whether there was any.
template <class T> __device__ inline bool clean(u32x4 &x)
{
    constexpr uint32_t top = __is_same(T, f16) ? 0x7c00u : 0x7f80u;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t keep = ~0u;
        if (sizeof(T) == 4) {
            if ((x[i] & 0x7f800000u) == 0x7f800000u) keep = 0;
        } else {
            if ((x[i] & top) == top) keep &= 0xffff0000u;
            if ((x[i] & top << 16) == top << 16) keep &= 0xffffu;
        }
        odd |= keep != ~0u;
        x[i] &= keep;
    }
    return odd;
}

// eight e4m3 in fp16 or bf16, exactly
template <class T, bool HIGH> __device__ inline vec<T, 2> widen2(uint32_t w)
{
    if constexpr (__is_same(T, f16))
        return __builtin_bit_cast(vec<T, 2>, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH));
    else
        return __builtin_bit_cast(vec<T, 2>, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}

template <class T> __device__ inline vec<T, 8> widen8(uint32_t lo, uint32_t hi)
{
    const vec<T, 2> a = widen2<T, false>(lo), b = widen2<T, true>(lo), c = widen2<T, false>(hi), d = widen2<T, true>(hi);
    return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The largest, or least, of the 32 lanes of each half.
template <bool LARGEST> __device__ inline int32_t across(int32_t x)
{
    const auto of = [](int32_t a, int32_t b) { return LARGEST ? max(a, b) : min(a, b); };
    x = of(x, __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true));   // rows of 16, turned by 8, 4, 2, 1
    x = of(x, __builtin_amdgcn_mov_dpp(x, 0x124, 0xf, 0xf, true));
    x = of(x, __builtin_amdgcn_mov_dpp(x, 0x122, 0xf, 0xf, true));
    x = of(x, __builtin_amdgcn_mov_dpp(x, 0x121, 0xf, 0xf, true));
    const auto y = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
    return of((int32_t)y[0], (int32_t)y[1]);
}

__device__ inline vec<float, 2> halves(float x)   // those of lanes r and 32 + r
{
    const auto y = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return {__builtin_bit_cast(float, (uint32_t)y[0]), __builtin_bit_cast(float, (uint32_t)y[1])};
}

// tanh, off by less than 2^-20 of itself (fp32: the library's)
template <bool F32> __device__ inline float tanh_of(float y)
{
    if constexpr (F32) {
        return tanhf(y);
    } else {
        const float a = fabsf(y), z = y * y;
        const float big = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(2.0f * kLog2e * a) + 1.0f);
        // y - y^3 / 3 + 2 y^5 / 15 - 17 y^7 / 315
        float small = a * (1.0f + z * (-0.33333333f + z * (0.13333333f + z * -0.05396825f)));
        small = a < 0.2f ? small : big;
        return copysignf(small, y);
    }
}

// Scores over the cap become capped ones in base-2 units (cap2).
template <bool F32> __device__ inline void cap_of(f32x16 &x, float cap2)
{
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = tanh_of<F32>(x[e]) * cap2;
}

// Sums held against the maximum `from`, against `to`: see paged_attention.h.
__device__ inline float rescale(float from, float to, float scale)
{
    return from == -HUGE_VALF ? 1.0f : __builtin_amdgcn_exp2f((from - to) * scale);
}

// The largest score that is weighed against m: `slack` base-2 units above it.
// Where fp32's own steps are that wide, m alone: rounded up to the next one the
// sum may be twice the slack above m, and fp16's weight of a score that high
// infinite (2^(11 + 4) is the largest that it is meant to have; half a unit
// more is in its range).
__device__ inline float limit_of(float m, float slack, float unit)
{
    const float y = m + slack / unit;
    return (y - m) * unit > slack + 0.5f ? m : y;
}

// T: type of the queries, CT: of the cache, DP: the head's size padded, WR:
// blocks of 32 rows in a workgroup.  Its waves, four, or eight of 256 rows, are
// WR x WK: those of a block of rows share out the keys of a tile.
// WHOLE: pages of a multiple of 16 slots, so that 16 keys lie in one page.
template <class T, class CT, int DP_, int WR_, bool WHOLE> struct Shape {
    static constexpr int DP = DP_, WR = WR_, WAVES = WR == 8 ? 8 : 4, BLOCK = 64 * WAVES, WK = WAVES / WR;
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int U = !F32 && WR >= 4 ? 2 : 1;          // times 32 keys of a tile for each wave
    // A tile is H steps of KS keys, KW of them a wave's: what has to be done
    // once a tile is done less often.
    static constexpr int H = (WR == 8 || (WR == 4 && DP == 64)) && sizeof(T) == 2 ? 2 : 1;
    static constexpr int KW = 32 * U, KS = WK * KW, KT = KS * H, M = 32 * WR;
    static constexpr int PITCH = DP * sizeof(T);               // of a row in shared memory
    static constexpr int NC = PITCH / 16;                      // its pieces of 16 bytes
    static constexpr int IN = DP * sizeof(CT) / 16;            // those of a row of the cache
    static constexpr int NQ = KT * IN / BLOCK;                // that a thread loads, of keys and of values
    static constexpr int TILE = KT * PITCH;                    // bytes of a tile's keys or values
    // Keys and values go to shared memory by themselves, a tile ahead, where
    // they need no widening and two tiles fit.
    static constexpr bool DMA = WHOLE && sizeof(CT) == sizeof(T) && 4 * TILE <= 144 * 1024;
    static constexpr int SUMS = 32 * DP * 4 * (WK - 1) * WR;   // outputs of waves that are joined
    static constexpr int TILES = (DMA ? 4 : 2) * TILE, LDS = TILES > SUMS ? TILES : SUMS;
    static constexpr int PER_CU = DP <= 128 && WR < 8 && LDS <= 78 * 1024 ? 2 : 1;   // workgroups, all resident at once
    static constexpr int PER_SIMD = PER_CU * WAVES / 4;
    // Rows of a wave's share of a tile, in groups of one page.
    static constexpr int SHARE = KT / WAVES, GROUP = SHARE < 16 ? SHARE : 16, GROUPS = SHARE / GROUP;
    static constexpr int RI = 64 / IN > 0 ? 64 / IN : 1;       // rows of the cache that a wave loads at once
    static constexpr int LOADS = GROUP / RI;                   // loads of a group's keys
    // Offset for the weights' exponents.  fp16 ends at 2^-24: weights up to
    // 2^15 (2^11 where they are held against the largest) keep all that are
    // above 2^-36 of the largest, in steps of 2^-35 at the end.
    static constexpr float SLACK = __is_same(T, f16) ? 4.0f : 8.0f, UP = __is_same(T, f16) ? 11.0f : 0.0f;
    // Pieces of a row are permuted by its number so that the lanes that read
    // a column meet different banks: 16 rows' pieces of keys (16 bytes a
    // lane), 4 rows of 64 bytes of values (read transposed).
    __device__ static int key_piece(int row, int c) { return c ^ (NC == 8 ? row >> 1 & 7 : row & 15); }
    __device__ static int value_piece(int row, int c)
    {
        return F32 ? c : c ^ (NC == 8 ? (row >> 1 & 1) << 2 : (row & 3) << 2);
    }
};

// Shared memory by its 32-bit address.
using lds_char = __attribute__((address_space(3))) char;
__device__ inline uint32_t address(const void *p) { return (uint32_t)(uintptr_t)(const lds_char *)p; }
template <class V> __device__ inline V shared(uint32_t at)
{
    return *(const __attribute__((address_space(3))) V *)(uintptr_t)at;
}

// 16 bytes a lane from global memory to 1,024 bytes of shared memory, not
// waited for.  (The builtin makes every later read of shared memory wait for
// it: the compiler does not see that it is to another tile.  No register is
// written; arrived() stands before the barrier that the readers pass.)
__device__ inline void to_shared(const void *from, uint32_t off, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(from)
                 : "memory", "m0");
}

// The kernel's argument, read where it is needed: what few tiles need does not
// take scalar registers from the others.
template <class P> __device__ inline const P &argument()
{
    auto at = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const P *)at;
}

// x, which is the same for all lanes, kept in scalar registers from here on (not
// read again from the kernel's argument)
template <class V> __device__ inline V kept(V x)
{
    asm volatile("" : "+s"(x));
    return x;
}

// a value that is the same for all lanes, in scalar registers
__device__ inline int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
template <class P> __device__ inline const P *uniform(const P *p)
{
    const uint64_t x = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (const P *)((uint64_t)hi << 32 | lo);
}

// x, as if it might be another from here on: what follows from it is computed
// again instead of kept in registers
__device__ inline uint32_t again(uint32_t x)
{
    asm("" : "+v"(x));
    return x;
}

// N operands from shared memory and the products of each, four operands ahead
// of their products: the compiler on its own reads each right before its
// product and waits.  `first` has the first four; other(i) comes before the
// products of i to i + 3.
template <int N, class A, class Read, class Mul, class Other>
__device__ inline void in_order(A (&first)[4], Read read, Mul mul, Other other)
{
    constexpr int kOnly = 0x2 | 0x4;   // vector and scalar arithmetic may move across
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        A next[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + 4 + k < N) next[k] = read(i + 4 + k);
        other(i);
        __builtin_amdgcn_sched_barrier(kOnly);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < N) mul(i + k, first[k]);
        __builtin_amdgcn_sched_barrier(kOnly);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + 4 + k < N) first[k] = next[k];
    }
}

__device__ inline void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <class T> struct Mfma;
template <> struct Mfma<f16> {
    __device__ static f32x16 mul(vec<f16, 8> a, vec<f16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<bf16> {
    __device__ static f32x16 mul(vec<bf16, 8> a, vec<bf16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// The left operand of keys 16 k to 16 k + 15 of a tile's values: the lane's
// place of the first is `at`.
template <class T, int PITCH> __device__ inline vec<T, 8> values(uint32_t at, int k)
{
    using lds4 = __attribute__((address_space(3))) s16x4;
    s16x4 part[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
        part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)(at + (16 * k + 8 * j) * PITCH));
    return __builtin_bit_cast(vec<T, 8>, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ inline float value_of(float x) { return x; }
__device__ inline float value_of(f16 x) { return (float)x; }
__device__ inline float value_of(bf16 x) { return (float)x; }
__device__ inline float value_of(e4m3 x) { return (x.bits & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f; }   // (or a finite one)

// A part of a block: the outputs of its rows, their maxima and sums.
struct Part {
    float *o, *m, *l;
    __device__ static Part of(const Params &p, int64_t slot)
    {
        float *o = p.part + slot * p.rows * (p.d + 2), *m = o + (int64_t)p.rows * p.d;
        return {o, m, m + p.rows};
    }
};

template <class T>
__device__ inline void write_row(const Params &p, int64_t t, int head, int d, f32x4 x)
{
    *reinterpret_cast<vec<T, 4> *>(static_cast<T *>(p.out) + t * p.out_row + head * p.out_head + d) = from_f32<T, 4>(x);
}

// What a row's outputs are multiplied by.  (One that attends to nothing has
// the sum 0, one that attends to a bad page NaN.)
__device__ inline float share_of(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

__device__ inline void write_lse(const Params &p, int64_t t, int head, float m, float unit, float offset, float l, float up)
{
    if (p.lse)
        p.lse[t * p.n_q_heads + head] = l == 0.0f ? -HUGE_VALF : (m * unit + offset + (__builtin_log2f(l) - up)) * kLn2;
}

// The scores' way from a product x with a cache head's keys (times the scales'
// sign) to a base-2 exponent, unit * score + offset.  Without cap and
// slopes a score is the product itself; with a cap alone where cap_of's short
// form will do, cap tanh(y) = cap - 2 cap / (exp(2 y) + 1), it is -1 / (exp(2 y)
// + 1); else the exponent.
struct Scores {
    float in, cap, slope;   // slope: of the row; all in base-2 units
    float unit, offset;
    bool raw, negative;
    __device__ static Scores of(const Params &p, int kv, float slope)
    {
        Scores s;
        const float signed_ = p.scale * (p.k_scale ? p.k_scale[kv] : 1.0f), scale = fabsf(signed_);
        s.negative = signed_ < 0.0f;
        s.raw = p.cap == 0.0f && !p.slopes;
        s.cap = p.cap * kLog2e;
        s.in = p.short_cap ? scale / p.cap * (2.0f * kLog2e) : p.cap > 0.0f ? scale / p.cap : scale * kLog2e;
        s.slope = slope * kLog2e;
        s.unit = s.raw ? s.in : p.short_cap ? 2.0f * s.cap : 1.0f;
        s.offset = p.short_cap ? s.cap : 0.0f;
        return s;
    }
};

// OB: blocks of 32 elements of a head that are multiplied.
template <class T, class CT, int DP, int WR, bool WHOLE, int OB>
__global__ __launch_bounds__((Shape<T, CT, DP, WR, WHOLE>::BLOCK))
__attribute__((amdgpu_waves_per_eu((Shape<T, CT, DP, WR, WHOLE>::PER_SIMD), (Shape<T, CT, DP, WR, WHOLE>::PER_SIMD)))) void k_rows(Params p)
{
    using S = Shape<T, CT, DP, WR, WHOLE>;
    constexpr int WK = S::WK, U = S::U, KT = S::KT, M = S::M;
    constexpr int QV = S::F32 ? OB * 4 : OB * 2;
    using Q = typename std::conditional<S::F32, f32x4, vec<T, 8>>::type;
    __shared__ __attribute__((aligned(1024))) char s_buf[S::LDS];
    __shared__ float s_m[S::WAVES][32], s_l[S::WAVES][32];
    __shared__ int2 s_range[S::WAVES];
    __shared__ uint32_t s_odd;
    __shared__ uint32_t s_bad[2][KT / 32], s_note[2], s_waves[2][S::WAVES];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WK, wk = wave - wr * WK;
    const uint32_t buf = address(s_buf);

    // this workgroup's run
    int s, kv, b;         // sequence, cache head, block of the sequence
    int32_t c0 = 0;
    int64_t left = 1, run = 0;
    int32_t index = blockIdx.x;
    Seq found{};
    if (p.direct) {
        // one block of one head: found among the sequences
        int32_t block = index / p.n_heads;
        kv = index - block * p.n_heads;
        for (s = 0; s < p.n_seq; s += 64) {
            Seq mine{};
            if (s + lane < p.n_seq) mine = seq_of(p, s + lane);
            const int32_t n = blocks_of(p, mine), incl = prefix(n);
            const uint64_t behind = __builtin_amdgcn_ballot_w64(block < incl);
            if (behind) {
                const int at = __builtin_ctzll(behind);
                block -= __builtin_amdgcn_readlane(incl - n, at);
                found.start = __builtin_amdgcn_readlane(mine.start, at);
                found.n = __builtin_amdgcn_readlane(mine.n, at);
                found.len = __builtin_amdgcn_readlane(mine.len, at);
                found.keys = __builtin_amdgcn_readlane(mine.keys, at);
                found.bad = __builtin_amdgcn_readlane(mine.bad, at);
                s += at;
                break;
            }
            block -= __builtin_amdgcn_readlane(incl, 63);
        }
        if (s >= p.n_seq) return;
        s = uniform(s);
        b = uniform(block);
    } else {
        // neighbouring runs on one XCD
        index = (index & 7) * (gridDim.x / 8) + (index >> 3);
        const int64_t total = p.base[p.n_seq] * p.n_heads, even = (total + gridDim.x - 1) / gridDim.x;
        run = even > kMinTiles ? even : kMinTiles;
        const int64_t begin = index * run, end = min(begin + run, total);
        if (begin >= total) {
            if (tid == 0) p.cut[index] = make_int4(0, 0, 0, 0);
            return;
        }
        left = end - begin;
        s = find([&](int32_t i) { return p.base[i] * p.n_heads; }, p.n_seq, begin);
        const int32_t first = p.first[s], n = p.first[s + 1] - first;
        const int64_t base = p.base[s], each = p.base[s + 1] - base, at = begin - base * p.n_heads;
        kv = (int)((at | each) >> 31 ? at / each : (uint32_t)at / (uint32_t)each);
        const int64_t z = at - kv * each;
        b = find([&](int32_t i) { return p.cost[first + i] - base; }, n, z);
        c0 = (int32_t)(z - (p.cost[first + b] - base));
    }
    int4 cut = make_int4(0, 0, 0, 0);
    bool padded = false;

    for (; left > 0; ++b, c0 = 0) {
        int2 span;
        Seq x;
        int32_t t0 = 0, n = 0, tiles = 0;
        if (p.direct) {
            left = 0;
            x = found;
            const int32_t r0 = b * M, r1 = min(r0 + M, x.n * p.group);
            span = span_of(p, x, s, r0 / p.group, (r1 - 1) / p.group, lane, 64);
            if (p.first_key) {
                if (span.y == 0) span.x = INT32_MAX;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    span.x = min(span.x, __shfl_xor(span.x, o));
                    span.y = max(span.y, __shfl_xor(span.y, o));
                }
                if (span.y == 0) span.x = 0;
            }
            n = tiles = tiles_of<KT>(span);
        } else {
            while (b >= p.first[s + 1] - p.first[s]) {   // the next head, or sequence
                b = 0;
                if (p.first[s + 1] == p.first[s] || ++kv == p.n_heads) {
                    kv = 0;
                    ++s;
                }
            }
            x = seq_of(p, s);
            span = p.span[p.first[s] + b];
            tiles = tiles_of<KT>(span);
            const int32_t cost = tiles + extra(M), c1 = (int32_t)(cost - c0 < left ? cost : c0 + left);
            left -= c1 - c0;
            t0 = max(c0 - extra(M), 0);
            n = max(c1 - extra(M), 0) - t0;
            if (n == 0) continue;   // the next run begins the block
        }
        t0 = uniform(t0);
        n = uniform(n);
        span = make_int2(uniform(span.x), uniform(span.y));
        // With a bias by distance from the last tile on: it makes the scores near
        // a row's own place the largest, and where those come first, nothing is
        // scaled.  (fp32 documents 123 us, from the first on 158; 4,096 tokens 911
        // and 1,370.  Without a bias trees take 2 to 5% longer so.)
        const int32_t ahead = p.slopes ? -KT : KT;   // keys from a tile to the next
        const int32_t first_key = (span.x / KT + (p.slopes ? uniform(tiles) - 1 : 0)) * KT;   // of tile 0
        const auto tile_key = [&](int32_t tile) { return first_key + tile * ahead; };
        if (span.y == 0) n = 0;   // (no keys: the rows are written all the same)

        __syncthreads();   // (the block before has been written)
        if (tid == 0) s_note[0] = s_note[1] = s_odd = 0;
        if (tid < KT / 32) s_bad[0][tid] = s_bad[1][tid] = 0;
        // Where the lane reads keys, row r of 32 and their piece g, and values,
        // transposed: elements 4 (lane % 4) on of 16 of rows 4 g + lane / 4 % 4.
        // (Pieces further on are reached by exclusive or: the tile begins at a
        // multiple of a row.)
        const uint32_t k_at = buf + (wk * S::KW + r) * S::PITCH + S::key_piece(r, g) * 16;
        const uint32_t v_row = 4 * g + (lane >> 2 & 3);
        const uint32_t v_at = buf + S::TILE + (wk * S::KW + v_row) * S::PITCH +
                              S::value_piece(v_row, 2 * (lane >> 4 & 1) + (lane & 3) / 2) * 16 + (lane & 1) * 8;

        const CT *kb = static_cast<const CT *>(p.k) + kv * p.head_stride;
        const CT *vb = static_cast<const CT *>(p.v) + kv * p.head_stride;
        const int32_t *table = p.table + s * p.table_stride;
        const int32_t last = t0 + n;
        u32x4 kx[S::DMA ? 1 : S::NQ], vx[S::DMA ? 1 : S::NQ];
        uint32_t bad_keys = 0;   // bit q: the page of piece q's key
        int32_t pages[S::DMA ? 1 : S::NQ];
        auto look = [&](int32_t k0) {   // (a tile ahead of the loads)
#pragma unroll
            for (int j = 0; j < (S::DMA ? 0 : S::NQ); ++j) {
                const int32_t key = min(max(k0 + (j * S::BLOCK + tid) / S::IN, span.x), span.y - 1);
                pages[j] = table[divide(key, p.page_mul, p.page_shift)];
            }
        };
        auto load = [&](int32_t k0) {
#pragma unroll
            for (int j = 0; j < (S::DMA ? 0 : S::NQ); ++j) {
                const int piece = j * S::BLOCK + tid, c = piece % S::IN;
                const int32_t key = min(max(k0 + piece / S::IN, span.x), span.y - 1);
                const int32_t of = divide(key, p.page_mul, p.page_shift), page = pages[j];
                const bool ok = page >= 0 && page < p.n_pages, used = c * (16 / (int)sizeof(CT)) < p.d;
                bad_keys = (bad_keys & ~(1u << j)) | (uint32_t)!ok << j;
                kx[j] = vx[j] = u32x4{0, 0, 0, 0};
                if (ok && used) {
                    const int64_t at = page * p.page_stride + (key - of * p.page_size) * p.slot_stride + c * (16 / (int)sizeof(CT));
                    kx[j] = *reinterpret_cast<const u32x4 *>(kb + at);
                    vx[j] = *reinterpret_cast<const u32x4 *>(vb + at);
                }
            }
        };
        // Pieces of the tile to shared memory.  Of tiles that not all rows
        // attend to all of, values that are not finite become 0, for a weight
        // of 0 would make them NaN: what they make of the rows that do attend
        // to them is put right behind the block.
        auto store = [&](int turn, bool partial) {
            char *const s_k = s_buf, *const s_v = s_buf + S::TILE;
            bool odd = false;
#pragma unroll
            for (int j = 0; j < (S::DMA ? 0 : S::NQ); ++j) {
                const int piece = j * S::BLOCK + tid, key = piece / S::IN, c = piece % S::IN;
                if (bad_keys >> j & 1) {
                    atomicOr(&s_bad[turn][key / 32], 1u << key % 32);
                    atomicOr(&s_note[turn], 1u);
                }
                if constexpr (sizeof(CT) == 1) {
                    const auto kk = __builtin_bit_cast(vec<uint32_t, 4>, kx[j]), vv = __builtin_bit_cast(vec<uint32_t, 4>, vx[j]);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const vec<T, 8> a = widen8<T>(kk[2 * half], kk[2 * half + 1]);
                        u32x4 v = __builtin_bit_cast(u32x4, widen8<T>(vv[2 * half], vv[2 * half + 1]));
                        if (partial) odd |= clean<T>(v);
                        *reinterpret_cast<vec<T, 8> *>(s_k + key * S::PITCH + S::key_piece(key, 2 * c + half) * 16) = a;
                        *reinterpret_cast<u32x4 *>(s_v + key * S::PITCH + S::value_piece(key, 2 * c + half) * 16) = v;
                    }
                } else {
                    *reinterpret_cast<u32x4 *>(s_k + key * S::PITCH + S::key_piece(key, c) * 16) = kx[j];
                    if (partial) odd |= clean<T>(vx[j]);
                    *reinterpret_cast<u32x4 *>(s_v + key * S::PITCH + S::value_piece(key, c) * 16) = vx[j];
                }
            }
            if (odd) s_odd = 1;
        };
        // The wave's share of a tile straight to shared memory.  The pages of
        // the next one are asked for a tile ahead.
        int32_t page[S::GROUPS], slot[S::GROUPS];
        constexpr int32_t kWhole = ~(S::GROUP - 1);
        const char *k_base = nullptr, *v_base = nullptr;
        const int32_t *entries = nullptr;
        uint32_t slot_bytes = 0, n_pages = 0, page_mul = 0, page_shift = 0;
        int64_t page_bytes = 0;
        int32_t page_size = 0, least_key = 0, most_key = 0, last_key = 0;
        if constexpr (S::DMA) {
            k_base = kept(reinterpret_cast<const char *>(uniform(kb)));
            v_base = kept(reinterpret_cast<const char *>(uniform(vb)));
            entries = kept(uniform(table));
            slot_bytes = kept((uint32_t)p.slot_stride * (uint32_t)sizeof(CT));
            page_bytes = kept(p.page_stride * (int64_t)sizeof(CT));
            n_pages = kept((uint32_t)p.n_pages);
            page_mul = kept(p.page_mul);
            page_shift = kept(p.page_shift);
            page_size = kept(p.page_size);
            least_key = kept(span.x);
            last_key = kept(span.y - 1);
            most_key = last_key & kWhole;
        }
        const auto group_key = [&](int32_t k0, int j) {   // the first key of a group, or of the nearest attended ones
            return min(max(k0 + wave * S::SHARE + j * S::GROUP, least_key & kWhole), most_key);
        };
        auto fetch = [&](int32_t tile) {
#pragma unroll
            for (int j = 0; j < S::GROUPS; ++j) {
                const int32_t key = group_key(tile_key(min(tile, last - 1)), j);
                const int32_t of = divide(key, page_mul, page_shift);
                page[j] = entries[of];
                slot[j] = key - of * page_size;
            }
        };
        // a lane's row of a load and its piece of it, from the first row's keys
        const int row0 = lane / S::IN, piece = lane % S::IN, first_row = wave * S::SHARE;
        uint32_t k_off[S::LOADS], v_off[S::LOADS];
#pragma unroll
        for (int c = 0; c < S::LOADS; ++c) {
            k_off[c] = (c * S::RI + row0) * slot_bytes + S::key_piece(first_row + c * S::RI + row0, piece) * 16;
            v_off[c] = (c * S::RI + row0) * slot_bytes + S::value_piece(c * S::RI + row0, piece) * 16;
        }
        const int exact = p.d == DP;
        auto send = [&](int32_t k0, int turn) {
            uint32_t bad = 0;
#pragma unroll
            for (int j = 0; j < S::GROUPS; ++j) {
                const int32_t key = group_key(k0, j), low = max(least_key - key, 0), high = min(last_key - key, S::GROUP - 1);
                const uint32_t k_to = turn * 2 * S::TILE + (first_row + j * S::GROUP) * S::PITCH, v_to = k_to + S::TILE;
                const uint32_t of = (uint32_t)uniform(page[j]);
                if (of >= n_pages) {   // (below 0 too)
                    bad |= 1u << j;   // (0: rows that do not attend to them must not see what lies there)
                    for (int c = lane; c < S::GROUP * S::PITCH / 16; c += 64) {
                        *reinterpret_cast<u32x4 *>(s_buf + k_to + c * 16) = u32x4{0, 0, 0, 0};
                        *reinterpret_cast<u32x4 *>(s_buf + v_to + c * 16) = u32x4{0, 0, 0, 0};
                    }
                    continue;
                }
                const int64_t at = of * page_bytes + (int64_t)((uint64_t)(uint32_t)uniform(slot[j]) * slot_bytes);
                const char *const k_from = k_base + at, *const v_from = v_base + at;
                if (exact && low == 0 && high == S::GROUP - 1) {
#pragma unroll
                    for (int c = 0; c < S::LOADS; ++c) {
                        to_shared(k_from, k_off[c], buf + k_to + c * 1024);
                        to_shared(v_from, v_off[c], buf + v_to + c * 1024);
                    }
                } else {   // (a key outside the attended ones stands for the nearest of them)
                    const uint32_t mine = again(lane), d = argument<Params>().d;
#pragma unroll 1
                    for (int c = 0; c < S::LOADS; ++c) {
                        const int row = c * S::RI + mine / S::IN;
                        const uint32_t off = __umul24(min(max(row, low), high), slot_bytes);
                        const uint32_t kp = S::key_piece(first_row + row, mine % S::IN), vp = S::value_piece(row, mine % S::IN);
                        if (kp * (16 / (int)sizeof(CT)) < d) to_shared(k_from, off + kp * 16, buf + k_to + c * 1024);
                        if (vp * (16 / (int)sizeof(CT)) < d) to_shared(v_from, off + vp * 16, buf + v_to + c * 1024);
                    }
                }
            }
            if (lane == 0) s_waves[turn][wave] = bad;
        };

        if (S::DMA && p.d < DP && (WK > 1 || !padded)) {   // what the padded rows' ends are multiplied as
            padded = true;
            for (int c = tid; c < S::TILES / 16; c += S::BLOCK) reinterpret_cast<u32x4 *>(s_buf)[c] = u32x4{0, 0, 0, 0};
            __syncthreads();
        }
        if (n > 0) {
            if constexpr (S::DMA) {
                fetch(t0);
                send(tile_key(t0), t0 & 1);
                fetch(t0 + 1);
            } else {
                look(tile_key(t0));
                load(tile_key(t0));
                look(tile_key(min(t0 + 1, last - 1)));
            }
        }
        // the lane's row
        const int32_t total_rows = x.n * p.group, row = b * M + wr * 32 + r;
        const bool valid = row < total_rows;
        const int32_t my = min(row, total_rows - 1), i = divide(my, p.group_mul, p.group_shift), h = my - i * p.group;
        const int32_t t = x.start + i, head = kv * p.group + h;
        Q q[QV];
        {
            const T *from = static_cast<const T *>(p.q) + t * p.q_row + head * p.q_head;
#pragma unroll
            for (int k = 0; k < QV; ++k) {
                const int at = (2 * k + g) * (S::F32 ? 4 : 8);
                q[k] = at < p.d ? *reinterpret_cast<const Q *>(from + at) : Q(0);
            }
        }
        const Range in = range_of(p, x, s, i);
        const Scores sc = Scores::of(p, kv, p.slopes ? p.slopes[head] : 0.0f);
        const uint32_t *mask = p.tree ? p.mask + t * p.mask_stride : nullptr;
        // All rows attend to the keys of [largest lo, least hi), and none of the
        // wave's to keys outside [wave_lo, wave_hi).
        int32_t all_lo = across<true>(in.lo), all_hi = across<false>(in.hi);
        int32_t wave_lo = across<false>(in.lo < in.hi ? in.lo : INT32_MAX), wave_hi = across<true>(in.hi);
        if (lane == 0) s_range[wave] = make_int2(all_lo, all_hi);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < S::WAVES; ++w) {
            all_lo = max(all_lo, s_range[w].x);
            all_hi = min(all_hi, s_range[w].y);
        }
        all_lo = uniform(all_lo);
        all_hi = uniform(all_hi);
        wave_lo = uniform(p.tree ? min(wave_lo, x.len) : wave_lo);
        wave_hi = uniform(p.tree ? x.keys : wave_hi);
        if (sc.negative) {
#pragma unroll
            for (int k = 0; k < QV; ++k) q[k] = -q[k];
        }

        // Weights are held against m, a score that is at most kSlack base-2
        // units below the row's largest: what is summed is scaled only where
        // one above `limit` comes.
        float m = -HUGE_VALF, limit = -HUGE_VALF, l = x.bad ? __builtin_nanf("") : 0.0f;
        f32x16 o[OB];
#pragma unroll
        for (int e = 0; e < OB; ++e) o[e] = f32x16(0.0f);

        // (here, so that no tile waits for them: the wait would be for the next
        // tile's keys too)
#pragma unroll
        for (int k = 0; k < QV; ++k) asm volatile("" : "+v"(q[k]));
        f32x16 sx[U];
        uint32_t in32[U], note = 0;
        float top = -HUGE_VALF;
        bool fresh = true, partial = false;
        // Weights of the scores: exp2((x - m) unit + UP), with one instruction
        // where the products with `unit` are far from where their rounding
        // shows.
        const auto weigh = [&]() {
            float base = m == -HUGE_VALF ? 0.0f : m;
            if (__builtin_amdgcn_ballot_w64(fabsf(base * sc.unit) > 0x1p10f) != 0) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sx[u][e] -= base;
                base = 0.0f;
            }
            const float add = S::UP - base * sc.unit;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) sx[u][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sx[u][e], sc.unit, add));
            if (partial && sc.unit == 0.0f) {   // (0 times -inf is NaN)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t mine = again(in32[u] >> 4 * g);
#pragma unroll
                    for (int e = 0; e < 16; ++e) sx[u][e] = mine >> (8 * (e / 4) + e % 4) & 1 ? sx[u][e] : 0.0f;
                }
            }
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e % 4] += sx[u][e];
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        };

        // What scales the outputs or adds to them one by one stands outside the
        // inner loop, which leaves it to them: a tile is begun again behind it.
        for (int32_t step = t0 * S::H;;) {
#pragma unroll 1
            for (; step < last * S::H; ++step, fresh = true) {
                const int32_t tile = step / S::H, half = step - tile * S::H;
                const int turn = tile & 1;
                const uint32_t now = (S::DMA ? turn * 2 * S::TILE : 0) + half * (S::KS * S::PITCH);   // the step's place in s_buf
                const int32_t k0 = tile_key(tile) + half * S::KS;
                partial = !(k0 >= all_lo && k0 <= all_hi - S::KS);
                const bool skip = k0 + wk * S::KW >= wave_hi || k0 <= wave_lo - (wk + 1) * S::KW;
                bool spread = false;
                int64_t from[S::GROUPS];
                uint32_t without = 0;   // groups of the tile without a page
                if (fresh && half == 0) {
                    const bool any = !(k0 >= all_lo && k0 <= all_hi - KT);
                    if constexpr (S::DMA) {
                        arrived();
                        __syncthreads();   // the tile is there, the one before has been read
                        // The next tile's loads one by one between the products,
                        // which would wait for their way out otherwise; those of
                        // a tile at an end of the keys, or without a page, at once.
                        if (tile + 1 < last) {
                            spread = exact && !skip;
#pragma unroll
                            for (int j = 0; j < S::GROUPS; ++j) {
                                const int32_t key = k0 + ahead + wave * S::SHARE + j * S::GROUP;
                                const uint32_t of = (uint32_t)uniform(page[j]);
                                spread &= key >= least_key && key + S::GROUP - 1 <= last_key && of < n_pages;
                                from[j] = of * page_bytes + (int64_t)((uint64_t)(uint32_t)uniform(slot[j]) * slot_bytes);
                            }
                            if (!spread) {
                                send(k0 + ahead, turn ^ 1);
                                fetch(tile + 2);
                            }
                        }
#pragma unroll
                        for (int w = 0; w < S::WAVES; ++w) without |= s_waves[turn][w];
                        note = 0;
                        if (any) {   // (see store)
                            u32x4 *const v = reinterpret_cast<u32x4 *>(s_buf + now + S::TILE) + tid;
                            constexpr int kPieces = S::TILE / 16 / S::BLOCK;
#pragma unroll
                            for (int c0 = 0; c0 < kPieces; c0 += 4) {
                                u32x4 y[4];
#pragma unroll
                                for (int c = 0; c < 4 && c0 + c < kPieces; ++c) y[c] = v[(c0 + c) * S::BLOCK];
#pragma unroll
                                for (int c = 0; c < 4 && c0 + c < kPieces; ++c)   // (padding is 0)
                                    if (clean<T>(y[c])) {
                                        v[(c0 + c) * S::BLOCK] = y[c];
                                        s_odd = 1;
                                    }
                            }
                            __syncthreads();
                        }
                    } else {
                        __syncthreads();   // the tile before has been read
                        store(turn, any);
                        if (tid == 0) s_note[turn ^ 1] = 0;
                        if (tid < KT / 32) s_bad[turn ^ 1][tid] = 0;
                        __syncthreads();
                        if (tile + 1 < last) {
                            load(k0 + ahead);
                            look(tile_key(min(tile + 2, last - 1)));
                        }
                        note = uniform((int32_t)s_note[turn]);
                    }
                }
                if (skip) {
                    if (S::DMA && fresh && half == 0) note |= uniform((int32_t)without) != 0;
                    continue;
                }

                // scores of the wave's keys (rows) and rows (columns)
#pragma unroll
                for (int u = 0; u < U; ++u) sx[u] = f32x16(0.0f);
                const uint32_t k_now = again(k_at + now);
                {
                    // (a block of 32 keys does not change a row's piece)
                    const auto read = [&](int i) { return shared<Q>((k_now ^ 32 * (i / U)) + 32 * (i % U) * S::PITCH); };
                    const auto mul = [&](int i, const Q &x) {
                        if constexpr (S::F32) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) sx[i % U] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], q[i / U][e], sx[i % U], 0, 0, 0);
                        } else {
                            sx[i % U] = Mfma<T>::mul(x, q[i / U], sx[i % U]);
                        }
                    };
                    Q a[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] = read(i);
                    if (spread) {
                        constexpr int kAll = 2 * S::GROUPS * S::LOADS, kEach = (kAll * 4 + QV * U - 1) / (QV * U);
                        in_order<QV * U>(a, read, mul, [&](int i) {
#pragma unroll
                            for (int k = i / 4 * kEach; k < (i / 4 + 1) * kEach && k < kAll; ++k) {
                                const int c = k / 2 % S::LOADS, j = k / 2 / S::LOADS;
                                const uint32_t to = buf + (turn ^ 1) * 2 * S::TILE + (first_row + j * S::GROUP) * S::PITCH + c * 1024;
                                if (k % 2 == 0)
                                    to_shared(k_base + from[j], k_off[c], to);
                                else
                                    to_shared(v_base + from[j], v_off[c], to + S::TILE);
                            }
                        });
                        if (lane == 0) s_waves[turn ^ 1][wave] = 0;
                        fetch(tile + 2);
                    } else {
                        in_order<QV * U>(a, read, mul, [](int) {});
                    }
                }
                if (S::DMA && fresh && half == 0) note |= uniform((int32_t)without) != 0;
                // element i of a lane's: key 8 (i / 4) + 4 g + i % 4 of 32
                if (!sc.raw) {
                    const auto &a = argument<Params>();
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int32_t kw = k0 + wk * S::KW + 32 * u;
                        if (a.short_cap) {
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                sx[u][e] = -__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(sx[u][e] * sc.in) + 1.0f);
                            continue;
                        }
                        sx[u] *= sc.in;
                        if (a.cap > 0.0f) cap_of<S::F32>(sx[u], sc.cap);
                        if (a.slopes) {
                            if (a.tree && kw > x.len - 32) {
#pragma unroll 1
                                for (int e = 0; e < 16; ++e) {   // (keys of nodes are where their nodes are)
                                    int32_t at = kw + 8 * (e / 4) + 4 * g + e % 4;
                                    if (at >= x.len)
                                        at = (int32_t)min((int64_t)x.len + max(a.depth[x.start + min(at - x.len, x.n - 1)], 0), (int64_t)INT32_MAX);
                                    const float y = sc.slope * (float)abs(in.position - at);
#pragma unroll
                                    for (int k = 0; k < 16; ++k) sx[u][k] -= k == e ? y : 0.0f;
                                }
                            } else {
                                const int32_t at = (int32_t)again(in.position - kw - 4 * g);
#pragma unroll
                                for (int e = 0; e < 16; ++e) sx[u][e] -= sc.slope * (float)abs(at - (8 * (e / 4) + e % 4));
                            }
                        }
                    }
                }
                if (partial) {
                    const auto &a = argument<Params>();
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int32_t kw = k0 + wk * S::KW + 32 * u;
                        const int32_t lo = min(max(in.lo - kw, 0), 32), hi = min(max(in.hi - kw, 0), 32);
                        in32[u] = (uint32_t)((1ull << hi) - 1) & ~(uint32_t)((1ull << lo) - 1);
                        if (a.tree && kw > x.len - 32 && kw < x.keys) {
                            // bits of the nodes from the first of these keys on
                            const int32_t node = kw - x.len, w = max(node, 0) >> 5;
                            uint64_t bits = mask[w];
                            if (w + 1 < a.mask_words) bits |= (uint64_t)mask[w + 1] << 32;
                            uint32_t word = node < 0 ? (uint32_t)(bits << -node) : (uint32_t)(bits >> (node & 31));
                            const int32_t end = x.keys - kw;   // > 0
                            if (end < 32) word &= (1u << end) - 1;
                            in32[u] |= word;
                        }
                        const uint32_t mine = again(in32[u] >> 4 * g);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            sx[u][e] = mine >> (8 * (e / 4) + e % 4) & 1 ? sx[u][e] : -HUGE_VALF;
                    }
                }
                if (note & 1) {
#pragma unroll 1
                    for (int u = 0; u < U; ++u) {
                        uint32_t bad = 0;   // bits of the keys without a page
                        if constexpr (S::DMA) {
                            for (int j = 0; j < 32 / S::GROUP; ++j) {
                                const int at = (half * S::KS + wk * S::KW + 32 * u) / S::GROUP + j;   // group of the tile
                                if (s_waves[turn][at / S::GROUPS] >> at % S::GROUPS & 1)
                                    bad |= ((1u << S::GROUP) - 1) << j * S::GROUP;
                            }
                        } else {
                            bad = s_bad[turn][(half * S::KS + wk * S::KW + 32 * u) / 32];
                        }
                        if ((partial ? u ? in32[U - 1] : in32[0] : ~0u) & bad) {
                            l = __builtin_nanf("");
                            if (int32_t *status = argument<Params>().status; status && valid) atomicOr(&status[s], DSIM_ST_BAD_PAGE);
                        }
                    }
                }
                top = sx[0][0];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, sx[u][e]);
                {
                    const auto y = halves(top);
                    top = fmaxf(y[0], y[1]);
                }
                if (__builtin_amdgcn_ballot_w64(top > limit) != 0) {
                    // (once a tile: whatever the scores, every loop ends)
                    if (fresh && __builtin_amdgcn_ballot_w64(top > limit && m != -HUGE_VALF) != 0) break;
                    // rows that had none: nothing to scale
                    m = m == -HUGE_VALF ? top : m;
                    limit = m == -HUGE_VALF ? m : limit_of(m, S::SLACK, sc.unit);
                }
                // outputs (rows) of the rows (columns); the first values come
                // while the weights are computed
                if constexpr (S::F32) {
                    const uint32_t v_now = again(buf + now + S::TILE + (wk * S::KW + 4 * g) * S::PITCH + 4 * r);
                    const auto read = [&](int i) {
                        const int e = i / OB, d = i % OB;
                        return shared<float>(v_now + (8 * (e / 4) + e % 4) * S::PITCH + 128 * d);
                    };
                    float a[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] = read(i);
                    weigh();
                    in_order<16 * OB>(a, read, [&](int i, float x) {
                        o[i % OB] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, sx[0][i / OB], o[i % OB], 0, 0, 0);
                    }, [](int) {});
                } else {
                    const uint32_t v_now = again(v_at + now);
                    const auto read = [&](int i) { return values<T, S::PITCH>(v_now ^ 64 * (i % OB), i / OB); };
                    // A weight enters the product as two numbers of T, 16 bits (fp16
                    // 22).  (As one, rounded as the result is: 8,192 tokens of one
                    // prompt 606 us for 817, capped chunks 426 for 491, e4m3 trees
                    // 718 for 885, and outputs off by 2.2e-3 of their norm in bf16 for
                    // 1.65e-3, one rounding's.)
                    vec<T, 8> a[4], w[2 * U], w2[2 * U];
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] = read(i);
                    weigh();
#pragma unroll
                    for (int k = 0; k < 2 * U; ++k) {
                        vec<float, 8> y;
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = sx[k / 2][8 * (k % 2) + e];
                        w[k] = from_f32<T, 8>(y);
                        w2[k] = from_f32<T, 8>(y - to_f32<T, 8>(w[k]));
                    }
                    in_order<2 * U * OB>(a, read, [&](int i, const vec<T, 8> &x) {
                        o[i % OB] = Mfma<T>::mul(x, w[i / OB], o[i % OB]);
                        o[i % OB] = Mfma<T>::mul(x, w2[i / OB], o[i % OB]);
                    }, [](int) {});
                }
            }
            if (step >= last * S::H) break;

            {
                const float to = top > limit ? top : m, f = rescale(m, to, sc.unit);
                l *= f;
#pragma unroll
                for (int e = 0; e < OB; ++e) o[e] *= f;
                m = to;
                limit = m == -HUGE_VALF ? m : limit_of(m, S::SLACK, sc.unit);
            }
            fresh = false;
        }

        // the halves' sums, and the waves that share the rows
        const uint32_t mine = again(lane), r_ = mine & 31, g_ = mine >> 5;
        {
            const auto y = halves(l);
            l = y[0] + y[1];
        }
        if constexpr (WK > 1) {
            if (g_ == 0) s_m[wave][r_] = m;
            __syncthreads();   // (and the last tile has been read)
            float top = m;
#pragma unroll
            for (int w = 0; w < WK; ++w) top = fmaxf(top, s_m[wr * WK + w][r_]);
            const float f = rescale(m, top, sc.unit);
            l *= f;
            m = top;
            if (g_ == 0) s_l[wave][r_] = l;
            f32x4 *const sums = reinterpret_cast<f32x4 *>(s_buf) + wr * (WK - 1) * (256 * OB) + mine;
#pragma unroll
            for (int e = 0; e < OB; ++e) {
                o[e] *= f;
                if (wk > 0)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sums[(wk - 1) * (256 * OB) + (4 * e + k) * 64] = f32x4{o[e][4 * k], o[e][4 * k + 1], o[e][4 * k + 2], o[e][4 * k + 3]};
            }
            __syncthreads();
            if (wk == 0) {
#pragma unroll
                for (int w = 1; w < WK; ++w) {
                    l += s_l[wr * WK + w][r_];
#pragma unroll
                    for (int e = 0; e < OB; ++e)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const f32x4 y = sums[(w - 1) * (256 * OB) + (4 * e + k) * 64];
#pragma unroll
                            for (int c = 0; c < 4; ++c) o[e][4 * k + c] += y[c];
                        }
                }
            }
        }
        const bool whole = p.direct || tiles == n || span.y == 0;
        if (wk == 0 && valid) {
            const float vs = (p.v_scale ? p.v_scale[kv] : 1.0f) * (whole ? share_of(l) : 1.0f);
            const Part part = Part::of(p, 2 * index + (t0 == 0 ? 1 : 0));
            const int at = wr * 32 + r_;
#pragma unroll
            for (int e = 0; e < OB; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int d = 32 * e + 8 * k + 4 * g_;
                    if (d >= p.d) continue;
                    const f32x4 y = f32x4{o[e][4 * k], o[e][4 * k + 1], o[e][4 * k + 2], o[e][4 * k + 3]} * vs;
                    if (whole)
                        write_row<T>(p, t, head, d, y);
                    else
                        *reinterpret_cast<f32x4 *>(part.o + at * p.d + d) = y;
                }
            if (g_ == 0) {
                if (whole) {
                    write_lse(p, t, head, m, sc.unit, sc.offset, l, S::UP);
                } else {
                    part.m[at] = m;
                    part.l[at] = l;
                }
            }
        }
        if (n > 0) {
            __syncthreads();   // (and every tile has been looked at)
            if (s_odd) {
                // The values that were taken as 0, added to the rows that attend
                // to them: infinities and NaN, a thread a column.
                __threadfence();
                const Part part = Part::of(p, 2 * index + (t0 == 0 ? 1 : 0));
                const int32_t a = tile_key(t0), z = tile_key(last - 1);
                const int32_t end = span.y - max(a, z) < KT ? span.y : max(a, z) + KT;
                for (int32_t key = max(min(a, z), span.x); key < end; ++key) {
                    const int32_t k0 = key / KT * KT;
                    if (k0 >= all_lo && k0 <= all_hi - KT) continue;   // (was not cleaned)
                    const int32_t of = divide(key, p.page_mul, p.page_shift), page = table[of];
                    if (page < 0 || page >= p.n_pages || tid >= p.d) continue;
                    const float v = value_of(vb[page * p.page_stride + (key - of * p.page_size) * p.slot_stride + tid]);
                    if (fabsf(v) < HUGE_VALF) continue;
                    const float y = v * (p.v_scale ? p.v_scale[kv] : 1.0f);
                    for (int at = 0; at < M && b * M + at < total_rows; ++at) {
                        const int32_t i = (b * M + at) / p.group, h = b * M + at - i * p.group;
                        if (!attends(p, x, s, i, key)) continue;
                        if (whole) {
                            T *const to = static_cast<T *>(p.out) + (x.start + i) * p.out_row + (kv * p.group + h) * p.out_head + tid;
                            *to = (T)((float)*to + y);
                        } else {
                            part.o[at * p.d + tid] += y;
                        }
                    }
                }
            }
        }
        if (t0 == 0 && !p.direct)   // parts: this one and the runs' behind
            cut = make_int4(whole ? 0 : 1 + (int)((tiles - n + run - 1) / run), s, kv, b);
    }
    if (tid == 0 && !p.direct) p.cut[index] = cut;
}

// Joins the parts of a block that a run's end cut, kJoinRows rows a
// workgroup: the rows' maxima and sums first, then four outputs a thread.
constexpr int kJoinRows = 32;
template <class T> __global__ __launch_bounds__(kJoin) void k_join(Params p, float up)
{
    constexpr int kWays = kJoin / kJoinRows;
    __shared__ float s_m[kWays][kJoinRows], s_l[kWays][kJoinRows];
    const int index = blockIdx.x, tid = threadIdx.x;
    const int4 cut = p.cut[index];
    const int n = cut.x, s = cut.y, kv = cut.z, first = blockIdx.y * kJoinRows;
    if (n == 0) return;
    const int32_t start = p.start[s], total_rows = (p.start[s + 1] - start) * p.group;
    const Scores sc = Scores::of(p, kv, 0.0f);
    auto part = [&](int j) { return Part::of(p, j == 0 ? 2 * index + 1 : 2 * (index + j)); };
    {
        const int at = tid % kJoinRows, way = tid / kJoinRows;
        float m = -HUGE_VALF, l = 0.0f;
        for (int j = way; j < n; j += kWays) m = fmaxf(m, part(j).m[first + at]);
        s_m[way][at] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWays; ++w) m = fmaxf(m, s_m[w][at]);
        for (int j = way; j < n; j += kWays) l += part(j).l[first + at] * rescale(part(j).m[first + at], m, sc.unit);
        s_l[way][at] = l;
        __syncthreads();
        if (way == 0) {
            s_m[0][at] = m;
#pragma unroll
            for (int w = 1; w < kWays; ++w) l += s_l[w][at];
            s_l[0][at] = l;
            const int32_t row = cut.w * p.rows + first + at, i = divide(row, p.group_mul, p.group_shift);
            if (row < total_rows) write_lse(p, start + i, kv * p.group + row - i * p.group, m, sc.unit, sc.offset, l, up);
        }
        __syncthreads();
    }
    const int quads = p.d / 4;
    for (int e = tid; e < kJoinRows * quads; e += kJoin) {
        const int at = e / quads, d = 4 * (e - at * quads);
        const int32_t row = cut.w * p.rows + first + at, i = divide(row, p.group_mul, p.group_shift);
        if (row >= total_rows) break;
        const float m = s_m[0][at];
        f32x4 o = {0, 0, 0, 0};
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
            const Part y = part(j);
            o += *reinterpret_cast<const f32x4 *>(y.o + (int64_t)(first + at) * p.d + d) * rescale(y.m[first + at], m, sc.unit);
        }
        write_row<T>(p, start + i, kv * p.group + row - i * p.group, d, o * share_of(s_l[0][at]));
    }
}

template <class T, class CT, int DP, int WR, bool WHOLE, int OB> dsim_status launch(Params &p, hipStream_t s)
{
    using S = Shape<T, CT, DP, WR, WHOLE>;
    const auto check = [](const char *what) {
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? DSIM_OK : hip_fail(e, what);
    };
    dsim_status st = DSIM_OK;
    if (!p.direct || p.status) {
        hipLaunchKernelGGL((k_plan<S::KT>), dim3(1), dim3(kPlan), 0, s, p);
        if ((st = check("attention plan launch"))) return st;
    }
    const int grid = p.direct ? (int)(p.max_blocks * p.n_heads) : kCus * S::PER_CU;
    hipLaunchKernelGGL((k_rows<T, CT, DP, WR, WHOLE, OB>), dim3(grid), dim3(S::BLOCK), 0, s, p);
    if ((st = check("attention launch")) || p.direct) return st;
    hipLaunchKernelGGL((k_join<T>), dim3(grid, S::M / kJoinRows), dim3(kJoin), 0, s, p, S::UP);
    return check("attention join launch");
}

template <class T, class CT, int DP, int WR> dsim_status launch(Params &p, hipStream_t s)
{
    // 16 slots of a page at offsets of 24-bit products
    const bool whole = p.page_size % 16 == 0 && p.slot_stride * (int64_t)sizeof(CT) < 1 << 24;
    if (!whole) return launch<T, CT, DP, WR, false, DP / 32>(p, s);
    if constexpr (DP > 64)
        if (p.d <= DP * 3 / 4) return launch<T, CT, DP, WR, true, DP / 32 * 3 / 4>(p, s);
    return launch<T, CT, DP, WR, true, DP / 32>(p, s);
}

template <class T, class CT, int DP> dsim_status launch(Params &p, hipStream_t s)
{
    if constexpr (DP <= 128)
        if (p.rows == 32) return launch<T, CT, DP, 1>(p, s);
    if (p.rows == 64) return launch<T, CT, DP, 2>(p, s);
    if constexpr (DP <= 128 && sizeof(T) == 2)
        if (p.rows == 256) return launch<T, CT, DP, 8>(p, s);
    return launch<T, CT, DP, 4>(p, s);
}

template <class T, class CT> dsim_status launch(Params &p, hipStream_t s)
{
    return p.d <= 64 ? launch<T, CT, 64>(p, s) : p.d <= 128 ? launch<T, CT, 128>(p, s) : launch<T, CT, 256>(p, s);
}

// by the queries' type, in a translation unit each
dsim_status launch_f32(Params &p, hipStream_t s);
dsim_status launch_f16(Params &p, bool e4m3_cache, hipStream_t s);
dsim_status launch_bf16(Params &p, bool e4m3_cache, hipStream_t s);

}  // namespace rows
}  // namespace dsim
