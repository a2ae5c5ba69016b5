// paged_attention.h -- the kernels of dsim_paged_attention: attention of one
// new token per sequence over its paged keys and values.
//
// Every key and value is read once, 4 flops a pair of elements and query head,
// so memory bounds all but the short calls (a group of 16 heads: 16 flops a
// byte in bf16; the card's balance is over 150), and what has to be kept up is
// loads in flight: 16 bytes a lane, a tile's keys requested again as soon as
// their scores are known, its values as soon as the outputs are.  One pass:
// the maximum and the sum run along in fp32, and weights keep fp32's bits.
// Matrix instructions make the products cheap; addresses, exponentials, the
// weights' parts and the widening of e4m3 take a fifth of the vector issue
// slots with bf16, 43% with e4m3.  A sequence's keys take part in the products
// straight from the loads, with nothing in shared memory.
// On MI355X (us a call, both launches, calls one after another on several
// copies of the tensors): bf16, 32 query and 8 cache heads of 128, 64 sequences
// of up to 4,096 tokens (538 MB) 98.7, 5.45 TB/s; 64 query heads, 4 of 131,072
// (2.1 GB) 330, 6.5 TB/s; e4m3, 128 of up to 8,192 (1.14 GB) 196, 5.8 TB/s;
// fp32, 16 sequences, 12 heads of 80, window 1,000 (100 MB) 27.9, 3.6 TB/s;
// fp16, one of 97 tokens, 12 heads of 64, 6.1.  Reads alone, in pieces of 4 to
// 64 KB, reach 6.0 to 6.5 TB/s.  Figures beside the rules below are of calls
// captured into a graph, on two copies in turn: up to 5% above or below.
#pragma once

#include "numeric.h"
#include "ops.h"

namespace dsim {
namespace attend {

constexpr int kWaves = 4;
constexpr int kBlock = 64 * kWaves;
constexpr int kCus = 256;
// Workgroups per CU by the padded head dimension and the size of the cache's
// elements, all resident at once.  Where the state of one fills the registers
// (heads of 256, two a CU spill: 71 us for 49) one; more than two do not pay
// (heads of 128, three: 10% more time; of 64, four: the same; e4m3, 256
// sequences of 2,000 tokens, three: 202 us for 204, four, which spill, 417).
constexpr int per_cu(int dp, int size) { return dp <= 128 || size == 1 ? 2 : 1; }
constexpr int kMaxGrid = kCus * 2;
// Of a run, a tile for every wave: what it begins of a context costs little
// where workgroups are left over (one sequence of 2,048 tokens, 8 cache heads
// of 128: 13.3 us, with runs of at least kExtra more 15.6).
constexpr int kMinTiles = 4;
// What a context costs beside its tiles, in tiles.  bf16, 64 sequences of up to
// 2,000 tokens with 8 cache heads of 128: 59.6 us (5: 58.7, 12: 62.6, 24:
// 67.3); e4m3 36.2 (40.6, 36.8, 39.5); fp32, 256 of 1,900 642 (640, 625, 631).
constexpr int kExtra = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// How the elements of a (query, cache) type pair go through the matrix
// instructions.  One tile is kKeys keys of one cache head and 16 query heads
// (those of the group, the rest zero):
//   scores   S[key][head] = K[key][:] . q[head][:]      rows = keys
//   output   O[d][head]  += V[key][d] P[key][head]      rows = d
// A lane l = 16 g + r of a 16 x 16 product holds row r of the left operand
// and column r of the right one for the reduction indices of its group g,
// and of the result column r, rows 4 g + i.  The result of the scores is
// therefore, lane for lane, the right operand of the output product, and the
// order of the reduction index is free as long as both operands agree:
//   keys: the lane's own rows 4 g + i of each 16-key product;
//   head dimension: chunk c = 4 step + g.
// Row r of output product e stands for d = E r + e, so a lane loads E
// consecutive elements of each of its keys' values and transposes inside its
// own registers; nothing crosses lanes and shared memory is not used.
template <class T> struct Mfma;
template <> struct Mfma<f16> {
    __device__ static f32x4 mul(vec<f16, 8> a, vec<f16, 8> b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mfma<bf16> {
    __device__ static f32x4 mul(vec<bf16, 8> a, vec<bf16, 8> b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};

struct Params {
    const void *k, *v, *q;
    void *out;
    const float *k_scale, *v_scale;
    const int32_t *table, *seq_len;
    float *lse;
    int32_t *status;
    float *part;          // partial results, 2 per workgroup
    int4 *cut;            // contexts that are cut: by context, or by the workgroup that begins it
    int64_t n_pages, page_stride, slot_stride, head_stride, table_stride, q_row, q_head, out_row, out_head;
    float scale;          // times log2 e
    int32_t n_seq, n_heads, n_q_heads, d, page_size, table_width, window;
    int32_t group, tiles_of_heads, part_heads;
    int32_t grid;         // runs that the work is cut into
    bool by_context;      // there are at most as many contexts
    bool direct;          // a workgroup per context, nothing is cut
    uint32_t div_mul, div_shift;   // t / page_size = t * div_mul >> div_shift, 0 <= t < 2^31
};

// Page and slot of a position.
struct Place {
    int32_t page, slot;   // of the sequence, of the page
    __device__ static Place of(const Params &p, int32_t t)
    {
        const int32_t q = (int32_t)((uint64_t)(uint32_t)t * p.div_mul >> p.div_shift);
        return {q, t - q * p.page_size};
    }
};

// The keys of a sequence in tiles: first tile, number of tiles (at least
// one, so that somebody writes the row; none if the row is left alone).
template <int KEYS> struct Span {
    int32_t first_key, len, first_tile, n;
    bool bad;
    __device__ int32_t cost() const { return n > 0 ? n + kExtra : 0; }
    __device__ static Span of(const Params &p, int32_t len)
    {
        Span s{0, len, 0, 0, false};
        if (len < 0) return s;
        s.bad = (int64_t)len > (int64_t)p.table_width * p.page_size;
        if (s.bad) s.len = 0;
        s.first_key = p.window > 0 && s.len > p.window ? s.len - p.window : 0;
        s.first_tile = s.first_key / KEYS;
        const int32_t end = (int32_t)(((int64_t)s.len + KEYS - 1) / KEYS);
        s.n = end > s.first_tile ? end - s.first_tile : 1;
        return s;
    }
};

// a value that is the same for all lanes, in scalar registers
__device__ inline int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// The values of the other groups' lanes r: halves and odd and even rows of a
// wave exchanged.
__device__ inline vec<float, 2> other_half(float x)
{
    const auto y = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return {__builtin_bit_cast(float, (uint32_t)y[0]), __builtin_bit_cast(float, (uint32_t)y[1])};
}

__device__ inline vec<float, 2> other_row(float x)
{
    const auto y = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return {__builtin_bit_cast(float, (uint32_t)y[0]), __builtin_bit_cast(float, (uint32_t)y[1])};
}

// Within each row of 16 lanes: the value N lanes on, and lane N's.
template <int N> __device__ inline float turn(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x120 + N, 0xf, 0xf, true));
}

template <int N> __device__ inline float spread(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x150 + N, 0xf, 0xf, true));
}

__device__ inline float max_groups(float x)
{
    const auto y = other_half(x);
    const auto z = other_row(fmaxf(y[0], y[1]));
    return fmaxf(z[0], z[1]);
}

__device__ inline float sum_groups(float x)
{
    const auto y = other_half(x);
    const auto z = other_row(y[0] + y[1]);
    return z[0] + z[1];
}

// What sums held against the maximum `from` count against the maximum `to`,
// both products of query and key, `scale` base-2 logarithms per unit.  Where
// there was none (-inf) they are held against 0: zero, or NaN, which has to
// stay.  (Differences are scaled, not maxima subtracted from scaled products:
// a scaled maximum above 2^31 is rounded by more than an exponent can be.)
__device__ inline float rescale(float from, float to, float scale)
{
    return from == -HUGE_VALF ? 1.0f : __builtin_amdgcn_exp2f((from - to) * scale);
}

// Running state of one wave: for column r (a query head) the largest product
// m, this lane's share of the sum l, and the output's rows.
template <int NT> struct Columns {
    float m, l;
    f32x4 o[NT];
    __device__ void clear()
    {
        m = -HUGE_VALF;
        l = 0.0f;
#pragma unroll
        for (int e = 0; e < NT; ++e) o[e] = f32x4{0, 0, 0, 0};
    }
    __device__ float sum() const { return sum_groups(l); }
};

// The running maximum takes in the products s; returns them as weights, 1 for
// one at the maximum.  scale >= 0: base-2 logarithms per unit of s.  `in`:
// bit i says whether s[i] counts (looked at unless `all`); one that does not
// becomes the weight 0.
template <int N, int NT>
__device__ inline void weigh(float (&s)[N], float scale, bool all, uint32_t in, Columns<NT> &st)
{
    if (!all) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = in >> i & 1 ? s[i] : -HUGE_VALF;
    }
    float top = s[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, s[i]);
    top = max_groups(top);
    if (__builtin_amdgcn_ballot_w64(top > st.m) != 0) {
        const float m = fmaxf(st.m, top);
        const float f = rescale(st.m, m, scale);
        st.l *= f;
#pragma unroll
        for (int e = 0; e < NT; ++e) st.o[e] *= f;
        st.m = m;
    }
    const float m = st.m == -HUGE_VALF ? 0.0f : st.m;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = __builtin_amdgcn_exp2f((s[i] - m) * scale);
    if (!all) {   // (a scale of 0 times -inf is NaN)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = in >> i & 1 ? s[i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) st.l += s[i];
}

// Keys and values; STREAM: they are read once and leave the caches soon.
template <bool STREAM, class V> __device__ inline V read(const void *p)
{
    return STREAM ? __builtin_nontemporal_load(static_cast<const V *>(p)) : *static_cast<const V *>(p);
}

// Whether rows of d elements, more than DP / 2 of them (but for the smallest
// DP) and padded to DP, reach beyond element `at`: the same for all lanes.
// What none of them needs is neither loaded nor multiplied (fp32, 64
// sequences, 12 cache heads of 176, 48 query heads, window 450: 116 us; with
// all of the padding 118; 12 of 80, window 1,000: 105 and 112).
template <int DP, bool EXACT> __device__ inline bool needed(const Params &p, int at)
{
    return EXACT || at <= (DP > 64 ? DP / 2 : 0) || at < p.d;
}

// What the passes by columns share.  DIM: see dim() of each.
template <class P, int DP, int KEYS> struct ByColumns {
    static constexpr int kMine = KEYS / 4;   // keys that a lane has the scores of
    using State = Columns<DP / 16>;

    // the lane's key i in the tile
    __device__ static int key(int i, int r, int g) { return i / 4 * 16 + 4 * g + i % 4; }

    __device__ static void weigh(float (&s)[kMine], float scale, bool all, uint32_t in, State &st)
    {
        attend::weigh(s, scale, all, in, st);
    }

    // the outputs times f to shared memory, a row per head
    template <int PAD> __device__ static void store(const State &st, float f, float (*o)[PAD], int heads, int r, int g)
    {
        if (r >= heads) return;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < DP / 16; e += 4)
                *reinterpret_cast<f32x4 *>(&o[r][P::dim(g, i, e)]) =
                    f32x4{st.o[e][i], st.o[e + 1][i], st.o[e + 2][i], st.o[e + 3][i]} * f;
    }
};

// 16-bit queries; keys and values of the same type or e4m3.
template <class T, class CT, int DP, bool EXACT, bool STREAM>
struct Pass : ByColumns<Pass<T, CT, DP, EXACT, STREAM>, DP, 32> {
    static constexpr int kKeys = 32, kE = DP / 16;
    static constexpr bool k8 = __is_same(CT, e4m3);
    static constexpr int kChunk = 16 / sizeof(CT);            // elements per 16-byte load of a key
    static constexpr int kSteps = DP / (4 * kChunk);          // loads of a key per lane
    static constexpr int kParts = kChunk / 8;                 // products per load
    using Query = vec<T, 8>[kSteps * kParts];

    using Keys = u32x4[2][kSteps];
    using Values = vec<CT, kE>[8];

    // negated for a negative scale
    __device__ static void load_query(const Params &p, const T *q, bool used, int g, Query &out)
    {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int h = 0; h < kParts; ++h) {
                const int at = (4 * s + g) * kChunk + 8 * h;
                vec<T, 8> x = used && at < p.d ? *reinterpret_cast<const vec<T, 8> *>(q + at) : vec<T, 8>(0);
                out[s * kParts + h] = p.scale < 0.0f ? -x : x;
            }
    }

    // rows: where the tile's keys lie
    template <class Rows> __device__ static void load_keys(const Params &p, const Rows &rows, int r, int g, Keys &x)
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const CT *row = rows.key(t, r);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int at = (4 * s + g) * kChunk;
                if (needed<DP, EXACT>(p, 4 * s * kChunk)) x[t][s] = read<STREAM, u32x4>(row + (EXACT || at < p.d ? at : 0));
            }
        }
    }

    template <class Rows> __device__ static void load_values(const Params &p, const Rows &rows, int r, int g, Values &x)
    {
        const int at = EXACT || kE * r < p.d ? kE * r : 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[4 * t + i] = read<STREAM, vec<CT, kE>>(rows.value(t, 4 * g + i) + at);
    }

    __device__ static vec<T, 8> part(u32x4 x, int h, bool in)
    {
        vec<T, 8> y;
        if constexpr (k8) {
            const uint32_t lo = h ? x[2] : x[0], hi = h ? x[3] : x[1];
            y = widen8(lo, hi);
        } else {
            y = __builtin_bit_cast(vec<T, 8>, x);
        }
        return in ? y : vec<T, 8>(0);
    }

    // two of the four e4m3 of a word, exactly
    template <class U, bool HIGH> __device__ static vec<U, 2> widen2(uint32_t w)
    {
        if constexpr (__is_same(U, f16))
            return __builtin_bit_cast(vec<U, 2>, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH));
        else
            return __builtin_bit_cast(vec<U, 2>, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
    }

    __device__ static vec<T, 8> widen8(uint32_t lo, uint32_t hi)
    {
        const vec<T, 2> a = widen2<T, false>(lo), b = widen2<T, true>(lo), c = widen2<T, false>(hi), d = widen2<T, true>(hi);
        return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }

    // Weights as the sums of three bf16 numbers of 8 bits, which hold fp32's 24
    // exactly and its range.  (Two, 16 bits, put the outputs five times as far
    // from the formula's as fp32 sums do.)  For values that may be infinite no
    // part is 0 unless the weight is, so that the three products' sum is that
    // infinity: fp32's smallest normal number stands in, below which weights
    // are 0 themselves.
    __device__ static void split(const float (&s)[8], vec<bf16, 8> (&w)[3])
    {
        uint32_t part[3][8];
        const auto rest = [](uint32_t x) {
            return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, x) - __builtin_bit_cast(float, x & 0xffff0000u));
        };
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            part[0][i] = __builtin_bit_cast(uint32_t, s[i]);
            part[1][i] = rest(part[0][i]);
            part[2][i] = rest(part[1][i]);
            if constexpr (!k8) {
                const uint32_t least = min(part[0][i], 0x00800000u);   // (as whole numbers: none is negative)
                part[1][i] = max(part[1][i], least);
                part[2][i] = max(part[2][i], least);
            }
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            vec<uint32_t, 4> x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_perm(part[k][2 * i + 1], part[k][2 * i], 0x07060302);
            w[k] = __builtin_bit_cast(vec<bf16, 8>, x);
        }
    }

    // The values of keys that do not count become 0: what stands in their
    // place, the nearest attended key's, may be infinite, and times the weight
    // 0 NaN.
    __device__ static void drop(Values &x, uint32_t in, int g)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(in >> i & 1)) x[i] = vec<CT, kE>(0);
    }

    // products of the lane's keys 16 t + 4 g + i with query head r
    __device__ static void scores(const Params &p, const Keys &x, const Query &q, int g, float (&s)[8])
    {
        // (products that need one another's result stand apart)
        f32x4 acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int h = 0; h < kParts; ++h)
#pragma unroll
                for (int t = 0; t < 2 && needed<DP, EXACT>(p, 4 * i * kChunk); ++t)
                    acc[t] = Mfma<T>::mul(part(x[t][i], h, EXACT || (4 * i + g) * kChunk < p.d), q[i * kParts + h], acc[t]);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * t + i] = acc[t][i];
    }

    // The values of those keys, times their weights.  bf16 and e4m3 values are
    // bf16 numbers, their products' operands as they are (64 sequences of up
    // to 4,096, bf16, 32 and 8 heads of 128: 98.8 us; with fp32 operands 102;
    // 128 of up to 8,192 in e4m3 202 and 273).  fp16 values are not, and fp16
    // weights would end at 2^-39 of the largest: both as fp32 (64 sequences of
    // up to 4,096 106 us; the values in two bf16 parts and five products 105,
    // but 256 of up to 300 with 12 heads of 64 40 us for 37).
    __device__ static void outputs(const Values &x, const float (&s)[8], Columns<DP / 16> &st)
    {
        if constexpr (__is_same(CT, f16)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const vec<float, kE> row = to_f32<f16, kE>(x[i]);
#pragma unroll
                for (int e = 0; e < kE; ++e) st.o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(row[e], s[i], st.o[e], 0, 0, 0);
            }
        } else {
            vec<bf16, 8> w[3];
            split(s, w);
            vec<bf16, kE> row[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) row[i] = to_bf16(x[i]);
            constexpr int kTogether = 4;
#pragma unroll
            for (int e0 = 0; e0 < kE; e0 += kTogether) {
                vec<bf16, 8> a[kTogether];
#pragma unroll
                for (int e = 0; e < kTogether; ++e)
#pragma unroll
                    for (int i = 0; i < 8; ++i) a[e][i] = row[i][e0 + e];
#pragma unroll
                for (int k = 0; k < 3; ++k)
#pragma unroll
                    for (int e = 0; e < kTogether; ++e) st.o[e0 + e] = Mfma<bf16>::mul(a[e], w[k], st.o[e0 + e]);
            }
        }
    }

    __device__ static vec<bf16, kE> to_bf16(vec<CT, kE> x)
    {
        if constexpr (k8) {
            const auto w = __builtin_bit_cast(vec<uint32_t, kE / 4>, x);
            vec<bf16, kE> y;
#pragma unroll
            for (int i = 0; i < kE / 4; ++i) {
                const vec<bf16, 2> a = widen2<bf16, false>(w[i]), b = widen2<bf16, true>(w[i]);
                y[4 * i] = a[0];
                y[4 * i + 1] = a[1];
                y[4 * i + 2] = b[0];
                y[4 * i + 3] = b[1];
            }
            return y;
        } else {
            return x;
        }
    }

    // the element of d that row 4 g + i of output product e stands for
    __device__ static int dim(int g, int i, int e) { return (4 * g + i) * kE + e; }
};

// fp32: the same with products of four reduction indices, 16 keys a tile.
template <int DP, bool EXACT, bool STREAM>
struct Pass<float, float, DP, EXACT, STREAM> : ByColumns<Pass<float, float, DP, EXACT, STREAM>, DP, 16> {
    static constexpr int kKeys = 16, kSteps = DP / 16, kQuads = DP / 64;
    using Query = f32x4[kSteps];

    using Keys = f32x4[kSteps];
    using Values = f32x4[4][kQuads];

    __device__ static void load_query(const Params &p, const float *q, bool used, int g, Query &out)
    {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = (4 * s + g) * 4;
            const f32x4 x = used && at < p.d ? *reinterpret_cast<const f32x4 *>(q + at) : f32x4{0, 0, 0, 0};
            out[s] = p.scale < 0.0f ? -x : x;
        }
    }

    template <class Rows> __device__ static void load_keys(const Params &p, const Rows &rows, int r, int g, Keys &x)
    {
        const float *row = rows.key(0, r);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = (4 * s + g) * 4;
            if (needed<DP, EXACT>(p, 16 * s)) x[s] = read<STREAM, f32x4>(row + at);
        }
    }

    template <class Rows> __device__ static void load_values(const Params &p, const Rows &rows, int r, int g, Values &x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float *val = rows.value(0, 4 * g + i);
#pragma unroll
            for (int j = 0; j < kQuads; ++j) {
                const int at = 64 * j + 4 * r;
                x[i][j] = read<STREAM, f32x4>(val + (EXACT || at < p.d ? at : 0));
            }
        }
    }

    __device__ static void drop(Values &x, uint32_t in, int g)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kQuads; ++j)
                if (!(in >> i & 1)) x[i][j] = f32x4{0, 0, 0, 0};
    }

    __device__ static void scores(const Params &p, const Keys &x, const Query &q, int g, float (&s)[4])
    {
        // four sums, so that no product waits for the one before
        f32x4 acc[4] = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (!needed<DP, EXACT>(p, 16 * i)) break;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i][e], q[i][e], acc[e], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = (acc[0][i] + acc[1][i]) + (acc[2][i] + acc[3][i]);
    }

    __device__ static void outputs(const Values &x, const float (&s)[4], Columns<DP / 16> &st)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kQuads; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    st.o[4 * j + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i][j][e], s[i], st.o[4 * j + e], 0, 0, 0);
    }

    __device__ static int dim(int g, int i, int e) { return 64 * (e / 4) + (4 * g + i) * 4 + e % 4; }
};

// fp32, a cache head with one query head: fifteen of the matrix instructions'
// sixteen columns would be empty, and in fp32 they are slow enough to show
// (16 sequences of 12 heads of 80, window 1,000: 30.8 us, this way 26.9; 256
// of up to 64 tokens 42.5 and 35.2; 64 of up to 4,096 193 and 188), so the products
// are ordinary ones.  Keys and values lie as above; a lane sums its
// chunks of key r's product, the groups' sums are added, and the weights of
// its own keys 4 g + i come from its row's lanes.
template <int DP, bool EXACT, bool STREAM> struct OnePass : Pass<float, float, DP, EXACT, STREAM> {
    using Base = Pass<float, float, DP, EXACT, STREAM>;
    using Base::kQuads;
    using Base::kSteps;
    static constexpr int kMine = 1;

    struct State {
        float m, l;
        f32x4 o[kQuads];
        __device__ void clear()
        {
            m = -HUGE_VALF;
            l = 0.0f;
#pragma unroll
            for (int j = 0; j < kQuads; ++j) o[j] = f32x4{0, 0, 0, 0};
        }
        // over a row, whose lanes have a key each (every row has the same)
        __device__ float sum() const
        {
            float x = l;
            x += turn<8>(x);
            x += turn<4>(x);
            x += turn<2>(x);
            return x + turn<1>(x);
        }
    };

    __device__ static int key(int i, int r, int g) { return r; }

    // (every row's lanes take the one head)
    __device__ static void load_query(const Params &p, const float *q, bool used, int g, typename Base::Query &out)
    {
        Base::load_query(p, q, true, g, out);
    }

    __device__ static void scores(const Params &p, const typename Base::Keys &x, const typename Base::Query &q, int g,
                                  float (&s)[1])
    {
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (!needed<DP, EXACT>(p, 16 * i)) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(x[i][e], q[i][e], sum[e]);
        }
        s[0] = sum_groups((sum[0] + sum[1]) + (sum[2] + sum[3]));
    }

    __device__ static void weigh(float (&s)[1], float scale, bool all, uint32_t in, State &st)
    {
        const bool counts = all || (in & 1);
        float top = counts ? s[0] : -HUGE_VALF;
        top = fmaxf(top, turn<8>(top));
        top = fmaxf(top, turn<4>(top));
        top = fmaxf(top, turn<2>(top));
        top = fmaxf(top, turn<1>(top));
        if (__builtin_amdgcn_ballot_w64(top > st.m) != 0) {
            const float m = fmaxf(st.m, top), f = rescale(st.m, m, scale);
            st.l *= f;
#pragma unroll
            for (int j = 0; j < kQuads; ++j) st.o[j] *= f;
            st.m = m;
        }
        const float m = st.m == -HUGE_VALF ? 0.0f : st.m;
        s[0] = __builtin_amdgcn_exp2f((s[0] - m) * scale);
        s[0] = counts ? s[0] : 0.0f;
        st.l += s[0];
    }

    // (`in` is key r's, the values are those of keys 4 g + i)
    __device__ static void drop(typename Base::Values &x, uint32_t in, int g)
    {
        Base::drop(x, (uint32_t)(__builtin_amdgcn_ballot_w64(in & 1) >> (4 * g)) & 15, g);
    }

    __device__ static void outputs(const typename Base::Values &x, const float (&s)[1], State &st)
    {
        // key 4 g + i's weight to lane i of row g, and from there to the row
        const int lane = threadIdx.x & 63;
        const float mine = __shfl(s[0], (lane / 16 * 4 + lane) % 16);
        const float w[4] = {spread<0>(mine), spread<1>(mine), spread<2>(mine), spread<3>(mine)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kQuads; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.o[j][e] = __builtin_fmaf(w[i], x[i][j][e], st.o[j][e]);
    }

    template <int PAD> __device__ static void store(const State &st, float f, float (*o)[PAD], int heads, int r, int g)
    {
#pragma unroll
        for (int j = 0; j < kQuads; ++j) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = sum_groups(st.o[j][e]) * f;
            if (g == 0) *reinterpret_cast<f32x4 *>(&o[0][64 * j + 4 * r]) = x;
        }
    }
};

// Where the keys of a tile lie, in two steps so that the table's entries can
// be on their way while an earlier tile is worked on: `fetch` reads the table
// for the tile that begins at k0, `resolve` checks the pages and sets the
// addresses.  A key outside the attended ones stands for the nearest of them,
// so nothing else is read, neither of the table nor of the cache.
// Pages of a multiple of 16 slots: 16 keys lie in one page, whose number and
// address are the same for all lanes.
template <class CT, int KEYS, bool WHOLE> struct Rows {
    static constexpr int kN = KEYS / 16;
    int32_t page[kN], slot[kN], low[kN], high[kN];
    const CT *k[kN], *v[kN];
    uint32_t slot_bytes;

    __device__ void fetch(const Params &p, const int32_t *row, int32_t k0, int32_t first_key, int32_t len, int lane)
    {
#pragma unroll
        for (int t = 0; t < kN; ++t) {
            const int32_t key = min(max(k0 + 16 * t, first_key & ~15), (len - 1) & ~15);
            const Place at = Place::of(p, key);
            page[t] = row[at.page];
            slot[t] = at.slot;
            low[t] = max(first_key - key, 0);
            high[t] = min(len - 1 - key, 15);
        }
    }
    __device__ bool resolve(const Params &p, const CT *kb, const CT *vb)
    {
        slot_bytes = (uint32_t)p.slot_stride * (uint32_t)sizeof(CT);
        bool ok = true;
#pragma unroll
        for (int t = 0; t < kN; ++t) {
            ok &= page[t] >= 0 && page[t] < p.n_pages;
            const int64_t off = page[t] * p.page_stride + slot[t] * p.slot_stride;
            k[t] = kb + off;
            v[t] = vb + off;
        }
        return ok;
    }
    __device__ const CT *at(const CT *base, int t, int i) const
    {
        return reinterpret_cast<const CT *>(reinterpret_cast<const char *>(base) +
                                            __umul24(min(max(i, low[t]), high[t]), slot_bytes));
    }
    __device__ const CT *key(int t, int i) const { return at(k[t], t, i); }
    __device__ const CT *value(int t, int i) const { return at(v[t], t, i); }
};

// Any page size: lane l holds the place of key l % KEYS.
template <class CT, int KEYS> struct Rows<CT, KEYS, false> {
    int32_t page, slot;
    int64_t off;
    const CT *kb, *vb;

    __device__ void fetch(const Params &p, const int32_t *row, int32_t k0, int32_t first_key, int32_t len, int lane)
    {
        const Place at = Place::of(p, min(max(k0 + lane % KEYS, first_key), len - 1));
        page = row[at.page];
        slot = at.slot;
    }
    __device__ bool resolve(const Params &p, const CT *kbase, const CT *vbase)
    {
        const bool ok = page >= 0 && page < p.n_pages;
        off = page * p.page_stride + slot * p.slot_stride;
        kb = kbase;
        vb = vbase;
        return __builtin_amdgcn_ballot_w64(!ok) == 0;
    }
    __device__ const CT *key(int t, int i) const { return kb + __shfl(off, 16 * t + i); }
    __device__ const CT *value(int t, int i) const { return vb + __shfl(off, 16 * t + i); }
};

// Four elements of a result row: out = x / l, or what a row without keys or
// with an error has.
template <class T>
__device__ inline void write_row(const Params &p, int b, int head, int d, f32x4 x, float l, bool empty, int32_t bad)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = bad ? __builtin_nanf("") : empty ? 0.0f : x[k] / l;
    *reinterpret_cast<vec<T, 4> *>(static_cast<T *>(p.out) + b * p.out_row + head * p.out_head + d) = from_f32<T, 4>(x);
}

__device__ inline void write_lse(const Params &p, int b, int head, float m, float scale, float l, bool empty, int32_t bad)
{
    if (p.lse)
        p.lse[(int64_t)b * p.n_q_heads + head] =
            bad ? __builtin_nanf("") : empty ? -HUGE_VALF : (m * scale + __builtin_log2f(l)) * kLn2;
}

// Base-2 logarithms per unit of the products with a cache head's keys (which
// are negated for a negative scale).
__device__ inline float scale_of(const Params &p, int kv) { return fabsf(p.scale) * (p.k_scale ? p.k_scale[kv] : 1.0f); }

// A part of a context: d outputs of each head, then the heads' maxima and
// sums; 16-byte aligned.
__host__ __device__ inline int64_t part_size(int heads, int d) { return (int64_t)heads * d + (2 * heads + 3) / 4 * 4; }

struct Part {
    float *o, *m, *l;
    __device__ static Part of(const Params &p, int64_t slot)
    {
        float *o = p.part + slot * part_size(p.part_heads, p.d), *m = o + p.part_heads * p.d;
        return {o, m, m + p.part_heads};
    }
};

// The tiles of all contexts -- (sequence, cache head, tile of 16 query heads)
// -- are laid end to end, each context behind kExtra that stand for its
// beginning and end, and cut into equal runs, one per workgroup; a workgroup's waves
// take the tiles of each context in turn and are joined in shared memory.  A
// context that lies in one run is finished here; the parts of the others go
// to the workspace (slot 0: a context begun by an earlier workgroup, slot 1:
// one that a later workgroup goes on with) for k_join.
template <class P, class T, class CT, int DP, bool WHOLE, bool EXACT>
__global__ __launch_bounds__(kBlock, per_cu(DP, sizeof(CT))) void k_attend(Params p)
{
    constexpr int kKeys = P::kKeys, kPad = DP + 4;
    __shared__ float s_o[kWaves][kTileHeads][kPad];
    __shared__ float s_m[kWaves][kTileHeads], s_l[kWaves][kTileHeads], s_top[kTileHeads];
    __shared__ int64_t s_sum[kWaves];
    __shared__ int32_t s_seq, s_len, s_bad[2];
    __shared__ int64_t s_at;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int units = p.n_heads * p.tiles_of_heads;   // contexts per sequence

    int b, unit, c0 = 0;
    int64_t left, run = 0;
    Span<kKeys> sp;
    if (tid < 2) s_bad[tid] = 0;
    if (p.direct) {
        b = blockIdx.x / units;
        unit = blockIdx.x - b * units;
        sp = Span<kKeys>::of(p, p.seq_len[b]);
        left = sp.cost();
        __syncthreads();
    } else {
        // this workgroup's run: tiles counted per thread, summed over the block
        const int per = (p.n_seq + kBlock - 1) / kBlock, lo = tid * per, hi = min(p.n_seq, lo + per);
        int64_t mine = 0;
        for (int b = lo; b < hi; ++b) mine += Span<kKeys>::of(p, p.seq_len[b]).cost();
        int64_t incl = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t x = __shfl_up(incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 63) s_sum[wave] = incl;
        __syncthreads();
        int64_t total = 0, before = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += s_sum[w];
            total += s_sum[w];
        }
        total = uniform(total) * units;
        constexpr int kRuns = kCus * per_cu(DP, sizeof(CT));   // the grid
        const int64_t even = (total + kRuns - 1) / kRuns;
        run = even > kMinTiles ? even : kMinTiles;
        const int64_t begin = blockIdx.x * run;
        if (begin >= total) {
            if (tid == 0 && !p.by_context) p.cut[blockIdx.x] = make_int4(0, 0, 0, 0);
            return;
        }
        const int64_t end = begin + run < total ? begin + run : total;
        const int64_t excl = (before + incl - mine) * units;
        if (begin >= excl && begin < excl + mine * units) {
            int64_t at = excl;
            for (int b = lo; b < hi; ++b) {
                const int32_t len = p.seq_len[b];
                const int64_t n = (int64_t)Span<kKeys>::of(p, len).cost() * units;
                if (begin < at + n) {
                    s_seq = b;
                    s_len = len;
                    s_at = begin - at;
                    break;
                }
                at += n;
            }
        }
        __syncthreads();
        b = __builtin_amdgcn_readfirstlane(s_seq);
        sp = Span<kKeys>::of(p, __builtin_amdgcn_readfirstlane(s_len));
        left = end - begin;
        {
            const int64_t at = uniform(s_at);
            const int cost = sp.cost();
            unit = at >> 32 == 0 ? (int)((uint32_t)at / (uint32_t)cost) : (int)(at / cost);   // (64 bits take 0.3 us)
            c0 = (int)(at - (int64_t)unit * cost);
        }
    }
    int4 cut = make_int4(0, 0, 0, 0);
    int turn = 0;

    for (; left > 0; ++unit, c0 = 0) {
        while (unit == units || sp.n == 0) {   // the next sequence (one may be left alone)
            sp = Span<kKeys>::of(p, p.seq_len[++b]);
            unit = 0;
        }
        const int cost = sp.cost(), c1 = (int)(cost - c0 < left ? cost : c0 + left);
        left -= c1 - c0;
        const int t0 = max(c0 - kExtra, 0), n = max(c1 - kExtra, 0) - t0;
        if (n == 0) continue;   // the next run begins the context
        const int kv = p.tiles_of_heads == 1 ? unit : unit / p.tiles_of_heads;
        const int hb = (unit - kv * p.tiles_of_heads) * kTileHeads;
        const int heads = min(kTileHeads, p.group - hb), q0 = kv * p.group + hb;
        const bool whole = n == sp.n;
        const int32_t *row = p.table + b * p.table_stride;

        const float scale = scale_of(p, kv);
        typename P::State st;
        st.clear();
        if (sp.len > 0) {
            // (in registers before an output of theirs is written: out may be q)
            typename P::Query q;
            P::load_query(p, static_cast<const T *>(p.q) + b * p.q_row + (q0 + (r < heads ? r : 0)) * p.q_head,
                          r < heads, g, q);
            const CT *kb = static_cast<const CT *>(p.k) + kv * p.head_stride;
            const CT *vb = static_cast<const CT *>(p.v) + kv * p.head_stride;
            // The next tile's keys are on their way as soon as the scores are
            // known, its values as soon as the outputs are; the table's
            // entries a tile ahead of both.
            typename P::Keys keys;
            typename P::Values values;
            Rows<CT, kKeys, WHOLE> rows;
            const int last = t0 + n;
            auto fetch = [&](int t) {
                rows.fetch(p, row, (sp.first_tile + min(t, last - 1)) * kKeys, sp.first_key, sp.len, lane);
            };
            bool ok = true;
            int t = t0 + wave;
            if (t < last) {
                fetch(t);
                ok = rows.resolve(p, kb, vb);
                if (ok) {
                    P::load_keys(p, rows, r, g, keys);
                    P::load_values(p, rows, r, g, values);
                    fetch(t + kWaves);
                }
            }
            while (ok && t < last) {
                const int next = t + kWaves;
                if (next < last) ok = rows.resolve(p, kb, vb);
                const bool more = ok && next < last;
                const int k0 = (sp.first_tile + t) * kKeys;
                const bool all = k0 >= sp.first_key && sp.len - k0 >= kKeys;
                uint32_t in = 0;
                if (!all) {
#pragma unroll
                    for (int i = 0; i < P::kMine; ++i) {
                        const int j = k0 + P::key(i, r, g);
                        if (j >= sp.first_key && j < sp.len) in |= 1u << i;
                    }
                }
                float s[P::kMine];
                P::scores(p, keys, q, g, s);
                if (more) P::load_keys(p, rows, r, g, keys);
                P::weigh(s, scale, all, in, st);
                if (!all) P::drop(values, in, g);
                P::outputs(values, s, st);
                if (more) {
                    P::load_values(p, rows, r, g, values);
                    fetch(next + kWaves);
                }
                t = next;
            }
            if (!ok) s_bad[turn] = DSIM_ST_BAD_PAGE;
        }

        // Join the waves.  Two barriers a context: what the next one writes
        // before its first is not read after this one's second, but for
        // s_bad, which takes turns.
        const float l = st.sum();
        if (g == 0) s_m[wave][r] = st.m;
        __syncthreads();
        float top = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        const float f = rescale(st.m, top, scale);
        P::store(st, f, s_o[wave], heads, r, g);
        if (g == 0) {
            s_l[wave][r] = l * f;
            if (wave == 0) s_top[r] = top;
        }
        if (tid == 0) s_bad[turn ^ 1] = 0;
        __syncthreads();
        const int32_t bad = sp.bad ? DSIM_ST_BAD_POSITION : s_bad[turn];
        turn ^= 1;
        const Part part = Part::of(p, 2 * blockIdx.x + (t0 == 0 ? 1 : 0));
        const float vs = p.v_scale ? p.v_scale[kv] : 1.0f;
        const int quads = EXACT ? DP / 4 : p.d / 4;
        for (int i = tid; i < heads * quads; i += kBlock) {
            const int h = i / quads, d = 4 * (i - h * quads);
            float sum = s_l[0][h];
            f32x4 o = *reinterpret_cast<const f32x4 *>(&s_o[0][h][d]);
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                sum += s_l[w][h];
                o += *reinterpret_cast<const f32x4 *>(&s_o[w][h][d]);
            }
            o *= vs;
            if (whole) {
                write_row<T>(p, b, q0 + h, d, o, sum, sp.len == 0, bad);
                if (d == 0) write_lse(p, b, q0 + h, s_top[h], scale, sum, sp.len == 0, bad);
            } else {
                *reinterpret_cast<f32x4 *>(part.o + h * p.d + d) = o;
                if (d == 0) {
                    part.m[h] = s_top[h];
                    part.l[h] = bad ? -1.0f : sum;   // (a sum is never negative)
                }
            }
        }
        if (whole && tid == 0 && p.status) p.status[b] = bad;
        if (t0 == 0) {
            // parts: this one, then the runs of the workgroups behind, the
            // last possibly short; 0 if nothing is cut off
            cut = make_int4(whole ? 0 : 1 + (int)((sp.n - n + run - 1) / run), b, q0, (int)blockIdx.x);
            if (p.by_context && tid == 0) p.cut[b * units + unit] = cut;
        }
    }
    if (tid == 0 && !p.by_context && !p.direct) p.cut[blockIdx.x] = cut;
}

// Joins the parts of the contexts that are cut.  W waves take a head of a
// context, or its share where the grid has several layers.  Their
// threads are `ways` rows, row w taking four elements each of the parts w,
// w + ways, ...  The first of those are on their way before the weights they
// get are known.
template <class T, int W> __global__ __launch_bounds__(kBlock) void k_join(Params p)
{
    constexpr int kThreads = 64 * W, kHeads = kBlock / kThreads, kAhead = 8;
    __shared__ float s_m[kWaves], s_l[kWaves];
    __shared__ int s_wrong[kWaves];
    __shared__ f32x4 s_o[kBlock];
    const int4 cut = p.cut[blockIdx.x];
    const int n = cut.x, b = cut.y, q0 = cut.z, w0 = cut.w;
    const int tid = threadIdx.x % kThreads, lane = tid & 63, wave = threadIdx.x / 64, mine = threadIdx.x / kThreads;
    const int h = blockIdx.y * kHeads + mine, first = wave / W * W;
    // (nobody begins the context of a row that is left alone)
    if (p.by_context && p.seq_len[blockIdx.x / (p.n_heads * p.tiles_of_heads)] < 0) return;
    if (n == 0) return;
    const bool used = h < p.part_heads && q0 + h < (q0 / p.group + 1) * p.group;   // (a last tile may have fewer heads)
    const float scale = scale_of(p, q0 / p.group);
    auto part = [&](int i) { return Part::of(p, i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)); };
    const int quads = p.d / 4 / (int)gridDim.z, ways = kThreads / quads, way = tid / quads;
    const int d0 = 4 * (tid - way * quads + (int)blockIdx.z * quads);
    const int count = used && way < ways ? n : 0;
    auto output = [&](int i) { return *reinterpret_cast<const f32x4 *>(part(i).o + h * p.d + d0); };
    f32x4 ahead[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (way + j * ways < count) ahead[j] = output(way + j * ways);

    float m = -HUGE_VALF;
    int wrong = 0;
    for (int i = tid; used && i < n; i += kThreads) {
        m = fmaxf(m, part(i).m[h]);
        wrong |= part(i).l[h] < 0.0f;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    wrong = __builtin_amdgcn_ballot_w64(wrong) != 0;
    if (W > 1) {
        if (lane == 0) {
            s_m[wave] = m;
            s_wrong[wave] = wrong;
        }
        __syncthreads();
        for (int w = first; w < first + W; ++w) {
            m = fmaxf(m, s_m[w]);
            wrong |= s_wrong[w];
        }
    }
    float l = 0.0f;
    for (int i = tid; used && i < n; i += kThreads) l += rescale(part(i).m[h], m, scale) * part(i).l[h];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o);
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (way + j * ways < count) o += rescale(part(way + j * ways).m[h], m, scale) * ahead[j];
#pragma unroll 4
    for (int i = way + kAhead * ways; i < count; i += ways) o += rescale(part(i).m[h], m, scale) * output(i);
    s_o[threadIdx.x] = o;
    if (lane == 0) s_l[wave] = l;
    __syncthreads();
    if (!used) return;
    l = 0.0f;
    for (int w = first; w < first + W; ++w) l += s_l[w];
    const int32_t bad = wrong ? DSIM_ST_BAD_PAGE : 0;
    if (tid < quads) {
        for (int w = 1; w < ways; ++w) o += s_o[mine * kThreads + w * quads + tid];
        write_row<T>(p, b, q0 + h, d0, o, l, false, bad);
    }
    if (tid == 0 && blockIdx.z == 0) {
        write_lse(p, b, q0 + h, m, scale, l, false, bad);
        if (p.status) p.status[b] = bad;
    }
}

template <template <bool, bool> class P, class T, class CT, int DP>
void launch_attend(const Params &p, bool stream, dim3 grid, hipStream_t s)
{
    // 16 slots of a page at offsets of 24-bit products
    const bool whole = p.page_size % 16 == 0 && p.slot_stride * (int64_t)sizeof(CT) < 1 << 24;
    if (whole && p.d == DP && stream)
        hipLaunchKernelGGL((k_attend<P<true, true>, T, CT, DP, true, true>), grid, dim3(kBlock), 0, s, p);
    else if (whole && p.d == DP)
        hipLaunchKernelGGL((k_attend<P<true, false>, T, CT, DP, true, true>), grid, dim3(kBlock), 0, s, p);
    else if (whole)
        hipLaunchKernelGGL((k_attend<P<false, false>, T, CT, DP, true, false>), grid, dim3(kBlock), 0, s, p);
    else
        hipLaunchKernelGGL((k_attend<P<false, false>, T, CT, DP, false, false>), grid, dim3(kBlock), 0, s, p);
}

template <class T, class CT, int DP> struct Passes {
    template <bool EXACT, bool STREAM> using ByColumn = Pass<T, CT, DP, EXACT, STREAM>;
    template <bool EXACT, bool STREAM> using One = OnePass<DP, EXACT, STREAM>;
};

template <class T, class CT, int DP> dsim_status launch(Params &p, hipStream_t s)
{
    using P = Pass<T, CT, DP, true, false>;
    const int64_t contexts = (int64_t)p.n_seq * p.n_heads * p.tiles_of_heads;
    p.grid = kCus * per_cu(DP, sizeof(CT));
    // Contexts that cannot be long (the block table has no room, or the window
    // is short) take a workgroup each and need neither the cut nor the join.
    // Where that leaves CUs idle, fewer tiles are worth the join the longer a
    // tile takes (us, a workgroup each and cut): bf16, 8 cache heads of 128,
    // 1 sequence of 512 tokens 11.0 and 13.3, of 768 13.4 and 13.2, of 1,000
    // 15.9 and 13.3; 4 of one head of 256, 384 tokens 15.3 and 16.0, 512 17.6
    // and 16.0; fp32, 8 heads of 128, 256 tokens 12.8 and 14.0, 384 16.0 and
    // 13.9.  Many contexts: 8 heads of 128 in bf16, a window of 1,000, 16
    // sequences 19.0 and 21.7, 64 45.5 and 51.2, in e4m3 24.8 and 32.7; fp32,
    // a window of 500, 64 48.2 and 54.1, but up to 1,000 tokens of any number
    // 71 and 63, for one long context is all that is left in the end; 16 heads
    // of 256, one workgroup a CU, bf16, a window of 1,000 193 and 183.
    int64_t most = (int64_t)p.table_width * p.page_size;
    if (p.window > 0 && p.window < most) most = p.window;
    const bool many = contexts >= kCus / 2 && per_cu(DP, sizeof(CT)) > 1;
    const int tiles = DP <= 64 || many ? 32 : DP <= 128 ? (sizeof(CT) == 4 ? 16 : 24) : 12;
    p.direct = most <= tiles * P::kKeys && contexts < 1 << 24;
    p.by_context = !p.direct && contexts <= p.grid;
    const dim3 grid((unsigned)(p.direct ? contexts : p.grid)), block(kBlock);
    // What the last-level cache (256 MB) cannot keep until the next step is
    // read past it: a batch of 64 up to 4,096 tokens (538 MB) 99 us, with
    // plain loads 108; 131,072 tokens x 4 (2.1 GB) 345 and 381.  What it may
    // keep is not: 8,000 tokens (33 MB) read again 18.7 us, streamed 20.0.
    // Nor are rows of other lengths than 64, 128 and 256, whose lines are
    // touched more than once (heads of 80: 97 us, with plain loads 76), nor
    // pages of other sizes than multiples of 16 (heads of 64: 61 and 63).
    const double row = 2.0 * p.d * sizeof(CT) * p.n_heads, cached = row * (double)p.n_pages * p.page_size;
    const double asked = row * (double)p.n_seq * (double)most;
    const bool stream = (asked < cached ? asked : cached) > 256e6;
    using Kinds = Passes<T, CT, DP>;
    if constexpr (sizeof(T) == 4) {
        if (p.group == 1)
            launch_attend<Kinds::template One, T, CT, DP>(p, stream, grid, s);
        else
            launch_attend<Kinds::template ByColumn, T, CT, DP>(p, stream, grid, s);
    } else {
        launch_attend<Kinds::template ByColumn, T, CT, DP>(p, stream, grid, s);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "paged attention launch");
    if (p.direct) return DSIM_OK;
    // Few heads have many parts each, and waves to spare.  32 query and 8
    // cache heads of 128, 8,000 tokens, by a wave a head, four waves, four
    // workgroups (us, both launches): 1 sequence 21.8, 18.4, 17.7; 4: 35.5,
    // 32.1, 32.3; 8: 56.8, 55.5, 58.9; 16: 97.8, 96.8, 107; with 2,500 tokens
    // 32 sequences 66.5 and 69.5 by a wave and by four.
    const unsigned x = (unsigned)(p.by_context ? contexts : p.grid), heads = (unsigned)p.part_heads;
    const int64_t joins = (int64_t)p.n_seq * p.n_q_heads;
    if (joins <= p.grid)
        hipLaunchKernelGGL((k_join<T, 4>), dim3(x, heads, joins * 4 <= p.grid ? 4 : 1), block, 0, s, p);
    else
        hipLaunchKernelGGL((k_join<T, 1>), dim3(x, (heads + 3) / 4), block, 0, s, p);
    e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "paged attention join launch");
}

template <class T, class CT> dsim_status launch(Params &p, hipStream_t s)
{
    return p.d <= 64 ? launch<T, CT, 64>(p, s) : p.d <= 128 ? launch<T, CT, 128>(p, s) : launch<T, CT, 256>(p, s);
}

// by the queries' type, in a translation unit each
dsim_status launch_f32(Params &p, hipStream_t s);
dsim_status launch_f16(Params &p, bool e4m3_cache, hipStream_t s);
dsim_status launch_bf16(Params &p, bool e4m3_cache, hipStream_t s);

}  // namespace attend
}  // namespace dsim
