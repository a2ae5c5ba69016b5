// paged_attention.hip -- attention of one new token per sequence over its
// paged keys and values (dsim_paged_attention).
#include "numeric.h"
#include "ops.h"

namespace dsim {
namespace {

constexpr int kWaves = 4;
constexpr int kBlock = 64 * kWaves;
constexpr int kGrid = 512;        // two workgroups per CU
constexpr int kMinTiles = 4;      // a tile for every wave
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
    int4 *cut;            // per workgroup: the context its last part is cut from
    int64_t n_pages, page_stride, slot_stride, head_stride, table_stride, q_row, q_head, out_row, out_head;
    float scale;          // times log2 e
    int32_t n_seq, n_heads, n_q_heads, d, page_size, table_width, window;
    int32_t group, tiles_of_heads, part_heads;
};

// The keys of a sequence in tiles: first tile, number of tiles (at least
// one, so that somebody writes the row; none if the row is left alone).
template <int KEYS> struct Span {
    int32_t first_key, len, first_tile, n;
    bool bad;
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

// Running state of one wave: for column r (a query head) the maximum m, this
// lane's share of the sum l, and the output's rows.
template <int NT> struct State {
    float m, l;
    f32x4 o[NT];
};

__device__ inline float max_groups(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

__device__ inline float sum_groups(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// What sums held against the maximum `from` count against the maximum `to`.
// Where there was none (-inf) they are held against 0: zero, or NaN, which
// has to stay.
__device__ inline float rescale(float from, float to)
{
    return from == -HUGE_VALF ? 1.0f : __builtin_amdgcn_exp2f(from - to);
}

// The running maximum takes in the scores s (base-2 logarithms); returns them
// as weights, 2^SHIFT for a score at the maximum.
template <int SHIFT, int N, int NT> __device__ inline void weigh(float (&s)[N], State<NT> &st)
{
    float top = s[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, s[i]);
    top = max_groups(top);
    if (__builtin_amdgcn_ballot_w64(top > st.m) != 0) {
        const float m = fmaxf(st.m, top);
        const float f = rescale(st.m, m);
        st.l *= f;
#pragma unroll
        for (int e = 0; e < NT; ++e) st.o[e] *= f;
        st.m = m;
    }
    const float m = st.m == -HUGE_VALF ? 0.0f : st.m - SHIFT;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = __builtin_amdgcn_exp2f(s[i] - m);
        st.l += s[i];
    }
}

// 16-bit queries; keys and values of the same type or e4m3.
template <class T, class CT, int DP> struct Pass {
    static constexpr int kKeys = 32, kE = DP / 16, kTiles = DP / 16;
    static constexpr bool k8 = __is_same(CT, e4m3);
    static constexpr int kChunk = 16 / sizeof(CT);            // elements per 16-byte load of a key
    static constexpr int kSteps = DP / (4 * kChunk);          // loads of a key per lane
    static constexpr int kParts = kChunk / 8;                 // products per load
    // fp16 ends at 2^-24: weights from 2^15 down keep a long tail of small
    // ones, which together may weigh as much as the largest
    static constexpr int kShift = __is_same(T, f16) ? 15 : 0;
    using Query = vec<T, 8>[kSteps * kParts];

    struct Data {
        u32x4 k[2][kSteps];
        vec<CT, kE> v[8];
    };

    __device__ static void load_query(const Params &p, const T *q, bool used, int g, Query &out)
    {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int h = 0; h < kParts; ++h) {
                const int at = (4 * s + g) * kChunk + 8 * h;
                out[s * kParts + h] = used && at < p.d ? *reinterpret_cast<const vec<T, 8> *>(q + at) : vec<T, 8>(0);
            }
    }

    // off: the lane's key's place (key lane % 32 of the tile)
    __device__ static void load(const Params &p, const CT *k, const CT *v, int64_t off, int r, int g, Data &x)
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const CT *row = k + __shfl(off, t * 16 + r);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int at = (4 * s + g) * kChunk;
                x.k[t][s] = *reinterpret_cast<const u32x4 *>(row + (at < p.d ? at : 0));
            }
        }
        const int at = kE * r < p.d ? kE * r : 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x.v[4 * t + i] = *reinterpret_cast<const vec<CT, kE> *>(v + __shfl(off, t * 16 + 4 * g + i) + at);
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

    __device__ static vec<T, 8> widen8(uint32_t lo, uint32_t hi)
    {
        vec<float, 8> f;
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, true);
        const auto c = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, true);
        f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1], f[4] = c[0], f[5] = c[1], f[6] = d[0], f[7] = d[1];
        return __builtin_convertvector(f, vec<T, 8>);
    }

    // A weight as the sum of two numbers of T: with one the output would carry
    // an error as large as its own rounding.  The first is cut off, the
    // second is never 0 (at least the type's smallest that the products keep,
    // 2^-39 of the largest weight in fp16), so that an infinite value times
    // both is that infinity.
    __device__ static void split(const float (&s)[8], vec<T, 8> &hi, vec<T, 8> &lo)
    {
        vec<float, 8> rest;
        if constexpr (__is_same(T, bf16)) {
            vec<uint32_t, 4> w;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t bits = __builtin_bit_cast(uint32_t, s[i]);
                rest[i] = fmaxf(s[i] - __builtin_bit_cast(float, bits & 0xffff0000u), 0x1p-126f);
                if (i % 2)
                    w[i / 2] |= bits & 0xffff0000u;
                else
                    w[i / 2] = bits >> 16;
            }
            hi = __builtin_bit_cast(vec<T, 8>, w);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const auto two = __builtin_amdgcn_cvt_pkrtz(s[i], s[i + 1]);
                hi[i] = (T)two[0];
                hi[i + 1] = (T)two[1];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) rest[i] = fmaxf(s[i] - (float)hi[i], 0x1p-24f);
        }
        lo = __builtin_convertvector(rest, vec<T, 8>);
    }

    // valid: bit 4 t + i of the lane's keys; all: every key of the tile counts
    __device__ static void compute(const Params &p, Data &x, const Query &q, float scale, int g, uint32_t valid,
                                   bool all, State<kTiles> &st)
    {
        float s[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int h = 0; h < kParts; ++h)
                    acc = Mfma<T>::mul(part(x.k[t][i], h, (4 * i + g) * kChunk < p.d), q[i * kParts + h], acc);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * t + i] = acc[i] * scale;
        }
        if (!all) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = valid >> i & 1;
                s[i] = in ? s[i] : -HUGE_VALF;
                x.v[i] = in ? x.v[i] : vec<CT, kE>(0);   // what lies there may be infinite or NaN
            }
        }
        weigh<kShift>(s, st);
        vec<T, 8> hi, lo;
        split(s, hi, lo);
        vec<T, kE> row[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) row[i] = to_t(x.v[i]);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            vec<T, 8> a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = row[i][e];
            st.o[e] = Mfma<T>::mul(a, hi, st.o[e]);
            st.o[e] = Mfma<T>::mul(a, lo, st.o[e]);
        }
    }

    __device__ static vec<T, kE> to_t(vec<CT, kE> x)
    {
        if constexpr (k8) {
            const auto w = __builtin_bit_cast(vec<uint32_t, kE / 4>, x);
            vec<T, kE> y;
#pragma unroll
            for (int i = 0; i < kE / 4; ++i) {
                const vec<T, 8> z = widen8(w[i], 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[4 * i + j] = z[j];
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
template <int DP> struct Pass<float, float, DP> {
    static constexpr int kKeys = 16, kTiles = DP / 16, kSteps = DP / 16, kQuads = DP / 64, kShift = 0;
    using Query = f32x4[kSteps];

    struct Data {
        f32x4 k[kSteps];
        f32x4 v[4][kQuads];
    };

    __device__ static void load_query(const Params &p, const float *q, bool used, int g, Query &out)
    {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = (4 * s + g) * 4;
            out[s] = used && at < p.d ? *reinterpret_cast<const f32x4 *>(q + at) : f32x4{0, 0, 0, 0};
        }
    }

    __device__ static void load(const Params &p, const float *k, const float *v, int64_t off, int r, int g, Data &x)
    {
        const float *row = k + __shfl(off, r);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = (4 * s + g) * 4;
            x.k[s] = *reinterpret_cast<const f32x4 *>(row + (at < p.d ? at : 0));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float *val = v + __shfl(off, 4 * g + i);
#pragma unroll
            for (int j = 0; j < kQuads; ++j) {
                const int at = 64 * j + 4 * r;
                x.v[i][j] = *reinterpret_cast<const f32x4 *>(val + (at < p.d ? at : 0));
            }
        }
    }

    __device__ static void compute(const Params &p, Data &x, const Query &q, float scale, int g, uint32_t valid,
                                   bool all, State<kTiles> &st)
    {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = (4 * i + g) * 4 < p.d;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? x.k[i][e] : 0.0f, q[i][e], acc, 0, 0, 0);
        }
        float s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = acc[i] * scale;
        if (!all) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = valid >> i & 1;
                s[i] = in ? s[i] : -HUGE_VALF;
#pragma unroll
                for (int j = 0; j < kQuads; ++j) x.v[i][j] = in ? x.v[i][j] : f32x4{0, 0, 0, 0};
            }
        }
        weigh<kShift>(s, st);
#pragma unroll
        for (int j = 0; j < kQuads; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    st.o[4 * j + e] =
                        __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[i][j][e], s[i], st.o[4 * j + e], 0, 0, 0);
    }

    __device__ static int dim(int g, int i, int e) { return 64 * (e / 4) + (4 * g + i) * 4 + e % 4; }
};

// A result row's elements: out = x / l, or what a row without keys or with an
// error has.
template <class T>
__device__ inline void write_row(const Params &p, int b, int head, int d, float x, float l, bool empty, int32_t bad)
{
    const float y = bad ? __builtin_nanf("") : empty ? 0.0f : x / l;
    static_cast<T *>(p.out)[b * p.out_row + head * p.out_head + d] = (T)y;
}

template <int SHIFT>
__device__ inline void write_lse(const Params &p, int b, int head, float m, float l, bool empty, int32_t bad)
{
    if (p.lse)
        p.lse[(int64_t)b * p.n_q_heads + head] =
            bad ? __builtin_nanf("") : empty ? -HUGE_VALF : (m + (__builtin_log2f(l) - SHIFT)) * kLn2;
}

// m, l of 16 heads and 16 x d outputs
__device__ inline float *part_of(const Params &p, int64_t slot)
{
    return p.part + slot * ((int64_t)p.part_heads * (p.d + 2));
}

// The tiles of all (sequence, cache head, tile of 16 query heads) are laid
// end to end and cut into equal runs, one per workgroup; a workgroup's waves
// take the tiles of each context in turn and are joined in shared memory.  A
// context that lies in one run is finished here; the parts of the others go
// to the workspace (slot 0: a context begun by an earlier workgroup, slot 1:
// one that a later workgroup goes on with) for k_join.
template <class T, class CT, int DP> __global__ __launch_bounds__(kBlock) void k_attend(Params p)
{
    using P = Pass<T, CT, DP>;
    constexpr int kKeys = P::kKeys, NT = P::kTiles, kPad = DP + 4;
    __shared__ float s_o[kWaves][kTileHeads][kPad];
    __shared__ float s_m[kWaves][kTileHeads], s_l[kWaves][kTileHeads];
    __shared__ int64_t s_sum[kWaves];
    __shared__ int32_t s_seq, s_bad;
    __shared__ int64_t s_at;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
    const int units = p.n_heads * p.tiles_of_heads;   // contexts per sequence

    // this workgroup's run: tiles counted per thread, summed over the block
    const int per = (p.n_seq + kBlock - 1) / kBlock, lo = tid * per, hi = min(p.n_seq, lo + per);
    int64_t mine = 0;
    for (int b = lo; b < hi; ++b) mine += Span<kKeys>::of(p, p.seq_len[b]).n;
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t x = __shfl_up(incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 63) s_sum[wave] = incl;
    if (tid == 0) s_seq = -1;
    __syncthreads();
    int64_t total = 0, before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s_sum[w];
        total += s_sum[w];
    }
    total *= units;
    const int64_t even = (total + gridDim.x - 1) / gridDim.x, run = even > kMinTiles ? even : kMinTiles;
    const int64_t begin = blockIdx.x * run;
    if (begin >= total) {
        if (tid == 0) p.cut[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }
    const int64_t end = begin + run < total ? begin + run : total;
    const int64_t excl = (before + incl - mine) * units;
    if (begin >= excl && begin < excl + mine * units) {
        int64_t at = excl;
        for (int b = lo; b < hi; ++b) {
            const int64_t n = (int64_t)Span<kKeys>::of(p, p.seq_len[b]).n * units;
            if (begin < at + n) {
                s_seq = b;
                s_at = begin - at;
                break;
            }
            at += n;
        }
    }
    __syncthreads();
    int b = s_seq;
    int64_t at = s_at, left = end - begin;
    int4 cut = make_int4(0, 0, 0, 0);

    while (left > 0) {
        const Span<kKeys> sp = Span<kKeys>::of(p, p.seq_len[b]);
        if (at >= (int64_t)sp.n * units) {   // (also a sequence that is left alone)
            ++b;
            at = 0;
            continue;
        }
        const int unit = (int)(at / sp.n), t0 = (int)(at % sp.n);
        const int n = (int)(sp.n - t0 < left ? sp.n - t0 : left);
        const int kv = unit / p.tiles_of_heads, hb = unit % p.tiles_of_heads * kTileHeads;
        const int heads = min(kTileHeads, p.group - hb), q0 = kv * p.group + hb;
        const bool whole = n == sp.n;
        const int32_t *row = p.table + b * p.table_stride;

        State<NT> st;
        st.m = -HUGE_VALF;
        st.l = 0.0f;
#pragma unroll
        for (int e = 0; e < NT; ++e) st.o[e] = f32x4{0, 0, 0, 0};
        if (tid == 0) s_bad = sp.bad ? DSIM_ST_BAD_POSITION : 0;
        __syncthreads();

        if (sp.len > 0) {
            typename P::Query q;
            P::load_query(p, static_cast<const T *>(p.q) + b * p.q_row + (q0 + (r < heads ? r : 0)) * p.q_head,
                          r < heads, g, q);
            const float scale = p.scale * (p.k_scale ? p.k_scale[kv] : 1.0f);
            const CT *kb = static_cast<const CT *>(p.k) + kv * p.head_stride;
            const CT *vb = static_cast<const CT *>(p.v) + kv * p.head_stride;
            bool wrong = false;
            for (int t = t0 + wave; t < t0 + n; t += kWaves) {
                const int k0 = (sp.first_tile + t) * kKeys;
                // keys outside [first_key, len) stand for the nearest inside
                const int key = min(max(k0 + lane % kKeys, sp.first_key), sp.len - 1);
                int32_t page = row[key / p.page_size];
                if (page < 0 || page >= p.n_pages) {
                    wrong = true;
                    page = 0;
                }
                const int64_t off = page * p.page_stride + key % p.page_size * p.slot_stride;
                if (__builtin_amdgcn_ballot_w64(wrong) != 0) break;
                typename P::Data x;
                P::load(p, kb, vb, off, r, g, x);
                const bool all = k0 >= sp.first_key && sp.len - k0 >= kKeys;
                uint32_t valid = 0;
#pragma unroll
                for (int i = 0; i < kKeys / 4; ++i) {
                    const int j = k0 + i / 4 * 16 + 4 * g + i % 4;
                    if (j >= sp.first_key && j < sp.len) valid |= 1u << i;
                }
                P::compute(p, x, q, scale, g, valid, all, st);
            }
            if (wrong) s_bad = DSIM_ST_BAD_PAGE;
        }

        // join the waves
        const float l = sum_groups(st.l);
        if (g == 0) {
            s_m[wave][r] = st.m;
            s_l[wave][r] = l;
        }
        __syncthreads();
        float top = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        const float f = rescale(st.m, top);
        if (r < heads) {
#pragma unroll
            for (int e = 0; e < NT; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) s_o[wave][r][P::dim(g, i, e)] = st.o[e][i] * f;
        }
        __syncthreads();
        const int32_t bad = s_bad;
        float *part = part_of(p, 2 * blockIdx.x + (t0 == 0 ? 1 : 0));
        const float vs = p.v_scale ? p.v_scale[kv] : 1.0f;
        for (int i = tid; i < heads * p.d; i += kBlock) {
            const int h = i / p.d, d = i % p.d;
            float m = s_m[0][h];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_m[w][h]);
            float sum = 0.0f, o = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                sum += s_l[w][h] * rescale(s_m[w][h], m);
                o += s_o[w][h][d];
            }
            o *= vs;
            if (whole) {
                write_row<T>(p, b, q0 + h, d, o, sum, sp.len == 0, bad);
                if (d == 0) write_lse<P::kShift>(p, b, q0 + h, m, sum, sp.len == 0, bad);
            } else {
                part[2 * p.part_heads + h * p.d + d] = o;
                if (d == 0) {
                    part[h] = m;
                    part[p.part_heads + h] = bad ? -1.0f : sum;   // (a sum is never negative)
                }
            }
        }
        if (whole) {
            if (tid == 0 && p.status) p.status[b] = bad;
        } else if (t0 == 0) {
            // this part, then the runs of the workgroups behind, the last
            // possibly short
            cut = make_int4(1 + (int)((sp.n - n + run - 1) / run), b, q0, heads);
        }
        at += n;
        left -= n;
        __syncthreads();
    }
    if (tid == 0) p.cut[blockIdx.x] = cut;
}

// Joins the parts of the contexts that workgroups begun and others went on
// with: workgroup (w, h) takes head h of the one begun by workgroup w.
template <class T, int SHIFT> __global__ __launch_bounds__(kBlock) void k_join(Params p)
{
    __shared__ float s_w[kGrid];
    __shared__ float s_red[kWaves];
    const int w0 = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int4 cut = p.cut[w0];
    const int n = cut.x, b = cut.y, q0 = cut.z;
    if (n == 0 || h >= cut.w) return;
    auto part = [&](int i) { return part_of(p, i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)); };
    float m = -HUGE_VALF;
    int wrong = 0;
    for (int i = tid; i < n; i += kBlock) {
        m = fmaxf(m, part(i)[h]);
        wrong |= part(i)[p.part_heads + h] < 0.0f;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) s_red[wave] = m;
    wrong = __syncthreads_or(wrong);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_red[w]);
    __syncthreads();
    float l = 0.0f;
    for (int i = tid; i < n; i += kBlock) {
        const float f = rescale(part(i)[h], m);
        s_w[i] = f;
        l += f * part(i)[p.part_heads + h];
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o);
    if (lane == 0) s_red[wave] = l;
    __syncthreads();
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += s_red[w];
    const int32_t bad = wrong ? DSIM_ST_BAD_PAGE : 0;
    for (int d = tid; d < p.d; d += kBlock) {
        float o = 0.0f;
        for (int i = 0; i < n; ++i) o += s_w[i] * part(i)[2 * p.part_heads + h * p.d + d];
        write_row<T>(p, b, q0 + h, d, o, l, false, bad);
    }
    if (tid == 0) {
        write_lse<SHIFT>(p, b, q0 + h, m, l, false, bad);
        if (p.status) p.status[b] = bad;
    }
}

template <class T, class CT> dsim_status launch(const Params &p, hipStream_t s)
{
    if (p.d <= 64)
        hipLaunchKernelGGL((k_attend<T, CT, 64>), dim3(kGrid), dim3(kBlock), 0, s, p);
    else if (p.d <= 128)
        hipLaunchKernelGGL((k_attend<T, CT, 128>), dim3(kGrid), dim3(kBlock), 0, s, p);
    else
        hipLaunchKernelGGL((k_attend<T, CT, 256>), dim3(kGrid), dim3(kBlock), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "paged attention launch");
    hipLaunchKernelGGL((k_join<T, Pass<T, CT, 64>::kShift>), dim3(kGrid, (unsigned)p.part_heads), dim3(kBlock), 0, s, p);
    e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "paged attention join launch");
}

}  // namespace

size_t attend_workspace(int32_t n_q_heads, int32_t n_heads, int32_t head_dim)
{
    const int group = n_q_heads / n_heads, heads = group < kTileHeads ? group : kTileHeads;
    return (size_t)kGrid * (sizeof(int4) + 2 * (size_t)heads * (size_t)(head_dim + 2) * sizeof(float));
}

dsim_status launch_attend(const AttendArgs &a, hipStream_t s)
{
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
    p.part = reinterpret_cast<float *>(p.cut + kGrid);
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
    p.window = a.window;
    p.group = a.n_q_heads / a.c.n_heads;
    p.tiles_of_heads = (p.group + kTileHeads - 1) / kTileHeads;
    p.part_heads = p.group < kTileHeads ? p.group : kTileHeads;
    if (a.dtype == DSIM_F32) return launch<float, float>(p, s);
    if (a.dtype == DSIM_F16) return a.c.dtype == DSIM_E4M3 ? launch<f16, e4m3>(p, s) : launch<f16, f16>(p, s);
    return a.c.dtype == DSIM_E4M3 ? launch<bf16, e4m3>(p, s) : launch<bf16, bf16>(p, s);
}

}  // namespace dsim
