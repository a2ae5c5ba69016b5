// kv_append.hip -- new keys and values rotated and written into a paged
// cache, queries rotated on the way (dsim_kv_append).
//
// A token is (n_q_heads + 2 n_heads) rows of head_dim elements read once and
// written once, and one row of the rotation table: 3 flops per 2 elements
// moved, so memory bounds it, and latency a call of few tokens.  On MI355X
// 24,588 tokens of prompts (bf16, 32 query and 8 cache heads of 128, 606 MB)
// take 108 us, 5.6 TB/s; one token of 12 heads of 64 takes the kernel 3.0 us and
// calls one after another 4.5.  A token's first wait is for its sequence and
// position, the second for its page, the third for the row (the load stands
// behind the page's check), the fourth for the row's other half and the
// rotation.  (Loading a thread's next chunk before the one at hand is stored
// costs the 24,588 tokens 14 us more.)
#include "numeric.h"
#include "ops.h"

namespace dsim {
namespace {

constexpr int kMaxBlock = 512;

template <class T, int VEC> __device__ inline vec<float, VEC> load_row(const void *p, int64_t at)
{
    return to_f32<T, VEC>(*reinterpret_cast<const vec<T, VEC> *>(static_cast<const T *>(p) + at));
}

// (streaming stores: with plain ones the 24,588 tokens below take 114 us)
template <class T, int VEC> __device__ inline void store_row(void *p, int64_t at, vec<float, VEC> x)
{
    __builtin_nontemporal_store(from_f32<T, VEC>(x), reinterpret_cast<vec<T, VEC> *>(static_cast<T *>(p) + at));
}

// Where a token goes: its place in the cache (elements, without the head)
// and its status.
struct Place {
    int64_t at;
    int32_t status, pos;
    bool skip;
};

__device__ inline Place place_of(const AppendArgs &a, int64_t t)
{
    Place p{0, 0, 0, false};
    const int32_t s = a.seq[t];
    p.pos = a.pos[t];
    p.skip = s < 0;
    if (p.skip) return p;
    if (s >= a.c.n_seq) p.status |= DSIM_ST_BAD_SEQUENCE;
    if (p.pos < 0 || (int64_t)p.pos >= (int64_t)a.c.table_width * a.c.page_size || (a.rope && p.pos >= a.n_rope))
        p.status |= DSIM_ST_BAD_POSITION;
    if (p.status) return p;
    const int32_t page = a.c.block_table[s * a.c.table_stride + p.pos / a.c.page_size];
    if (page < 0 || page >= a.c.n_pages)
        p.status = DSIM_ST_BAD_PAGE;
    else
        p.at = page * a.c.page_stride + (p.pos % a.c.page_size) * a.c.slot_stride;
    return p;
}

// j / n for mul = ceil(2^32 / n), 0 for n = 1; exact for j < 2^26, n <= 64 (a
// call's chunks a token: 2^17, a row's: 64)
__device__ inline uint32_t divide(uint32_t j, uint32_t mul) { return mul ? __umulhi(j, mul) : j; }

// T: type of the new rows; CT: of the cache; VEC: elements per load.  A
// thread takes one chunk of VEC elements, or, where pairs (i, i + R/2) are
// rotated, one chunk of each half.
template <class T, class CT, int VEC> __global__ __launch_bounds__(kMaxBlock) void k_append(AppendArgs a, uint32_t mul_head, uint32_t mul_value)
{
    using V = vec<float, VEC>;
    const int d = a.c.head_dim, rot = a.rot_dim;
    const int n_rot = a.interleaved ? rot / VEC : rot / 2 / VEC;   // chunks that are rotated
    const int per_head = n_rot + (d - rot) / VEC, per_value = d / VEC;
    const int n_q = a.n_q_heads * per_head, n_k = a.c.n_heads * per_head, n_v = a.c.n_heads * per_value;
    for (int64_t t = blockIdx.x; t < a.n_tok; t += gridDim.x) {
        const Place p = place_of(a, t);
        if (threadIdx.x == 0 && a.status) a.status[t] = p.status;
        if (p.skip) continue;
        const float *cs = a.rope ? a.rope + (p.status ? 0 : (int64_t)p.pos * rot) : nullptr;
        for (int i = threadIdx.x; i < n_q + n_k + n_v; i += blockDim.x) {
            if (i >= n_q + n_k) {   // a value: copied
                if (p.status) continue;
                const uint32_t j = i - n_q - n_k, h = divide(j, mul_value), e = (j - __umul24(h, per_value)) * VEC;
                V x = load_row<T, VEC>(a.v.data, t * a.v.row_stride + h * a.v.head_stride + e);
                if (a.c.v_scale) x /= a.c.v_scale[h];
                store_row<CT, VEC>(a.c.v, p.at + h * a.c.head_stride + e, x);
                continue;
            }
            const bool query = i < n_q;
            const uint32_t j = query ? i : i - n_q, h = divide(j, mul_head);
            const int c = j - __umul24(h, per_head);
            const dsim_rows &src = query ? a.q : a.k;
            const int64_t from = t * src.row_stride + h * src.head_stride;
            const int64_t to = query ? t * a.q_out.row_stride + h * a.q_out.head_stride
                                     : p.at + h * a.c.head_stride;
            const bool turned = c < n_rot, two = turned && !a.interleaved;
            const int e = turned ? c * VEC : rot + (c - n_rot) * VEC, e2 = e + rot / 2;
            if (p.status) {
                if (query) {
                    const V nan = V(__builtin_nanf(""));
                    store_row<T, VEC>(a.q_out.data, to + e, nan);
                    if (two) store_row<T, VEC>(a.q_out.data, to + e2, nan);
                }
                continue;
            }
            V x = load_row<T, VEC>(src.data, from + e), y;
            if (two) {
                y = load_row<T, VEC>(src.data, from + e2);
                const V cosv = *reinterpret_cast<const V *>(cs + e), sinv = *reinterpret_cast<const V *>(cs + rot / 2 + e);
                const V z = x * cosv - y * sinv;
                y = y * cosv + x * sinv;
                x = z;
            } else if (turned) {
                using H = vec<float, VEC / 2>;
                const H co = *reinterpret_cast<const H *>(cs + e / 2), si = *reinterpret_cast<const H *>(cs + (rot + e) / 2);
#pragma unroll
                for (int k = 0; k < VEC; k += 2) {
                    const float z = x[k] * co[k / 2] - x[k + 1] * si[k / 2];
                    x[k + 1] = x[k + 1] * co[k / 2] + x[k] * si[k / 2];
                    x[k] = z;
                }
            }
            if (query) {
                store_row<T, VEC>(a.q_out.data, to + e, x);
                if (two) store_row<T, VEC>(a.q_out.data, to + e2, y);
            } else {
                if (a.c.k_scale) {
                    x /= a.c.k_scale[h];
                    if (two) y /= a.c.k_scale[h];
                }
                store_row<CT, VEC>(a.c.k, to + e, x);
                if (two) store_row<CT, VEC>(a.c.k, to + e2, y);
            }
        }
    }
}

template <class T, class CT, int VEC> void launch(const AppendArgs &a, hipStream_t s)
{
    // A workgroup takes a token.  Few tokens: a thread for every chunk, up to
    // 512 (bf16, 32 query and 8 cache heads of 128: 256 tokens 4.1 us, with
    // 128 threads 5.4).  Many: fewer and busier threads, so that fewer
    // workgroups start (24,588 tokens 114 us, with 512 threads 173, both
    // with plain stores); one wave where a token has few chunks, or an e4m3
    // cache needs more arithmetic for each.  8,192 tokens by one wave and two,
    // bf16 of 96 chunks 10.9 and 11.9 us, 128 11.9 and 12.4, 192 16.4 and
    // 15.8, 448 33.7 and 33.7; fp16 neighbours into e4m3 of 192 chunks 12.7 and
    // 14.3, 288 17.0 and 18.2, 336 20.6 and 21.6, 384 19.9 and 19.9, 480 37.2
    // and 35.4.  (At 2,048 tokens e4m3 loses from 240 chunks on: 288 7.6 and
    // 7.0.)
    const int n_rot = a.interleaved ? a.rot_dim / VEC : a.rot_dim / 2 / VEC, rest = (a.c.head_dim - a.rot_dim) / VEC;
    const int64_t chunks = (int64_t)(a.n_q_heads + a.c.n_heads) * (n_rot + rest) + (int64_t)a.c.n_heads * (a.c.head_dim / VEC);
    const int64_t few = sizeof(CT) == 1 ? 320 : 128;
    const int64_t most = a.n_tok < 1024 ? kMaxBlock : chunks <= few ? 64 : 128, rounds = (chunks + most - 1) / most;
    const int block = (int)((chunks + 64 * rounds - 1) / (64 * rounds)) * 64;
    const dim3 grid((unsigned)(a.n_tok < (1 << 20) ? a.n_tok : (1 << 20)));
    const auto mul = [](int n) { return n > 1 ? (uint32_t)((((uint64_t)1 << 32) + n - 1) / n) : 0u; };
    hipLaunchKernelGGL((k_append<T, CT, VEC>), grid, dim3(block), 0, s, a, mul(n_rot + rest), mul(a.c.head_dim / VEC));
}

template <class T, class CT> void launch(const AppendArgs &a, hipStream_t s)
{
    // chunks of 16 bytes of T; 4 elements where a half of the rotated part
    // is no whole number of 8
    if constexpr (sizeof(T) == 4) {
        launch<T, CT, 4>(a, s);
    } else {
        if (a.rot_dim % 16)
            launch<T, CT, 4>(a, s);
        else
            launch<T, CT, 8>(a, s);
    }
}

}  // namespace

dsim_status launch_append(const AppendArgs &a, hipStream_t s)
{
    if (a.dtype == DSIM_F32)
        launch<float, float>(a, s);
    else if (a.dtype == DSIM_F16 && a.c.dtype == DSIM_F16)
        launch<f16, f16>(a, s);
    else if (a.dtype == DSIM_BF16 && a.c.dtype == DSIM_BF16)
        launch<bf16, bf16>(a, s);
    else if (a.dtype == DSIM_F16)
        launch<f16, e4m3>(a, s);
    else
        launch<bf16, e4m3>(a, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "append launch");
}

}  // namespace dsim
