// kv_compact.hip -- kept tokens of a sequence move to its front
// (dsim_kv_compact).
//
// Bound by memory: each kept row is read and written once.  A place that is
// written may be one that another kept token still has to be read from, but
// never one that a later token of the ascending list comes from (the list's
// j-th entry is at least j), so a workgroup that takes its share of every row
// in the list's order, and reads a batch before it writes it, needs no second
// copy.  Its share is a piece of one layer's keys or values of one head.
//
// On MI355X 8 contexts of 4,096 to 16,384 tokens of which half stay (two layers,
// 8 heads of 128, bf16: 336 MB read and as many written) take 174 us, 3.9 TB/s:
// every batch waits for its rows, and its stores stand before the next ones'
// loads.  (Entries, pages and rows asked for three, two and one batch ahead, so
// that nothing waits for anything of its own batch: 172 us, but a short list
// 6.3 to 9.3 us for 5.5.)  The path of a tree, a list of a few entries, takes
// the call 5.5 us: a chain of four loads.
#include "multi_ops.h"
#include "numeric.h"

namespace dsim {
namespace {

// Pieces of 16 bytes that a thread has in flight (of long lists with 4: 178 us).
constexpr int rows_at_once(int block) { return block > 256 ? 6 : 8; }

// blockIdx.x: sequence; y: layer's keys or values; z: columns, pieces of 16
// bytes of a token's rows, `per` of them.  A thread takes one of them of
// every `ways`-th token.
template <int BLOCK> __global__ __launch_bounds__(BLOCK) void k_compact(Layers l, CompactArgs a, int per)
{
    __shared__ int32_t s_n, s_bad;
    const int32_t s = blockIdx.x;
    const int64_t start = a.start[s], room = (int64_t)a.table_width * l.page_size;
    const int32_t *keep = a.keep + s * a.keep_stride;
    const int32_t want = min(max(a.n_keep[s], 0), a.keep_width);
    if (threadIdx.x == 0) {
        s_n = start < 0 ? 0 : want;
        s_bad = 0;
    }
    __syncthreads();
    // the list ends before the first entry that does not ascend or has no place
    for (int32_t j = threadIdx.x; j < want; j += BLOCK) {
        const int32_t k = keep[j];
        if (k < 0 || (j > 0 && k <= keep[j - 1]) || start + k >= room) {
            atomicMin(&s_n, j);
            break;
        }
    }
    __syncthreads();
    const int32_t n = s_n;
    const int ways = BLOCK / per, way = threadIdx.x / per, column = blockIdx.z * per + threadIdx.x - way * per;
    const int head = column / l.chunks;
    const bool used = way < ways && head < l.n_heads;
    u32x4 *base = static_cast<u32x4 *>(l.p[blockIdx.y]) + head * l.head_stride + (column - head * l.chunks);
    constexpr int kRows = rows_at_once(BLOCK);
    // Long lists stream past the caches (plain stores 182 us, plain loads too 187,
    // all with 4 pieces).
    constexpr bool kLong = BLOCK > 256;
    bool ok = true;
    int64_t from[kRows], to[kRows];   // of the batch that begins at j0; to < 0: nothing moves
    const int32_t *table = a.table + s * a.table_stride;
    auto find = [&](int32_t j0) {
        // (every load stands without a condition, so that none waits for another)
        int32_t of[kRows], src[kRows], dst[kRows], src_page[kRows], dst_page[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int32_t j = j0 + i * ways + way;
            of[i] = keep[j < n ? j : 0];
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int32_t j = j0 + i * ways + way;
            const bool moves = used && j < n && of[i] != j;
            to[i] = moves ? 0 : -1;
            src[i] = (int32_t)start + (moves ? of[i] : 0);
            dst[i] = (int32_t)start + (moves ? j : 0);
            src_page[i] = (int32_t)((uint64_t)(uint32_t)src[i] * a.div_mul >> a.div_shift);
            dst_page[i] = (int32_t)((uint64_t)(uint32_t)dst[i] * a.div_mul >> a.div_shift);
            src[i] -= src_page[i] * l.page_size;
            dst[i] -= dst_page[i] * l.page_size;
            src_page[i] = table[src_page[i]];
            dst_page[i] = table[dst_page[i]];
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const bool there = src_page[i] >= 0 && src_page[i] < l.n_pages && dst_page[i] >= 0 && dst_page[i] < l.n_pages;
            ok &= there || to[i] < 0;
            from[i] = src_page[i] * l.page_stride + src[i] * l.slot_stride;
            to[i] = there && to[i] == 0 ? dst_page[i] * l.page_stride + dst[i] * l.slot_stride : -1;
        }
    };
    if (n > 0) find(0);
    for (int32_t j0 = 0; j0 < n; j0 += kRows * ways) {
        u32x4 x[kRows];
        int64_t now[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            now[i] = to[i];
            if (now[i] >= 0) x[i] = kLong ? __builtin_nontemporal_load(base + from[i]) : base[from[i]];
        }
        if (j0 + kRows * ways < n) find(j0 + kRows * ways);   // (places of the next, while these are on their way)
        // All of the batch is read when the first of it is written; what
        // the next one reads is not written here, so nobody waits for stores.
#pragma unroll
        for (int i = 0; i < kRows; ++i) asm volatile("" : "+v"(x[i]));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (now[i] >= 0) {
                if constexpr (kLong)
                    __builtin_nontemporal_store(x[i], base + now[i]);
                else
                    base[now[i]] = x[i];
            }
    }
    if (a.status && blockIdx.y == 0 && blockIdx.z == 0) {
        if (!ok) atomicOr(&s_bad, DSIM_ST_BAD_PAGE);
        __syncthreads();
        if (threadIdx.x == 0) a.status[s] = s_bad | (n < want || start < 0 ? DSIM_ST_BAD_POSITION : 0);
    }
}

}  // namespace

dsim_status launch_compact(const Layers &l, const CompactArgs &args, hipStream_t s)
{
    CompactArgs a = args;
    // ceil(2^(31 + k) / n), k = ceil(log2 n): t / n = t * mul >> shift for t < 2^31
    int k = 0;
    while ((1 << k) < l.page_size) ++k;
    a.div_shift = 31 + k;
    a.div_mul = (uint32_t)((((uint64_t)1 << a.div_shift) + l.page_size - 1) / l.page_size);
    const int64_t columns = (int64_t)l.n_heads * l.chunks;
    const int block = a.keep_width > 64 ? 512 : 256;
    // as many columns as leave enough ways for the list at once, 128 bytes at least,
    // shared out evenly (of 9 pieces of 16 bytes 5 and 4)
    int64_t per = (int64_t)block * rows_at_once(block) / (a.keep_width > 0 ? a.keep_width : 1);
    per = per < 8 ? 8 : per > block ? block : per;
    if (per > columns) per = columns;
    const int64_t parts = (columns + per - 1) / per;
    per = (columns + parts - 1) / parts;
    const dim3 grid(a.n_seq, 2 * l.n, (unsigned)parts);
    if (block == 512)
        hipLaunchKernelGGL((k_compact<512>), grid, dim3(512), 0, s, l, a, (int)per);
    else
        hipLaunchKernelGGL((k_compact<256>), grid, dim3(256), 0, s, l, a, (int)per);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "compact launch");
}

}  // namespace dsim
