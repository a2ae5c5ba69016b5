// kv_compact.hip -- kept tokens of a sequence move to its front
// (dsim_kv_compact).
//
// Bound by memory: each kept row is read and written once.  A place that is
// written may be one that another kept token still has to be read from, but
// never one that a later token of the ascending list comes from (the list's
// j-th entry is at least j), so a workgroup that takes its share of every row
// in the list's order, and reads a batch before it writes it, needs no second
// copy.  Its share is a piece of one layer's keys or values of one head.
#include "multi_ops.h"
#include "numeric.h"

namespace dsim {
namespace {

constexpr int kBlock = 256;
constexpr int kRows = 8;   // pieces of 16 bytes that a thread has in flight

__device__ inline int64_t place(const Layers &l, const CompactArgs &a, int32_t s, int64_t at, bool &ok)
{
    const int64_t page = a.table[s * a.table_stride + at / l.page_size];
    ok &= page >= 0 && page < l.n_pages;
    return page * l.page_stride + at % l.page_size * l.slot_stride;
}

// blockIdx.x: sequence; y: layer's keys or values; z: head and piece of its rows
__global__ __launch_bounds__(kBlock) void k_compact(Layers l, CompactArgs a, int pieces, int per_row, bool tells)
{
    __shared__ int32_t s_n, s_bad;
    const int32_t s = blockIdx.x;
    const int head = blockIdx.z / pieces, piece = blockIdx.z - head * pieces;
    const int64_t start = a.start[s], room = (int64_t)a.table_width * l.page_size;
    const int32_t *keep = a.keep + s * a.keep_stride;
    const int32_t want = min(max(a.n_keep[s], 0), a.keep_width);
    if (threadIdx.x == 0) {
        s_n = start < 0 ? 0 : want;
        s_bad = 0;
    }
    __syncthreads();
    // the list ends before the first entry that does not ascend or has no place
    for (int32_t j = threadIdx.x; j < want; j += kBlock) {
        const int32_t k = keep[j];
        if (k < 0 || (j > 0 && k <= keep[j - 1]) || start + k >= room) {
            atomicMin(&s_n, j);
            break;
        }
    }
    __syncthreads();
    const int32_t n = s_n;
    const int chunk = threadIdx.x % per_row + piece * per_row, way = threadIdx.x / per_row, ways = kBlock / per_row;
    const bool used = way < ways && chunk < l.chunks;
    u32x4 *base = static_cast<u32x4 *>(l.p[blockIdx.y]) + head * l.head_stride + chunk;
    bool ok = true;
    for (int32_t j0 = 0; j0 < n; j0 += kRows * ways) {
        u32x4 x[kRows];
        int64_t to[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int32_t j = j0 + i * ways + way;
            to[i] = -1;
            if (!used || j >= n || keep[j] == j) continue;
            bool there = true;
            const int64_t from = place(l, a, s, start + keep[j], there);
            const int64_t dst = place(l, a, s, start + j, there);
            ok &= there;
            if (!there) continue;
            to[i] = dst;
            x[i] = base[from];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (to[i] >= 0) base[to[i]] = x[i];
    }
    if (tells && a.status && blockIdx.y == 0 && blockIdx.z == 0) {
        if (!ok) atomicOr(&s_bad, DSIM_ST_BAD_PAGE);
        __syncthreads();
        if (threadIdx.x == 0) a.status[s] = s_bad | (n < want || start < 0 ? DSIM_ST_BAD_POSITION : 0);
    }
}

}  // namespace

dsim_status launch_compact(const Layers &l, const CompactArgs &a, hipStream_t s)
{
    const int pieces = (l.chunks + 7) / 8, per_row = (l.chunks + pieces - 1) / pieces;
    hipLaunchKernelGGL(k_compact, dim3(a.n_seq, 2 * l.n, l.n_heads * pieces), dim3(kBlock), 0, s, l, a, pieces, per_row,
                       a.status != nullptr);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "compact launch");
}

}  // namespace dsim
