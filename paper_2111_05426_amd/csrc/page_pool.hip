// page_pool.hip -- the pages of a cache: dsim_kv_reserve, dsim_kv_release,
// dsim_kv_fork, dsim_kv_copy_pages.
//
// Who gets which page has to be the same on every run, so one workgroup deals:
// the rows' (or forks') needs are summed in order, the free pages are the set
// bits of a bitmap taken from its lowest word on, and page number r of the
// second goes to need number r of the first.  A bitmap of a million pages is
// 128 KB; counts that only go up or down by atomic additions need no order.
// What is bound by memory, copying and whole rows of the table, is spread over
// the GPU in a launch behind it.
//
// On MI355X a beam search's step over 128 rows (64 released, as many forked over
// 1 to 2,048 tokens with a half page of four layers each, a place reserved in
// each; 16 MB) takes 24.8 us in its calls' four launches: release 3.9, fork 7.2,
// copy 6.8, reserve 6.7, each a chain of three or four loads and the barriers of
// its sums.  A reserve for rows that hold pages in advance looks at those that the
// row grows into: 128 rows of 500 of them 22 us, 4 rows of 4,096 20.
#include "multi_ops.h"
#include "numeric.h"

namespace dsim {
namespace {

constexpr int kDeal = 1024;          // threads of the dealing workgroup
constexpr int kDealWaves = kDeal / 64;
constexpr int kWindow = 4096;        // pages that are dealt at once, in shared memory
constexpr int kCopy = 256;

// Sums over the workgroup: exclusive prefix of x and the total, both waves'
// and lanes'.  Two barriers; `s` holds kDealWaves numbers.
__device__ inline int64_t scan(int64_t x, int64_t *s, int64_t &total)
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
    for (int w = 0; w < kDealWaves; ++w) {
        if (w < wave) before += s[w];
        total += s[w];
    }
    __syncthreads();
    return before + incl - x;
}

__device__ inline int32_t load(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// the bits of word w that stand for free pages
__device__ inline uint32_t free_word(const dsim_page_pool &p, int64_t w)
{
    const int64_t rest = p.n_pages - 32 * w;
    return p.free[w] & (rest >= 32 ? ~0u : (1u << rest) - 1);
}

struct Need {
    int64_t pages;    // that are wanted
    int32_t status;
    bool skip;        // left alone
};

// Deals free pages to n takers in order.  take(i) is what i needs, got(i,
// status) is told once whether it gets it, put(i, j, page) where its j-th page
// is.  take must give the same until all is dealt.  All threads call it together,
// also for i >= n, who need nothing, and settle(i, need) behind a barrier: what the
// threads have to find together.
template <class Take, class Settle, class Got, class Put>
__device__ inline void deal(const dsim_page_pool &p, int64_t n, Take take, Settle settle, Got got, Put put)
{
    __shared__ int64_t s_sum[kDealWaves];
    __shared__ int32_t s_page[kWindow];
    const int tid = threadIdx.x;
    const int64_t words = (p.n_pages + 31) / 32;
    int64_t total, mine = 0;
    for (int64_t w = tid; w < words; w += kDeal) mine += __popc(free_word(p, w));
    // (what the first kDeal need is kept: it takes three loads in a row)
    Need mine_ = take(tid);
    scan(mine, s_sum, total);
    const int64_t avail = total;
    settle(tid, mine_);
    const auto later = [&](int64_t i) {
        Need x = take(i);
        __syncthreads();
        settle(i, x);
        return x;
    };

    int64_t before = 0, dealt = 0, at_ = 0;
    for (int64_t i0 = 0; i0 < n; i0 += kDeal) {
        const int64_t i = i0 + tid;
        const Need x = i0 == 0 ? mine_ : later(i);
        const int64_t at = before + scan(x.pages, s_sum, total);
        if (i0 == 0) at_ = at;
        const bool enough = x.pages == 0 || at + x.pages <= avail;
        if (i < n && !x.skip) got(i, x.status | (enough ? 0 : DSIM_ST_NO_PAGE));
        if (before + total <= avail) {
            dealt += total;
        } else {   // who gets theirs come first: the sum to the last of them is what is dealt
            int64_t sum;
            scan(x.pages > 0 && enough ? x.pages : 0, s_sum, sum);
            dealt += sum;
        }
        before += total;
    }
    for (int64_t r0 = 0; r0 < dealt; r0 += kWindow) {
        const int64_t r1 = min(r0 + kWindow, dealt);
        // free pages number r0 to r1 - 1 (those before are taken by now)
        int64_t rank = r0;
        for (int64_t w0 = 0; w0 < words && rank < r1; w0 += kDeal) {
            const int64_t w = w0 + tid;
            uint32_t bits = w < words ? free_word(p, w) : 0, taken = 0;
            int64_t r = rank + scan(__popc(bits), s_sum, total);
            for (; bits && r < r1; bits &= bits - 1, ++r) {
                const int bit = __ffs(bits) - 1;
                taken |= 1u << bit;
                s_page[r - r0] = (int32_t)(32 * w + bit);
                p.refs[32 * w + bit] = 1;
            }
            if (taken) p.free[w] &= ~taken;
            rank += total;
        }
        __syncthreads();
        before = 0;
        for (int64_t i0 = 0; i0 < n && before < r1; i0 += kDeal) {
            const int64_t i = i0 + tid;
            const Need x = i0 == 0 ? mine_ : later(i);
            int64_t at = at_;
            if (n > kDeal) at = before + scan(x.pages, s_sum, total);
            if (at + x.pages <= avail)
                for (int64_t r = max(at, r0); r < min(at + x.pages, r1); ++r) put(i, r - at, s_page[r - r0]);
            before += total;
        }
        __syncthreads();
    }
}

__device__ inline int64_t pages_of(int64_t places, int32_t page_size) { return (places + page_size - 1) / page_size; }

// Why a page of a row may not be written to, in bits.
__device__ inline int32_t unwritable(const dsim_page_pool &p, int32_t page)
{
    return page < 0 || page >= p.n_pages ? DSIM_ST_BAD_PAGE : p.refs[page] > 1 ? DSIM_ST_SHARED_PAGE : 0;
}

// Of entries first, first + step, ... below end of a row of the table, four at a
// time, all of them together.
__device__ inline int32_t unwritable(const dsim_page_pool &p, const int32_t *entries, int32_t first, int32_t end, int32_t step)
{
    constexpr int kAtOnce = 4;
    int32_t found = 0;
    for (int64_t j0 = first; j0 < end; j0 += kAtOnce * step) {
        int32_t page[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) page[k] = entries[min(j0 + k * step, (int64_t)end - 1)];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) found |= unwritable(p, page[k]);
    }
    return found;
}

__global__ __launch_bounds__(kDeal) void k_reserve(dsim_page_pool p, const int32_t *seq_len, const int32_t *new_len,
                                                   int32_t *status)
{
    // Rows grow into pages that they hold already, from that of place seq_len on.
    // Mostly that is one, in which a row's tokens end; of a row that went back, or
    // holds pages in advance, it may be thousands, and those are shared out among
    // the waves.
    constexpr int kAlone = 16;
    __shared__ int32_t s_much, s_first[kDeal], s_end[kDeal], s_found[kDeal];
    const auto told = [](int32_t found) { return found & DSIM_ST_BAD_PAGE ? DSIM_ST_BAD_PAGE : found; };
    const auto range = [&](int64_t s, int64_t want, int64_t len, int64_t held) {
        return make_int2((int32_t)len / p.page_size, (int32_t)min(held, pages_of(want, p.page_size)));
    };
    if (threadIdx.x == 0) s_much = 0;
    __syncthreads();
    auto take = [&](int64_t s) {
        Need x{0, 0, true};
        if (s >= p.n_seq) return x;
        const int64_t want = new_len[s], len = seq_len[s], held = p.held[s], pages = pages_of(want, p.page_size);
        x.skip = want < 0;
        if (x.skip) return x;
        if (pages > p.table_width || held < 0 || held > p.table_width || len < 0 || len > held * p.page_size) {
            x.status = DSIM_ST_BAD_POSITION;
        } else if (want > len) {
            const int2 grown = range(s, want, len, held);
            const int32_t *entries = p.block_table + s * p.table_stride;
            if (grown.y - grown.x > kAlone)
                s_much = 1;   // (stays so: settle looks for such rows)
            else if (grown.x < grown.y)
                x.status = told(unwritable(p, entries[grown.x]) | unwritable(p, entries, grown.x + 1, grown.y, 1));
        }
        if (!x.status && pages > held) x.pages = pages - held;
        return x;
    };
    auto settle = [&](int64_t s, Need &x) {
        if (s_much == 0) return;
        const int tid = threadIdx.x, lane = tid & 63;
        int2 grown = make_int2(0, 0);
        if (!x.skip && !x.status && new_len[s] > seq_len[s]) grown = range(s, new_len[s], seq_len[s], p.held[s]);
        const bool much = grown.y - grown.x > kAlone;
        s_first[tid] = grown.x;
        s_end[tid] = much ? grown.y : grown.x;
        __syncthreads();
        for (int t = tid >> 6; t < kDeal; t += kDealWaves) {
            const int32_t first = s_first[t], end = s_end[t];
            if (first == end) continue;
            int32_t found = 0;
            if (first + lane < end) found = unwritable(p, p.block_table + (s - tid + t) * p.table_stride, first + lane, end, 64);
            const bool bad = __builtin_amdgcn_ballot_w64(found & DSIM_ST_BAD_PAGE) != 0;
            const bool shared = __builtin_amdgcn_ballot_w64(found & DSIM_ST_SHARED_PAGE) != 0;
            if (lane == 0) s_found[t] = (bad ? DSIM_ST_BAD_PAGE : 0) | (shared ? DSIM_ST_SHARED_PAGE : 0);
        }
        __syncthreads();
        if (much && s_found[tid]) x = Need{0, told(s_found[tid]), false};
    };
    deal(p, p.n_seq, take, settle, [&](int64_t s, int32_t st) { status[s] = st; },
         [&](int64_t s, int64_t j, int32_t page) { p.block_table[s * p.table_stride + p.held[s] + j] = page; });
    for (int64_t s = threadIdx.x; s < p.n_seq; s += kDeal) {
        const int64_t want = new_len[s], more = pages_of(want, p.page_size) - p.held[s];
        if (want >= 0 && status[s] == 0 && more > 0) p.held[s] += (int32_t)more;
    }
}

// A workgroup a row.  Two entries of one row: each takes the pages between
// its length and what the other left.
__global__ __launch_bounds__(kCopy) void k_release(dsim_page_pool p, int64_t n, const int32_t *row, const int32_t *keep_len,
                                                   int32_t *status)
{
    __shared__ int32_t s_held, s_bad;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int32_t s = row[i];
        const int64_t keep = pages_of(max(keep_len[i], 0), p.page_size);
        __syncthreads();   // (the row before has read s_held)
        if (threadIdx.x == 0) {
            s_bad = s >= p.n_seq ? DSIM_ST_BAD_SEQUENCE : 0;
            s_held = s >= 0 && s < p.n_seq ? atomicMin(&p.held[s], (int32_t)min(keep, (int64_t)INT32_MAX)) : 0;
        }
        __syncthreads();
        const int64_t held = min(s_held, p.table_width);
        for (int64_t j = keep + threadIdx.x; j < held; j += kCopy) {
            int32_t *entry = p.block_table + s * p.table_stride + j;
            const int32_t page = *entry;
            *entry = -1;
            const int32_t refs = page >= 0 && page < p.n_pages ? atomicSub(&p.refs[page], 1) : 0;
            if (refs == 1)
                atomicOr(&p.free[page / 32], 1u << page % 32);
            else if (refs <= 0) {
                if (page >= 0 && page < p.n_pages) atomicAdd(&p.refs[page], 1);
                atomicOr(&s_bad, DSIM_ST_BAD_PAGE);
            }
        }
        __syncthreads();
        if (threadIdx.x == 0 && status) status[i] = s_bad;
    }
}

// The forks' rows are claimed by their number (below any count, the lowest
// wins), so that a row that two want, or one that is copied from, is known
// before anything of it changes.
__global__ __launch_bounds__(kDeal) void k_fork(dsim_page_pool p, int32_t *seq_len, int64_t n, const int32_t *src,
                                                const int32_t *dst, int32_t *status)
{
    auto claim = [](int64_t i) { return (int32_t)(i - ((int64_t)1 << 31)); };
    for (int64_t i = threadIdx.x; i < n; i += kDeal) {
        const int32_t d = dst[i];
        if (d >= 0 && d < p.n_seq && load(&p.held[d]) <= 0) atomicMin(&p.held[d], claim(i));
    }
    __syncthreads();
    auto take = [&](int64_t i) {
        Need x{0, 0, i >= n};
        if (i >= n) return x;
        const int32_t d = dst[i], s = src[i];
        if (d < 0) return x;
        if (d >= p.n_seq || s < 0 || s >= p.n_seq) {
            x.status = DSIM_ST_BAD_SEQUENCE;
        } else if (load(&p.held[d]) != claim(i)) {
            x.status = DSIM_ST_IN_USE;
        } else {
            const int64_t held = load(&p.held[s]), len = seq_len[s];
            if (held < 0)
                x.status = DSIM_ST_BAD_SEQUENCE;
            else if (held > p.table_width || len < 0 || len > held * p.page_size)
                x.status = DSIM_ST_BAD_POSITION;
            else
                x.pages = len % p.page_size != 0;
        }
        return x;
    };
    deal(p, n, take, [](int64_t, Need &) {}, [&](int64_t i, int32_t st) { status[i] = st; },
         [&](int64_t i, int64_t, int32_t page) {
             p.block_table[dst[i] * p.table_stride + seq_len[src[i]] / p.page_size] = page;
         });
    __syncthreads();
    // (a row that is copied from is nobody's dst: what is read here is not written here)
    for (int64_t i = threadIdx.x; i < n; i += kDeal) {
        const int32_t d = dst[i];
        if (d < 0 || d >= p.n_seq || load(&p.held[d]) != claim(i)) continue;
        const bool done = status[i] == 0;
        if (done) seq_len[d] = seq_len[src[i]];
        __hip_atomic_store(&p.held[d], done ? (int32_t)pages_of(seq_len[src[i]], p.page_size) : 0, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    }
}

// `slots` first places of a page of every layer; blockIdx.y: which cache's
// keys or values; blockIdx.z of gridDim.z parts.
__device__ inline void copy_slots(const Layers &l, int which, int64_t from, int64_t to, int32_t slots)
{
    const u32x4 *src = static_cast<const u32x4 *>(l.p[which]) + from * l.page_stride;
    u32x4 *dst = static_cast<u32x4 *>(l.p[which]) + to * l.page_stride;
    const int64_t n = (int64_t)l.n_heads * slots * l.chunks, step = (int64_t)kCopy * gridDim.z;
    const bool heads_inside = l.head_stride < l.slot_stride;   // the nearer of the two runs faster
    const uint32_t inner = heads_inside ? l.n_heads : slots;
    constexpr int kAhead = 4;
    for (int64_t i0 = blockIdx.z * (int64_t)kCopy + threadIdx.x; i0 < n; i0 += kAhead * step) {
        u32x4 x[kAhead];
        int64_t at[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t i = i0 + k * step;
            if (i >= n) continue;
            const uint32_t row = (uint32_t)(i / l.chunks), c = (uint32_t)(i - (int64_t)row * l.chunks);
            const uint32_t a = row / inner, b = row - a * inner;
            at[k] = (heads_inside ? b : a) * l.head_stride + (heads_inside ? a : b) * l.slot_stride + c;
            x[k] = src[at[k]];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i0 + k * step < n) dst[at[k]] = x[k];
    }
}

// blockIdx.y 0 (of the first launch): the row of the table; the others: a
// layer's keys or values each.
__global__ __launch_bounds__(kCopy) void k_fork_copy(Layers l, dsim_page_pool p, const int32_t *seq_len, int64_t n,
                                                     const int32_t *src, const int32_t *dst, int32_t *status, bool first)
{
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int32_t d = dst[i], s = src[i];
        if (d < 0 || (load(&status[i]) & ~DSIM_ST_BAD_PAGE)) continue;
        const int32_t len = seq_len[d], whole = len / p.page_size, rest = len % p.page_size;
        const int32_t *from = p.block_table + s * p.table_stride;
        int32_t *to = p.block_table + d * p.table_stride;
        if (first && blockIdx.y == 0) {
            for (int32_t j = blockIdx.z * kCopy + threadIdx.x; j < whole + (rest > 0); j += kCopy * gridDim.z) {
                const int32_t page = from[j];
                const bool ok = page >= 0 && page < p.n_pages;
                if (!ok) atomicOr(&status[i], DSIM_ST_BAD_PAGE);
                if (j == whole) continue;
                to[j] = ok ? page : -1;
                if (ok) atomicAdd(&p.refs[page], 1);
            }
        } else if (rest > 0) {
            const int32_t a = from[whole], b = to[whole];
            if (a >= 0 && a < p.n_pages && b >= 0 && b < p.n_pages) copy_slots(l, blockIdx.y - first, a, b, rest);
        }
    }
}

__global__ __launch_bounds__(kCopy) void k_copy_pages(Layers l, int64_t n, const int32_t *src, const int32_t *dst)
{
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int32_t a = src[i], b = dst[i];
        if (a < 0 || b < 0 || a >= l.n_pages || b >= l.n_pages || a == b) continue;
        copy_slots(l, blockIdx.y, a, b, l.page_size);
    }
}

dsim_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, what);
}

// parts of a page's copy: about 32 KB each
unsigned parts(const Layers &l)
{
    const int64_t bytes = (int64_t)l.n_heads * l.page_size * l.chunks * 16, n = (bytes + 32767) / 32768;
    return (unsigned)(n < 1 ? 1 : n > 64 ? 64 : n);
}

unsigned workgroups(int64_t n, int64_t most) { return (unsigned)(n < most ? n : most); }

}  // namespace

dsim_status launch_reserve(const dsim_page_pool &p, const int32_t *seq_len, const int32_t *new_len, int32_t *status,
                           hipStream_t s)
{
    hipLaunchKernelGGL(k_reserve, dim3(1), dim3(kDeal), 0, s, p, seq_len, new_len, status);
    return launched("reserve launch");
}

dsim_status launch_release(const dsim_page_pool &p, int64_t n, const int32_t *row, const int32_t *keep_len,
                           int32_t *status, hipStream_t s)
{
    hipLaunchKernelGGL(k_release, dim3(workgroups(n, 1 << 16)), dim3(kCopy), 0, s, p, n, row, keep_len, status);
    return launched("release launch");
}

dsim_status launch_fork(const Layers *layers, int n_launches, const dsim_page_pool &p, int32_t *seq_len, int64_t n,
                        const int32_t *src, const int32_t *dst, int32_t *status, hipStream_t s)
{
    hipLaunchKernelGGL(k_fork, dim3(1), dim3(kDeal), 0, s, p, seq_len, n, src, dst, status);
    dsim_status st = launched("fork launch");
    for (int i = 0; i < n_launches && !st; ++i) {
        const Layers &l = layers[i];
        hipLaunchKernelGGL(k_fork_copy, dim3(workgroups(n, 1 << 16), 2 * l.n + (i == 0), parts(l)), dim3(kCopy), 0, s, l, p,
                           seq_len, n, src, dst, status, i == 0);
        st = launched("fork copy launch");
    }
    return st;
}

dsim_status launch_copy_pages(const Layers &l, int64_t n, const int32_t *src, const int32_t *dst, hipStream_t s)
{
    hipLaunchKernelGGL(k_copy_pages, dim3(workgroups(n, 1 << 16), 2 * l.n, parts(l)), dim3(kCopy), 0, s, l, n, src, dst);
    return launched("page copy launch");
}

}  // namespace dsim
