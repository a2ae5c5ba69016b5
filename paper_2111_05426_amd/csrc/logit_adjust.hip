// logit_adjust.hip -- penalties for repeated tokens, biases and grammar masks
// on logits (dsim_logit_adjust).
//
// A row is read once and written once; what a token's history says about it
// has to be looked up on the way.  A workgroup takes a slice of one row,
// counts the history's tokens that lie in it in shared memory (whole
// numbers: the order of the atomics does not matter) and passes over the
// slice, so the row's counts never reach memory.  Every workgroup of a row
// reads the whole history, from L2 after the first.
//
// On MI355X the kernel takes, for 512 rows of 50,257 in fp16, histories up to
// 1,024, 300 biases and a mask (108 MB) 30 us, 3.6 TB/s; for 64 rows of 131,072
// in bf16, histories up to 8,192, 16 biases and a mask (36 MB) 14.0; for one
// row 3.7 (calls one after another 33.7, 15.1 and 3.9).  Memory bounds
// the bare pass (18.6 us of the 30, 5.9 of the 14.0); the rest is a chain of
// short phases between barriers that the few workgroups of a CU hide only in
// part: counting 4 and 6 us, mask 2.5, biases 3.  (Penalties applied by the
// threads that hold the history's tokens, each token claimed once by an atomic
// bit, take 4 us more; one pass of shared memory for counts and biases
// together, and slices of 4,096, gain nothing.)
#include "numeric.h"
#include "ops.h"

namespace dsim {
namespace {

constexpr uint32_t kPrompt = 1u << 31, kMade = kPrompt - 1;

// N elements at any element's alignment
template <class T, int N> __device__ inline vec<T, N> load_any(const T *p)
{
    vec<T, N> x;
    __builtin_memcpy(&x, p, sizeof x);
    return x;
}
template <class T, int N> __device__ inline void store_any(T *p, vec<T, N> x) { __builtin_memcpy(p, &x, sizeof x); }

// tokens i .. i + 3 of n
__device__ inline void tokens(const int32_t *h, int32_t i, int32_t n, int32_t (&t)[4])
{
    if (i < n - 3) {
        const vec<int32_t, 4> v = load_any<int32_t, 4>(h + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = v[k];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = i < n - k ? h[i + k] : -1;
    }
}

// SLICE tokens per workgroup of BLOCK threads.  Every load that needs no
// other's result is on its way at once: the logits, the first tokens of the
// history (as many as its rows are wide, whatever the row's length) and the
// first biases; one wait for memory, not four in a row, is what a workgroup
// takes beside its share of the bandwidth.
template <class T, int SLICE, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_logits(dsim_logits a, int32_t slices, bool by_xcd)
{
    constexpr int N = 16 / sizeof(T), kLoads = SLICE / (N * BLOCK), kAhead = 1;
    static_assert(SLICE % (N * BLOCK) == 0, "whole vectors");
    // first the history's counts, then the biases' places
    __shared__ uint32_t s_of[SLICE];
    // workgroups go to the eight XCDs in turn
    const int32_t i = by_xcd ? blockIdx.x / 8 : blockIdx.x;
    const int64_t b = by_xcd ? (int64_t)(i / slices) * 8 + blockIdx.x % 8 : i / slices;
    if (b >= a.n_rows) return;
    const int tid = threadIdx.x;
    const T *in = static_cast<const T *>(a.logits) + b * a.logits_stride;
    T *out = static_cast<T *>(a.out) + b * a.out_stride;
    // slices begin at 16-byte aligned addresses, the first at or before the row
    const int32_t lo = (i % slices) * SLICE - (int32_t)((uintptr_t)in / sizeof(T) % N);
    const bool counting = a.history != nullptr, biased = a.n_bias > 0;

    vec<T, N> x[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int32_t t = lo + (j * BLOCK + tid) * N;
        if (t >= 0 && t + N <= a.vocab)
            x[j] = load_any<T, N>(in + t);
        else
#pragma unroll
            for (int k = 0; k < N; ++k) x[j][k] = t + k >= 0 && t + k < a.vocab ? in[t + k] : (T)0.0f;
    }
    const int32_t *h = a.history + b * a.history_stride;
    const int32_t *ids = a.bias_id + b * a.n_bias;
    int32_t token[kAhead][4], id = -1, len = 0, prompt = 0;
    float rep = 1.0f, freq = 0.0f, pres = 0.0f;
    if (counting) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) tokens(h, (i * BLOCK + tid) * 4, a.history_width, token[i]);
        len = min(max(a.history_len[b], 0), a.history_width);
        prompt = a.prompt_len ? min(max(a.prompt_len[b], 0), len) : 0;
        if (a.repetition) rep = a.repetition[b];
        if (a.frequency) freq = a.frequency[b];
        if (a.presence) pres = a.presence[b];
    }
    if (biased && tid < a.n_bias) id = ids[tid];
    // the mask's bits of a vector's tokens
    uint32_t bits[kLoads];
    if (a.mask) {
        const uint32_t *mask = a.mask + b * a.mask_stride;
        const int32_t last = (a.vocab - 1) / 32;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int32_t t = lo + (j * BLOCK + tid) * N, first = max(min(t, a.vocab - 1), 0);
            // (the second word is the one after the first unless `first`
            // begins a word: then no bit of it counts)
            const uint64_t w = (uint64_t)mask[min((first + 31) / 32, last)] << 32 | mask[first / 32];
            bits[j] = (uint32_t)(w >> (first % 32)) << (t < 0 ? -t : 0);
        }
    }

    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < SLICE / (4 * BLOCK); ++i) reinterpret_cast<u32x4 *>(s_of)[i * BLOCK + tid] = u32x4{0, 0, 0, 0};
    };
    // a token's place in the slice, if it has one
    auto place = [&](int32_t t, uint32_t &at) {
        at = (uint32_t)t - (uint32_t)lo;
        return t >= 0 && t < a.vocab && at < (uint32_t)SLICE;
    };
    float y[kLoads][N];   // (single registers: whole vectors get copied at every branch)
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int k = 0; k < N; ++k) y[j][k] = (float)x[j][k];

    if (counting) {
        clear();
        __syncthreads();
        auto count = [&](int i, int32_t t) {
            uint32_t at;
            if (i < len && place(t, at)) {
                if (i < prompt)
                    atomicOr(&s_of[at], kPrompt);
                else
                    atomicAdd(&s_of[at], 1u);
            }
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) count((i * BLOCK + tid) * 4 + k, token[i][k]);
#pragma unroll 4
        for (int i = (kAhead * BLOCK + tid) * 4; i < len; i += BLOCK * 4) {
            int32_t more[4];
            tokens(h, i, len, more);
#pragma unroll
            for (int k = 0; k < 4; ++k) count(i + k, more[k]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
#pragma unroll
            for (int q = 0; q < N / 4; ++q) {
                const u32x4 c4 = reinterpret_cast<const u32x4 *>(s_of + (j * BLOCK + tid) * N)[q];
                if ((c4[0] | c4[1] | c4[2] | c4[3]) == 0) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t made = c4[k] & kMade;
                    float v = y[j][4 * q + k];
                    if (c4[k]) {
                        v = v > 0.0f ? v / rep : v * rep;
                        v = v - (freq * (float)made + (made ? pres : 0.0f));
                    }
                    y[j][4 * q + k] = v;
                }
            }
    }
    if (biased) {
        if (counting) __syncthreads();
        clear();
        __syncthreads();
        uint32_t at;
        if (place(id, at)) atomicMax(&s_of[at], (uint32_t)tid + 1);
        for (int i = BLOCK + tid; i < a.n_bias; i += BLOCK)
            if (place(ids[i], at)) atomicMax(&s_of[at], (uint32_t)i + 1);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
#pragma unroll
            for (int q = 0; q < N / 4; ++q) {
                const u32x4 i4 = reinterpret_cast<const u32x4 *>(s_of + (j * BLOCK + tid) * N)[q];
                if ((i4[0] | i4[1] | i4[2] | i4[3]) == 0) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i4[k]) y[j][4 * q + k] = y[j][4 * q + k] + a.bias[b * a.n_bias + i4[k] - 1];
            }
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int32_t t = lo + (j * BLOCK + tid) * N;
        if (a.mask) {
#pragma unroll
            for (int k = 0; k < N; ++k) y[j][k] = bits[j] >> k & 1 ? y[j][k] : -HUGE_VALF;
        }
        vec<float, N> w;
#pragma unroll
        for (int k = 0; k < N; ++k) w[k] = y[j][k];
        const vec<T, N> z = from_f32<T, N>(w);
        if (t >= 0 && t + N <= a.vocab)
            store_any<T, N>(out + t, z);
        else
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (t + k >= 0 && t + k < a.vocab) out[t + k] = z[k];
    }
}

template <class T, int SLICE, int BLOCK> dsim_status launch(const dsim_logits &a, hipStream_t s)
{
    constexpr int N = 16 / sizeof(T);
    // a row may begin inside a vector
    const bool aligned = (uintptr_t)a.logits % 16 == 0 && (a.n_rows == 1 || a.logits_stride % N == 0);
    const int32_t slices = (int32_t)(((int64_t)a.vocab + (aligned ? 0 : N - 1) + SLICE - 1) / SLICE);
    // The slices of a row on one XCD, whose L2 its history and biases then enter
    // once, if that leaves none of the eight with much more to do: 128 rows of
    // 131,072, histories up to 8,192, 23.6 us (in order 25.5), 512 of 50,257
    // 29.9 (31.0); 9 rows 8.1 (7.9).
    const bool by_xcd = a.n_rows >= 16;
    const int64_t blocks = (by_xcd ? (a.n_rows + 7) / 8 * 8 : a.n_rows) * slices;
    if (blocks >= ((int64_t)1 << 32) / BLOCK) return fail(DSIM_ERANGE, "logits: n_rows * vocab is too large for one call");
    hipLaunchKernelGGL((k_logits<T, SLICE, BLOCK>), dim3((unsigned)blocks), dim3(BLOCK), 0, s, a, slices, by_xcd);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "logits launch");
}

// Few rows: slices small enough to give every CU one.  50,257 in fp16, 300
// biases, a mask: 1 row 5.4 us (with the large slices 6.7), 32 rows 6.5 (7.4),
// 128 rows 12.9 (12.3), 512 33.4 (30.3).  But a long history takes longer than
// the slice, and more threads read it sooner: large slices again, with 1,024
// threads, as many as find room at once.  50,257 in fp16, 16 biases, a mask: 1
// row with a history of 32,768 10.1 us (small slices 18.9), 32 rows 11.0
// (22.3), 16 with one of 4,096 6.7 (7.0), 64 (448 slices) with 8,192 in fp32
// 11.9 (512 threads 13.0).
template <class T> dsim_status launch(const dsim_logits &a, hipStream_t s)
{
    const int64_t large = a.n_rows * ((a.vocab + 8191) / 8192);
    if (large <= 512 && a.history && a.history_width >= 4096) return launch<T, 8192, 1024>(a, s);
    return large < 256 ? launch<T, 2048, 256>(a, s) : launch<T, 8192, 512>(a, s);
}

}  // namespace

dsim_status launch_logits(const dsim_logits &a, hipStream_t s)
{
    if (a.dtype == DSIM_F32) return launch<float>(a, s);
    if (a.dtype == DSIM_F16) return launch<f16>(a, s);
    return launch<bf16>(a, s);
}

}  // namespace dsim
