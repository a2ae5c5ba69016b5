// logit_adjust.hip -- penalties for repeated tokens, biases and grammar masks
// on logits (dsim_logit_adjust).
//
// A row is read once and written once; what a token's history says about it
// has to be looked up on the way.  A workgroup takes a slice of one row,
// counts the history's tokens that lie in it in shared memory (whole
// numbers: the order of the atomics does not matter) and passes over the
// slice, so the row's counts never reach memory.  Every workgroup of a row
// reads the whole history, from L2 after the first.
#include "numeric.h"
#include "ops.h"

namespace dsim {
namespace {

constexpr uint32_t kPrompt = 1u << 31, kBiased = 1u << 30, kMade = kBiased - 1;

// N elements at any element's alignment
template <class T, int N> __device__ inline vec<T, N> load_any(const T *p)
{
    vec<T, N> x;
    __builtin_memcpy(&x, p, sizeof x);
    return x;
}
template <class T, int N> __device__ inline void store_any(T *p, vec<T, N> x) { __builtin_memcpy(p, &x, sizeof x); }

// SLICE tokens per workgroup of BLOCK threads.
template <class T, int SLICE, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_logits(dsim_logits a, int32_t slices)
{
    constexpr int N = 16 / sizeof(T), kLoads = SLICE / (N * BLOCK);
    static_assert(SLICE % (N * BLOCK) == 0, "whole vectors");
    extern __shared__ uint32_t s_mem[];
    uint32_t *s_count = s_mem;                                  // generated tokens, kPrompt, kBiased
    int32_t *s_bias = reinterpret_cast<int32_t *>(s_mem + SLICE);   // the last bias of a token that has one
    const int64_t b = blockIdx.x / slices;
    const int tid = threadIdx.x;
    const T *in = static_cast<const T *>(a.logits) + b * a.logits_stride;
    T *out = static_cast<T *>(a.out) + b * a.out_stride;
    // slices begin at 16-byte aligned addresses, the first at or before the row
    const int32_t lo = (int32_t)(blockIdx.x % slices) * SLICE - (int32_t)((uintptr_t)in / sizeof(T) % N);
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
    if (counting || biased) {
#pragma unroll
        for (int i = 0; i < SLICE / (4 * BLOCK); ++i)
            reinterpret_cast<u32x4 *>(s_count)[i * BLOCK + tid] = u32x4{0, 0, 0, 0};
        __syncthreads();
        if (counting) {
            const int32_t len = min(max(a.history_len[b], 0), a.history_width);
            const int32_t prompt = a.prompt_len ? min(max(a.prompt_len[b], 0), len) : 0;
            const int32_t *h = a.history + b * a.history_stride;
#pragma unroll 4
            for (int i = tid; i < len; i += BLOCK) {
                const int32_t id = h[i];
                const uint32_t at = (uint32_t)id - (uint32_t)lo;
                if (id >= 0 && id < a.vocab && at < (uint32_t)SLICE) {
                    if (i < prompt)
                        atomicOr(&s_count[at], kPrompt);
                    else
                        atomicAdd(&s_count[at], 1u);
                }
            }
        }
        if (biased) {
            const int32_t *ids = a.bias_id + b * a.n_bias;
            for (int i = tid; i < a.n_bias; i += BLOCK) {
                const uint32_t at = (uint32_t)ids[i] - (uint32_t)lo;
                if (ids[i] >= 0 && ids[i] < a.vocab && at < (uint32_t)SLICE) {
                    atomicOr(&s_count[at], kBiased);
                    s_bias[at] = -1;
                }
            }
            __syncthreads();
            for (int i = tid; i < a.n_bias; i += BLOCK) {
                const uint32_t at = (uint32_t)ids[i] - (uint32_t)lo;
                if (ids[i] >= 0 && ids[i] < a.vocab && at < (uint32_t)SLICE) atomicMax(&s_bias[at], i);
            }
        }
        __syncthreads();
    }
    const float rep = a.repetition ? a.repetition[b] : 1.0f, freq = a.frequency ? a.frequency[b] : 0.0f,
                pres = a.presence ? a.presence[b] : 0.0f;
    const uint32_t *mask = a.mask ? a.mask + b * a.mask_stride : nullptr;
    const int32_t last = (a.vocab - 1) / 32;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int i = (j * BLOCK + tid) * N;
        const int32_t t = lo + i;
        if (t + N <= 0 || t >= a.vocab) continue;
        vec<float, N> y = to_f32<T, N>(x[j]);
        if (counting || biased) {
#pragma unroll
            for (int q = 0; q < N / 4; ++q) {
                const u32x4 c4 = reinterpret_cast<const u32x4 *>(s_count + i)[q];
                if ((c4[0] | c4[1] | c4[2] | c4[3]) == 0) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t c = c4[k], made = c & kMade;
                    float v = y[4 * q + k];
                    if (c & ~kBiased) {
                        v = v > 0.0f ? v / rep : v * rep;
                        v = v - (freq * (float)made + (made ? pres : 0.0f));
                    }
                    if (c & kBiased) v = v + a.bias[b * a.n_bias + s_bias[i + 4 * q + k]];
                    y[4 * q + k] = v;
                }
            }
        }
        if (mask) {
            const int32_t first = max(t, 0);
            const uint64_t w = (uint64_t)mask[min((first + 31) / 32, last)] << 32 | mask[first / 32];
            // bits of tokens first.., the second word being the one after the
            // first unless `first` begins a word (then no bit of it counts)
            const uint32_t bits = (uint32_t)(w >> (first % 32)) << (first - t);
#pragma unroll
            for (int k = 0; k < N; ++k) y[k] = bits >> k & 1 ? y[k] : -HUGE_VALF;
        }
        const vec<T, N> z = from_f32<T, N>(y);
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
    const int32_t slices = (int32_t)(((int64_t)a.vocab + N - 1 + SLICE - 1) / SLICE);   // (a row may begin inside a vector)
    const int64_t blocks = a.n_rows * slices;
    if (blocks >= ((int64_t)1 << 32) / BLOCK) return fail(DSIM_ERANGE, "logits: n_rows * vocab is too large for one call");
    const size_t shared = (size_t)SLICE * 4 * (a.n_bias > 0 ? 2 : 1);
    hipLaunchKernelGGL((k_logits<T, SLICE, BLOCK>), dim3((unsigned)blocks), dim3(BLOCK), shared, s, a, slices);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "logits launch");
}

// Few rows: slices small enough to give every CU one.
template <class T> dsim_status launch(const dsim_logits &a, hipStream_t s)
{
    return a.n_rows * ((a.vocab + 8191) / 8192) < 256 ? launch<T, 2048, 256>(a, s) : launch<T, 8192, 512>(a, s);
}

}  // namespace

dsim_status launch_logits(const dsim_logits &a, hipStream_t s)
{
    if (a.dtype == DSIM_F32) return launch<float>(a, s);
    if (a.dtype == DSIM_F16) return launch<f16>(a, s);
    return launch<bf16>(a, s);
}

}  // namespace dsim
