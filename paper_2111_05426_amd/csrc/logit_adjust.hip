// logit_adjust.hip -- penalties for repeated tokens, biases and grammar masks
// on logits (dsim_logit_adjust).
#include "numeric.h"
#include "ops.h"

namespace dsim {
namespace {

constexpr int kBlock = 512;
constexpr int kSlice = 8192;          // tokens of one row per workgroup

constexpr uint32_t kPrompt = 1u << 31;

// One workgroup takes kSlice tokens of one row: it counts the history's
// tokens that lie there in shared memory (whole numbers, so their order does
// not matter), then passes over the slice once.
template <class T> __global__ __launch_bounds__(kBlock) void k_logits(dsim_logits a, int32_t slices)
{
    __shared__ uint32_t s_count[kSlice];
    __shared__ int32_t s_bias[kSlice];
    const int64_t b = blockIdx.x / slices;
    const int32_t lo = (int32_t)(blockIdx.x % slices) * kSlice, n = min(kSlice, a.vocab - lo), tid = threadIdx.x;
    const bool counting = a.history != nullptr, biased = a.n_bias > 0;
    if (counting)
        for (int i = tid; i < kSlice; i += kBlock) s_count[i] = 0;
    if (biased)
        for (int i = tid; i < kSlice; i += kBlock) s_bias[i] = -1;
    __syncthreads();
    if (counting) {
        const int32_t len = min(max(a.history_len[b], 0), a.history_width);
        const int32_t prompt = a.prompt_len ? min(max(a.prompt_len[b], 0), len) : 0;
        const int32_t *h = a.history + b * a.history_stride;
        for (int i = tid; i < len; i += kBlock) {
            const uint32_t at = (uint32_t)h[i] - (uint32_t)lo;
            if (h[i] >= 0 && at < (uint32_t)n) {
                if (i < prompt)
                    atomicOr(&s_count[at], kPrompt);
                else
                    atomicAdd(&s_count[at], 1u);
            }
        }
    }
    if (biased)
        for (int i = tid; i < a.n_bias; i += kBlock) {
            const int32_t id = a.bias_id[b * a.n_bias + i];
            const uint32_t at = (uint32_t)id - (uint32_t)lo;
            if (id >= 0 && at < (uint32_t)n) atomicMax(&s_bias[at], i);
        }
    __syncthreads();
    const float rep = a.repetition ? a.repetition[b] : 1.0f, freq = a.frequency ? a.frequency[b] : 0.0f,
                pres = a.presence ? a.presence[b] : 0.0f;
    const T *in = static_cast<const T *>(a.logits) + b * a.logits_stride + lo;
    T *out = static_cast<T *>(a.out) + b * a.out_stride + lo;
    for (int i = tid; i < n; i += kBlock) {
        float x = (float)in[i];
        if (counting) {
            const uint32_t c = s_count[i];
            if (c) {
                x = x > 0.0f ? x / rep : x * rep;
                const uint32_t made = c & ~kPrompt;
                x = x - (freq * (float)made + (made ? pres : 0.0f));
            }
        }
        if (biased && s_bias[i] >= 0) x = x + a.bias[b * a.n_bias + s_bias[i]];
        if (a.mask && !(a.mask[b * a.mask_stride + (lo + i) / 32] >> ((lo + i) % 32) & 1)) x = -HUGE_VALF;
        out[i] = (T)x;
    }
}

}  // namespace

dsim_status launch_logits(const dsim_logits &a, hipStream_t s)
{
    const int32_t slices = (a.vocab + kSlice - 1) / kSlice;
    const int64_t blocks = a.n_rows * slices;
    if (blocks >= ((int64_t)1 << 32) / kBlock) return fail(DSIM_ERANGE, "logits: n_rows * vocab is too large for one call");
    const dim3 grid((unsigned)blocks), block(kBlock);
    if (a.dtype == DSIM_F32)
        hipLaunchKernelGGL(k_logits<float>, grid, block, 0, s, a, slices);
    else if (a.dtype == DSIM_F16)
        hipLaunchKernelGGL(k_logits<f16>, grid, block, 0, s, a, slices);
    else
        hipLaunchKernelGGL(k_logits<bf16>, grid, block, 0, s, a, slices);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DSIM_OK : hip_fail(e, "logits launch");
}

}  // namespace dsim
