// numeric.h -- element types of the operators' kernels: vectors, loads and
// conversions between them and fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsim {

using f16 = _Float16;
using bf16 = __bf16;
struct e4m3 {
    uint8_t bits;
};

template <class T, int N> struct Vec {
    typedef T type __attribute__((ext_vector_type(N)));
};
template <int N> struct Vec<e4m3, N> {
    typedef uint8_t type __attribute__((ext_vector_type(N)));
};
template <class T, int N> using vec = typename Vec<T, N>::type;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// N elements of T in fp32, exactly
template <class T, int N> __device__ inline vec<float, N> to_f32(vec<T, N> x)
{
    return __builtin_convertvector(x, vec<float, N>);
}

// fp32 to T, one rounding to nearest even; e4m3 saturates at +-448 and keeps NaN
template <class T, int N> __device__ inline vec<T, N> from_f32(vec<float, N> x)
{
    if constexpr (__is_same(T, e4m3)) {
        static_assert(N % 4 == 0, "whole words");
        vec<uint32_t, N / 4> w;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = x[i] != x[i] ? x[i] : __builtin_amdgcn_fmed3f(x[i], -448.0f, 448.0f);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            int p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
            p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], p, true);
            w[i] = (uint32_t)p;
        }
        return __builtin_bit_cast(vec<T, N>, w);
    } else {
        return __builtin_convertvector(x, vec<T, N>);
    }
}

}  // namespace dsim
