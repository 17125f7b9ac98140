// Pieces shared by the operators around int8 Dense layers whose scales are real numbers taken at run time (rows_scaled.hip,
// gemm_scaled.hip): element types, activations, rounding.
//
// Arithmetic is in 32-bit floating point throughout; int8 products are summed exactly in 32-bit integers.  A value is rounded to
// fewer bits once, where it is stored (round to nearest, ties to even).
#pragma once
#include <type_traits>

#include "ivit_kernels.hpp"

namespace ivit {
namespace scaled {

typedef float v8f __attribute__((ext_vector_type(8)));

// Activations.  exp is the hardware's base-2 power of x log2(e), divisions by 1 + exp are its reciprocal: each within a few units
// of the 24th bit; quotients below 2^-126 may come as 0.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float sigmoid_times(float x, float slope) { return x * __builtin_amdgcn_rcpf(1.0f + exp_of(-slope)); }

// x Phi(x) = x (1 - erfc(x / sqrt 2) / 2).  With z = |x| / sqrt 2, erfc(z) = exp(-z^2) erfcx(z), and erfcx is t P(t) of
// t = 1 / (1 + 0.44 z): P is of degree 7, fitted for the smallest relative error over z = 0 .. 10 (4.4e-7 in 32 bits, with no
// cancellation for negative x).
__device__ __forceinline__ float gelu_erf(float x) {
    const float z = __builtin_fabsf(x) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.44f, 1.0f));
    float p = 0.0712218164925265f;
    p = __builtin_fmaf(p, t, -0.27794108477127516f);
    p = __builtin_fmaf(p, t, 0.29667536290798585f);
    p = __builtin_fmaf(p, t, -0.020169272333122264f);
    p = __builtin_fmaf(p, t, 0.2158060273719711f);
    p = __builtin_fmaf(p, t, 0.21731550077073722f);
    p = __builtin_fmaf(p, t, 0.24887085499863532f);
    p = __builtin_fmaf(p, t, 0.24822097579955119f);
    const float half = 0.5f * t * p * exp_of(-z * z);
    return x * (x < 0.0f ? half : 1.0f - half);
}

template <int ACT> __device__ __forceinline__ float activation(float x) {
    if (ACT == ACT_RELU) return x > 0.0f ? x : x != x ? x : 0.0f;
    if (ACT == ACT_SILU) return sigmoid_times(x, x);
    if (ACT == ACT_GELU) return gelu_erf(x);
    if (ACT == ACT_GELU_TANH)                  // (1 + tanh a) / 2 = sigma(2 a), a = sqrt(2 / pi) (x + 0.044715 x^3)
        return sigmoid_times(x, x * __builtin_fmaf(x * x, 0.0713548162726f, 1.59576912160573f));
    if (ACT == ACT_GELU_SIGMOID) return sigmoid_times(x, 1.702f * x);
    return x;
}

// f(std::integral_constant<int, ACT>()) for the activation of a call
template <class F> __host__ __device__ __forceinline__ auto with_activation(int act, F&& f) {
    switch (act) {
        case ACT_RELU: return f(std::integral_constant<int, ACT_RELU>());
        case ACT_SILU: return f(std::integral_constant<int, ACT_SILU>());
        case ACT_GELU: return f(std::integral_constant<int, ACT_GELU>());
        case ACT_GELU_TANH: return f(std::integral_constant<int, ACT_GELU_TANH>());
        case ACT_GELU_SIGMOID: return f(std::integral_constant<int, ACT_GELU_SIGMOID>());
        default: return f(std::integral_constant<int, ACT_NONE>());
    }
}

// Eight consecutive elements at any address that one element of the type may have, as 32-bit values and back.
template <class T> struct Eight {
    typedef T at __attribute__((ext_vector_type(8)));
    typedef T mem __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};
template <class T> __device__ __forceinline__ v8f load8(const T* p) {
    typename Eight<T>::at v = *reinterpret_cast<const typename Eight<T>::mem*>(p);
    return __builtin_convertvector(v, v8f);
}
template <class T> __device__ __forceinline__ void store8(T* p, v8f v) {
    *reinterpret_cast<typename Eight<T>::mem*>(p) = __builtin_convertvector(v, typename Eight<T>::at);
}
// ... the first n < 8 of them; the others are 0
template <class T> __device__ __forceinline__ v8f load_some(const T* p, int n) {
    v8f v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) v[e] = (float)p[e];
    return v;
}
template <class T> __device__ __forceinline__ void store_some(T* p, v8f v, int n) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) p[e] = (T)v[e];
}

// The nearest whole number (ties to even) of a b, |a b| < 2^22, in the low bits of the result: the sum with 1.5 2^23 has a unit
// of 1 in its last place, and the multiply-add rounds once.
__device__ __forceinline__ uint32_t round_bits(float a, float b) { return __float_as_uint(__builtin_fmaf(a, b, 12582912.0f)); }
// the low bytes of four words
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
}

}  // namespace scaled
}  // namespace ivit
