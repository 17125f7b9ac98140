// Pieces shared by the operators around int8 Dense layers whose scales are real numbers taken at run time (rows_scaled.hip,
// gemm_scaled.hip, gemm_scaled_rows.hip) and those that bring float rows into a cache (rotary.hip): element types, activations, rounding.
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

// x Phi(x) = max(x, 0) - |x| Phi(-|x|).  log2 Phi(-z) is smooth and falls without end: a polynomial of degree 8, fitted on z = 0 .. 6 for
// the smallest error of z Phi(-z), which is 6e-8 in 32 bits and at most 2 units of the 24th bit of x (beyond z = 6 the term is below
// 6e-9 and the polynomial goes on falling).  16 instruction slots, and vector instructions bound the layers with this activation.  Of
// itself the result has 2e-4 at x = -4, 0.6 % at -6 and half at -8: gelu_tail is for where that counts.
__device__ __forceinline__ float gelu_erf(float x) {
    const float z = __builtin_fabsf(x);
    float p = -1.2805152209693915e-06f;
    p = __builtin_fmaf(p, z, 2.0718478481285274e-05f);
    p = __builtin_fmaf(p, z, -9.715531632537022e-05f);
    p = __builtin_fmaf(p, z, -0.0003534583083819598f);
    p = __builtin_fmaf(p, z, 0.00734937796369195f);
    p = __builtin_fmaf(p, z, -0.05269759148359299f);
    p = __builtin_fmaf(p, z, -0.4591396450996399f);
    p = __builtin_fmaf(p, z, -1.1511139869689941f);
    p = __builtin_fmaf(p, z, -0.9999998211860657f);
    // (+inf: the second term is 0; -inf: NaN, as x Phi(x) and the other forms here give, so that an overflow does not pass for a 0)
    return __builtin_fmaxf(x, 0.0f) - __builtin_fabsf(__builtin_fminf(x, 0x1p100f)) * __builtin_amdgcn_exp2f(p);
}

// The same with the tail to 24 bits.  Phi(-z) = t Q(t) exp(-z^2 / 2) with t = 1 / (1 + 0.305 z): the quotient of the two is smooth, and a
// polynomial Q of degree 7 fitted on z = 0 .. 13.3 (beyond, the term is below 2^-126) has it to 1e-7 of itself.  In 32 bits the result is
// within (12 + x^2) 2^-24 of itself, x^2 from the argument of the power.  23 slots: for every GELU, 20000 x 1536 rows of hidden values took
// 33.3 us for 26.5 and a Dense layer of 8192 x 8192 x 4096 257 for 247.
__device__ __forceinline__ float gelu_tail(float x) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(x), 0.305f, 1.0f));
    float q = 0.03669919818639755f;
    q = __builtin_fmaf(q, t, -0.15298832952976227f);
    q = __builtin_fmaf(q, t, 0.18571694195270538f);
    q = __builtin_fmaf(q, t, -0.03797685354948044f);
    q = __builtin_fmaf(q, t, 0.12102168798446655f);
    q = __builtin_fmaf(q, t, 0.10342086106538773f);
    q = __builtin_fmaf(q, t, 0.12246681749820709f);
    q = __builtin_fmaf(q, t, 0.12163973599672318f);
    const float phi = q * (t * __builtin_amdgcn_exp2f(x * x * -0.72134752044448170f));
    return __builtin_fmaxf(x, 0.0f) - __builtin_fabsf(__builtin_fminf(x, 0x1p100f)) * phi;      // (infinities as above)
}

// TAIL: GELU with its tail
template <int ACT, bool TAIL> __device__ __forceinline__ float activation(float x) {
    if (ACT == ACT_RELU) return x > 0.0f ? x : x != x ? x : 0.0f;
    if (ACT == ACT_SILU) return sigmoid_times(x, x);
    if (ACT == ACT_GELU) return TAIL ? gelu_tail(x) : gelu_erf(x);
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

// Ahead of and behind the loads of one of two branches that differ in the kind of load alone: the compiler would make one of them, of the
// ordinary kind.
__device__ __forceinline__ void keep_apart() { asm volatile("" ::: "memory"); }

// The nearest whole number (ties to even) of a b, |a b| < 2^22, in the low bits of the result: the sum with 1.5 2^23 has a unit
// of 1 in its last place, and the multiply-add rounds once.
constexpr float kRound = 12582912.0f;
__device__ __forceinline__ uint32_t round_bits(float a, float b) { return __float_as_uint(__builtin_fmaf(a, b, kRound)); }
// the low bytes of four words
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
}

constexpr uint32_t kNormal = 0x00800000u, kInf = 0x7f800000u;      // the bits of |v|, as unsigned numbers, are in the order of |v|; NaN comes last

// What a row's int8 form needs: the largest |v|, 127 / it in 32 bits, and the scale of a row whose v still lack `factor`.  A row of zeros (or
// whose factor leaves nothing of it) has the scale 0; a row with a NaN or an infinite value, or with one that the factor takes beyond the range,
// NaN; both count as rows with a largest of 0: zeros.
struct Quant { float top, inv, scale; };
__device__ __forceinline__ Quant quant_of(uint32_t top_bits, float factor) {
    const float top = __uint_as_float(top_bits);
    if (top_bits >= kInf) return Quant{0.0f, 0.0f, __uint_as_float(0x7fc00000u)};
    const float most = top * factor, scale = most / 127.0f;
    if (most > 0x1.fffffep127f) return Quant{0.0f, 0.0f, __uint_as_float(0x7fc00000u)};
    if (scale == 0.0f) return Quant{0.0f, 0.0f, 0.0f};
    return Quant{top, 127.0f / top, scale};
}

// q = round(127 v / top), ties to even, of the exact quotient.  v inv is within 127 units of 2^-24 of it, so a value whose v inv is not that near a
// tie is rounded as it stands, by one multiply-add.  Next to ties (half of the largest is one: 63.5) 64 bits decide: there the quotient is
// within 2^-45, a quotient of two 24-bit numbers that is no tie is 2^-32 from one at least, and adding and taking away 1.5 2^12 leaves it at a
// multiple of 2^-40, ties as they are.  Tiny rows, whose inv may not be finite, go the same way.
__device__ __forceinline__ int32_t nearest(float v, double up) { return (int32_t)__builtin_rint(__builtin_fma((double)v, up, 6144.0) - 6144.0); }
__device__ __forceinline__ void store_q(int8_t* p, const v8f& v, const Quant& q, int n) {
    uint32_t w[8];
    float far = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        w[e] = round_bits(v[e], q.inv);
        far = __builtin_fmaxf(far, __builtin_fabsf(__builtin_fmaf(v[e], q.inv, kRound - __uint_as_float(w[e]))));
    }
    if (__builtin_expect(far >= 0.5f - 0x1p-16f || q.top < 0x1p-100f, 0)) {
        const double up = q.top > 0.0f ? 127.0 / (double)q.top : 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = q.top > 0.0f ? (uint32_t)nearest(v[e], up) : 0u;
    }
    typedef uint32_t v2u __attribute__((ext_vector_type(2), aligned(1)));
    const v2u out = {pack4(w[0], w[1], w[2], w[3]), pack4(w[4], w[5], w[6], w[7])};
    if (n >= 8) { *reinterpret_cast<v2u*>(p) = out; return; }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) p[e] = (int8_t)(out[e >> 2] >> (8 * (e & 3)));
}

}  // namespace scaled
}  // namespace ivit
