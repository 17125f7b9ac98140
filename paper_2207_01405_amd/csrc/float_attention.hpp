// Pieces shared by the attention kernels over float rows (prompt_attention.hip, cached_attention.hip).
//
// Matrix instruction 32 x 32 x 16 of 16-bit elements: lane l holds row l % 32 of an operand, elements 8 (l / 32) .. + 8 of the 16; of the result
// column l % 32 and, in register r, row 8 (r / 4) + 4 (l / 32) + r % 4.
#pragma once
#include "ivit_kernels.hpp"

namespace ivit {
namespace fatt {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

template <class T> struct Elem {
    typedef T v8 __attribute__((ext_vector_type(8)));
    typedef T v2 __attribute__((ext_vector_type(2)));
    // Weights are at most 2^8 times the largest (see softmax_step).  float16 ends at 2^-24 below: there they are 2^7 times larger throughout.
    static constexpr float kUp = __is_same(T, _Float16) ? 7.0f : 0.0f;
};
__device__ __forceinline__ v16f mfma(Elem<__bf16>::v8 a, Elem<__bf16>::v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v16f mfma(Elem<_Float16>::v8 a, Elem<_Float16>::v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
// c + a[0] + a[1]
__device__ __forceinline__ float add_pair(Elem<__bf16>::v2 a, float c) { return __builtin_amdgcn_fdot2_f32_bf16(a, Elem<__bf16>::v2{(__bf16)1.0f, (__bf16)1.0f}, c, false); }
__device__ __forceinline__ float add_pair(Elem<_Float16>::v2 a, float c) { return __builtin_amdgcn_fdot2(a, Elem<_Float16>::v2{(_Float16)1.0f, (_Float16)1.0f}, c, false); }

// The largest of three, NaN if one is (the other kind of maximum would quiet the operands first, an instruction a score)
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
// The larger of a lane's value and that of its place in the other half of the wavefront; their sum
__device__ __forceinline__ float max_halves(float x) {
    const v2u r = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
    const v2u r = __builtin_bit_cast(v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The largest of a lane's 16 N scores and of the other half's.
template <int N> __device__ __forceinline__ float largest_of(const v16f (&s)[N]) {
    float a = max3(s[0][0], s[0][1], s[0][2]), b = max3(s[0][3], s[0][4], s[0][5]);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = i ? 0 : 6; r < 16; r += 4) {
            a = max3(a, s[i][r], s[i][r + 1]);
            if (r + 2 < 16) b = max3(b, s[i][r + 2], s[i][r + 3]);
        }
    return max_halves(__builtin_elementwise_maximum(a, b));
}

// The 16-byte pieces of a key's row are stored at piece ^ mix(row), so that reads of many rows are spread over the banks: for keys 16 lanes read the
// same piece of 16 rows, for values 32 lanes read 64 bytes of four rows (4 n .. 4 n + 3).
template <int D> __device__ __forceinline__ int mix_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D> __device__ __forceinline__ int mix_v(int row) { return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); }

// The fragment of values for the keys of registers 8 t .. 8 t + 7 of a lane's scores, k0 = 16 t: keys k0 + 4 half + 0 .. 3 and k0 + 8 + 4 half + 0 .. 3 of
// dimension 32 i + lane % 32.  The transposing read takes 4 rows x 16 elements from 16 lanes, 8 bytes each, and gives a lane one column.
template <int D> __device__ __forceinline__ int transposed_at(int i, int lane) {              // where its first row's bytes are, of k0 = 0
    const int row = 4 * (lane >> 5) + ((lane >> 2) & 3), col = 32 * i + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    return row * 2 * D + 16 * ((col >> 3) ^ mix_v<D>(row)) + 2 * (col & 7);
}
template <class T, int D> __device__ __forceinline__ typename Elem<T>::v8 transposed(const int8_t* p) {
    typedef v4s __attribute__((address_space(3)))* at;
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(p + 8 * 2 * D));      // (mix_v(row + 8) is mix_v(row))
    return __builtin_bit_cast(typename Elem<T>::v8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// One step of the softmax of a lane's query over 32 KB scores (both halves of the wavefront hold one query's): the weights of the scores, rounded and
// packed, and their sum; maximum, sum and output brought along.  The maximum that the weights stand against is moved only where a score exceeds it by
// more than 2^8 in weight: the output's 16 DT registers are rescaled a few times in all then, not at every step, and no weight exceeds 2^8.
template <int DT> __device__ __forceinline__ void move_largest(float top, float& m, float& l, v16f (&acc)[DT], float c) {
    if (__builtin_expect(__any((top - m) * c > 8.0f), 0)) {             // (m = -infinity to begin with; -infinity less -infinity is NaN and not more)
        const float to = __builtin_fmaxf(top, m), f = to > m ? __builtin_amdgcn_exp2f((m - to) * c) : 1.0f;
        m = to;
        l *= f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] *= f;
    }
}
// what the exponents of the weights start from
template <class T> __device__ __forceinline__ float base_of(float m, float c) { return Elem<T>::kUp - (m == -__builtin_inff() ? 0.0f : m * c); }
// weights r and r + 1 of a lane's 16 scores
template <class T> __device__ __forceinline__ void weigh(const v16f& s, int r, typename Elem<T>::v8 (&p)[2], float& l, float c, float base) {
    const v2f w = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, base)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], c, base))};
    const typename Elem<T>::v2 q = __builtin_convertvector(w, typename Elem<T>::v2);
    l = add_pair(q, l);
    p[r / 8][r % 8] = q[0];
    p[r / 8][r % 8 + 1] = q[1];
}
template <class T, int KB, int DT>
__device__ __forceinline__ void softmax_step(const v16f (&s)[KB], typename Elem<T>::v8 (&p)[KB][2], float& m, float& l, v16f (&acc)[DT], float c) {
    move_largest<DT>(largest_of(s), m, l, acc, c);
    const float base = base_of<T>(m, c);
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 2) weigh<T>(s[b], r, p[b], l, c, base);
}

// The same over 16 scores, for values of int8 rows: what leaves are weights times the values' scales, in float16 and in units of 2^(ref - 15), as the output is; the sum
// is that of the weights alone.  ref is a query's own and goes by the largest product so far, not by the largest scale (a key of next to no weight and large
// values would push those that count below float16's numbers): products of less than 2^ref are less than 2^15, the largest is 2^7 at least when ref is set, so a product is off by
// 2^-11 of itself or by 2^-32 of the largest.  ref falls as the weights do that a new largest score leaves to what came before.
constexpr float kRefLeast = -110.0f;                                    // (2^(15 - ref) and 2^(ref - 15) are normal numbers; ref starts here)
template <int DT>
__device__ __forceinline__ void softmax_step_scaled(const v16f (&s)[1], Elem<_Float16>::v8 (&p)[2], float& m, float& l, v16f (&acc)[DT], float c, float& ref,
                                                    const float (&scale)[16]) {
    const float top = largest_of(s);
    const bool moves = (top - m) * c > 8.0f;                            // (as in move_largest)
    const float down = moves ? (m - top) * c : 0.0f;                    // what came before is to be multiplied by 2^down
    m = moves ? top : m;
    l *= __builtin_amdgcn_exp2f(down);
    const float base = m == -__builtin_inff() ? 0.0f : -(m * c);
    float t[16], largest = 0x1p-118f;                                   // (a NaN among them leaves the others)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][r], c, base));
        l += w;
        t[r] = w * scale[r];
        largest = __builtin_fmaxf(largest, t[r]);
    }
    const float most = __builtin_fminf(max_halves(largest), 0x1p121f);
    const float power = (float)__builtin_amdgcn_frexp_expf(most);       // products are less than 2^power
    if (__builtin_expect(__any(moves || power > ref), 0)) {
        const float to = moves || power > ref ? __builtin_fmaxf(power + 7.0f, __builtin_floorf(ref + down)) : ref;
        const float f = __builtin_amdgcn_exp2f(down + (ref - to));
        ref = to;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] *= f;
    }
    const float unit = __builtin_amdgcn_exp2f(15.0f - ref);
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r / 8][r % 8] = (_Float16)(t[r] * unit);
}

template <int DT> __device__ __forceinline__ bool not_finite(const v16f (&acc)[DT]) {
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) z = __builtin_fmaf(acc[i][r], 0.0f, z);
    return z != z;
}

// The state of a lane's query after those of the keys first .. last that count, one key after the other, from memory.
template <class T, int D, class Counts>
__device__ __forceinline__ void key_by_key(const T* q, const T* k, int64_t ldk, const T* v, int64_t ldv, int first, int last, float c, int half, float& m,
                                           float& l, v16f (&acc)[D / 32], Counts&& counts) {
    auto score = [&](int j) __attribute__((always_inline)) {
        const T* const kj = k + j * ldk;
        float sum = 0.0f;
#pragma unroll 1
        for (int e = 0; e < D; ++e) sum = __builtin_fmaf((float)q[e], (float)kj[e], sum);
        return sum;
    };
    m = -__builtin_inff();
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] = v16f{};
#pragma unroll 1
    for (int j = first; j <= last; ++j)
        if (counts(j)) m = __builtin_fmaxf(m, score(j));
    const float base = Elem<T>::kUp - (m == -__builtin_inff() ? 0.0f : m * c);
#pragma unroll 1
    for (int j = first; j <= last; ++j) {
        if (!counts(j)) continue;
        const float w = (float)(T)__builtin_amdgcn_exp2f(__builtin_fmaf(score(j), c, base));
        const T* const vj = v + j * ldv + 4 * half;
        l += half ? 0.0f : w;                                           // (the halves' sums are added in the end)
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] = __builtin_fmaf(w, (float)vj[32 * i + 8 * (r / 4) + r % 4], acc[i][r]);
    }
}

// A query's row of 32 DT elements from a lane's registers, 8 bytes a store (for few rows).
template <class T, int DT> __device__ __forceinline__ void store_rows(T* o, const v16f (&acc)[DT], float inv, int half) {
    typedef T v4 __attribute__((ext_vector_type(4)));
    typedef float v4f __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const v4f f = {acc[i][4 * g] * inv, acc[i][4 * g + 1] * inv, acc[i][4 * g + 2] * inv, acc[i][4 * g + 3] * inv};
            *reinterpret_cast<v4*>(o + 32 * i + 8 * g + 4 * half) = __builtin_convertvector(f, v4);
        }
}

}  // namespace fatt
}  // namespace ivit
