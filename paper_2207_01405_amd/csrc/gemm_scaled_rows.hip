// The Dense layer with real scales (see gemm_scaled.hip) for few rows: single tokens, batches of them, one image.
//
// Hardly a weight is used twice, so what bounds it is how fast the weights come in (16.8 MB of them, N = K = 4096, are 3.3 us at a
// copy's rate) and, below that, the latencies of a launch.  A workgroup of W wavefronts has 16 CT channels and 8 XT tokens; the
// wavefronts split K.  Each has D steps of 128 bytes of K in flight, direct loads of whole lines into LDS that no other wavefront reads, so
// nobody waits for anybody before the end; there the partial sums, integers, meet in LDS.  What the epilogue reads is requested first.
// Loads straight into the registers of the matrix instruction ask for 64 bytes of a row at a time and were slower (1 x 4096 x 4096 5.7
// against 5.1 us, 16 x 11008 x 4096 13.9 and 9.4).
#include "regst_common.hpp"
#include "scaled_common.hpp"

namespace ivit {
namespace {

using namespace scaled;
using namespace regst;

// four consecutive results of a row at element `at`, the first n of them
template <class T> __device__ __forceinline__ void store4(void* y, int64_t at, const float* v, int n) {
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    T* const p = static_cast<T*>(y) + at;
    if (n >= 4) { *reinterpret_cast<four*>(p) = four{(T)v[0], (T)v[1], (T)v[2], (T)v[3]}; return; }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < n) p[e] = (T)v[e];
}
// The bits of four consecutive elements, the first n of them, and their values: apart, so that nothing waits where they are requested.
template <class T> __device__ __forceinline__ v4i bits4(const void* r, int64_t at, int n) {
    const T* const p = static_cast<const T*>(r) + at;
    if constexpr (sizeof(T) == 4) {
        typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
        if (n >= 4) return __builtin_bit_cast(v4i, *reinterpret_cast<const four*>(p));
        v4i v = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) v[e] = __builtin_bit_cast(int, p[e]);
        return v;
    } else {
        typedef uint32_t two __attribute__((ext_vector_type(2), aligned(2)));
        if (n >= 4) {
            const two v = *reinterpret_cast<const two*>(p);
            return v4i{(int)v[0], (int)v[1], 0, 0};
        }
        uint32_t b[3] = {0, 0, 0};
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) b[e] = __builtin_bit_cast(uint16_t, p[e]);
        return v4i{(int)(b[0] | b[1] << 16), (int)b[2], 0, 0};
    }
}
__device__ __forceinline__ float value_of(v4i v, int e, int type) {
    if (type == TYPE_F32) return __builtin_bit_cast(float, (int)v[e]);
    const uint32_t h = (uint32_t)v[e >> 1] >> (16 * (e & 1));
    return type == TYPE_BF16 ? __builtin_bit_cast(float, h << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}

// XT: 8-row pieces of x (tokens / 8); a step is 128 bytes of K
template <int CT, int XT, int W, int D>
__global__ __launch_bounds__(64 * W) void gemm_scaled_rows_kernel(ScaledArgs P, int steps, int count, FastDiv cols) {
    constexpr int MT = (XT + 1) / 2, PER = 2 * CT + XT, STEP = PER * 1024, RING = D * STEP;
    __shared__ __align__(1024) int8_t lds[RING > CT * MT * 1024 ? W * RING : W * CT * MT * 1024];
    v4i (*part)[CT * MT][64] = reinterpret_cast<v4i (*)[CT * MT][64]>(lds);
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, lg = lane >> 4;
    uint32_t tn;
    const int64_t m0 = (int64_t)cols.divide(blockIdx.x, tn) * (8 * XT);
    const int n0 = (int)tn * 16 * CT, K = P.K, N = P.N;
    const int rows = (int)min64(P.M - m0, 8 * XT);
    const int first = wv * count, mine = min(count, steps - first);      // of this wavefront's steps
    const uint32_t own = lds_offset(lds) + wv * RING;
    const int8_t* const own_p = lds + wv * RING;
    const int8_t* const wg = uniform_ptr(P.w + (int64_t)n0 * K);
    const int8_t* const xg = uniform_ptr(P.x + m0 * P.ldx);
    const int lr = lane >> 3, lc = 16 * ((lane & 7) ^ lr);
    uint32_t wo[2 * CT], xo[XT];
#pragma unroll
    for (int i = 0; i < 2 * CT; ++i) wo[i] = (uint32_t)min(8 * i + lr, N - 1 - n0) * (uint32_t)K;
#pragma unroll
    for (int i = 0; i < XT; ++i) xo[i] = (uint32_t)min(8 * i + lr, rows - 1) * (uint32_t)P.ldx;
    // the 16 x 16 results that this wavefront finishes: channels n .. n + 3 of token m0 + row
    static_assert(CT * MT <= W && D <= 3, "a result a wavefront; the waits below");
    const int n = n0 + 16 * (wv / MT) + 4 * lg, row = 16 * (wv % MT) + li, left = wv < CT * MT && row < rows ? N - n : 0;
    v4i res = {}, ws = {}, bi = {};
    float xs = 0.0f;
    if (left > 0) {
        xs = P.x_scale[P.one_scale ? 0 : m0 + row];
        ws = bits4<float>(P.w_scale, n, left);
        if (P.bias) bi = bits4<float>(P.bias, n, left);
        if (P.residual) {
            const int64_t at = (m0 + row) * P.ld_res + n;
            res = P.y_type == TYPE_F32 ? bits4<float>(P.residual, at, left) : bits4<__bf16>(P.residual, at, left);
        }
    }
    auto request = [&](int i, int slot) __attribute__((always_inline)) {
        const uint32_t k = (uint32_t)min(128 * (first + i) + lc, K - 16);
#pragma unroll
        for (int j = 0; j < 2 * CT; ++j) dma16(wg, wo[j] + k, own + slot * STEP + j * 1024);
#pragma unroll
        for (int j = 0; j < XT; ++j) dma16(xg, xo[j] + k, own + slot * STEP + CT * 2048 + j * 1024);
    };
    v4i acc[CT][MT] = {};
    auto multiply = [&](int i, int slot) __attribute__((always_inline)) {
        const int8_t* const at = own_p + slot * STEP;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int pc = 16 * ((4 * h + lg) ^ (li & 7));
            const bool real = 128 * (first + i) + 64 * h + 16 * lg < K;
            v4i w[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                w[c] = *reinterpret_cast<const v4i*>(at + (16 * c + li) * 128 + pc);
                w[c] = real ? w[c] : v4i{0, 0, 0, 0};
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int row = 16 * m + (XT == 1 ? li & 7 : li);
                const v4i x = *reinterpret_cast<const v4i*>(at + CT * 2048 + row * 128 + pc);
#pragma unroll
                for (int c = 0; c < CT; ++c) acc[c][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[c], x, acc[c][m], 0, 0, 0);
            }
        }
    };
    if (mine > 0) {
#pragma unroll
        for (int i = 0; i < D; ++i)
            if (i < mine) request(i, i);
        int i = 0;
#pragma unroll 1
        for (; i + D < mine; ++i) {
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"((D - 1) * PER) : "memory");
            const int slot = i % D;
            multiply(i, slot);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            request(i + D, slot);
        }
#pragma unroll
        for (int d = D - 1; d >= 0; --d) {
            if (i >= mine) break;
            if (mine - 1 - i < d) continue;
            switch (d) {
                case 0: asm volatile("s_waitcnt vmcnt(%0)" : : "n"(0) : "memory"); break;
                case 1: asm volatile("s_waitcnt vmcnt(%0)" : : "n"(PER) : "memory"); break;
                default: asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * PER) : "memory"); break;
            }
            multiply(i, i % D);
            ++i;
        }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int m = 0; m < MT; ++m) part[wv][c * MT + m][lane] = acc[c][m];
    __syncthreads();

    if (left <= 0) return;
    v4i sum = part[0][wv][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) sum += part[w][wv][lane];
    float v[4];
    with_activation(P.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = __builtin_fmaf((float)sum[e] * value_of(ws, e, TYPE_F32), xs, value_of(bi, e, TYPE_F32));
            v[e] = P.y_type == TYPE_F32 ? activation<decltype(act)::value, true>(v[e]) : activation<decltype(act)::value, false>(v[e]);
        }
    });
    const int64_t at = (m0 + row) * P.ldy + n;
    if (P.y_type == TYPE_I8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)clamp8((int32_t)__builtin_rintf(v[e] * P.inv_step));     // (NaN: 0)
        store4<int8_t>(P.y, at, v, left);
        return;
    }
    if (P.residual) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += value_of(res, e, P.y_type);
    }
    if (P.y_type == TYPE_BF16) store4<__bf16>(P.y, at, v, left);
    else if (P.y_type == TYPE_F16) store4<_Float16>(P.y, at, v, left);
    else store4<float>(P.y, at, v, left);
}

template <int CT, int XT, int W, int D> hipError_t launch(hipStream_t s, const ScaledArgs& a) {
    const int steps = (a.K + 127) / 128, count = (steps + W - 1) / W;
    const int64_t tn = (a.N + 16 * CT - 1) / (16 * CT), tiles = (a.M + 8 * XT - 1) / (8 * XT) * tn;
    hipLaunchKernelGGL((gemm_scaled_rows_kernel<CT, XT, W, D>), dim3((unsigned)tiles), dim3(64 * W), 0, s, a, steps, count, FastDiv((uint32_t)tn));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_scaled_rows(hipStream_t s, const ScaledArgs& a) {
    // Eight wavefronts with two steps each in flight where half of the CUs have no tile: 1 x 1000 x 4096 3.6 -> 3.1 us, 8 x 1000 x 8192
    // 5.2 -> 4.7, 48 x 768 x 4096 4.2 -> 3.9; with a tile a CU nothing is gained (16 x 4096 x 4096 5.1 and 5.0), with several
    // they lose (1 x 11008 x 4096, 688 tiles, 9.0 and 9.4).
    const int64_t tn = ((int64_t)a.N + 15) / 16, tiles = (a.M + 31) / 32 * tn;
    const bool few = 2 * tiles <= num_cus();
    if (a.M <= 8) return few ? launch<1, 1, 8, 2>(s, a) : launch<1, 1, 4, 3>(s, a);
    if (a.M <= 16) return few ? launch<1, 2, 8, 2>(s, a) : launch<1, 2, 4, 3>(s, a);
    if (few) return launch<1, 4, 8, 2>(s, a);
    // 16 channels for 32 rows while one such tile a CU takes the shape, 32 channels beyond (197 x 384 x 1536, 168 tiles: 3.4 and 3.6 us;
    // 48 x 4096 x 4096, 512: 7.4 and 6.3)
    if (a.M <= 32 || tiles <= num_cus()) return launch<1, 4, 4, 3>(s, a);
    return launch<2, 4, 4, 2>(s, a);
}

}  // namespace ivit
