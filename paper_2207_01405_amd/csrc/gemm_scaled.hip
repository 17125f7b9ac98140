// int8 x int8 -> int32 Dense on the gfx950 matrix cores with real scales and the epilogue of a float layer:
//   y[m][n] = act(s_x[m] s_w[n] sum_k x[m][k] w[n][k] + bias[n]) + r[m][n]
//
// The plain form: a wavefront computes 32 tokens x 32 channels straight from memory.  The weights are the MFMA "A" operand, so a lane
// holds channels 8 q + 4 g + r of token lane % 32 (q, r = 0 .. 3; g = lane / 32).
#include "regst_common.hpp"
#include "scaled_common.hpp"

namespace ivit {
namespace {

using namespace scaled;

__device__ __forceinline__ void store_one(void* y, int64_t at, int type, float v, float inv_step) {
    if (type == TYPE_BF16) static_cast<__bf16*>(y)[at] = (__bf16)v;
    else if (type == TYPE_F16) static_cast<_Float16*>(y)[at] = (_Float16)v;
    else if (type == TYPE_F32) static_cast<float*>(y)[at] = v;
    else static_cast<int8_t*>(y)[at] = (int8_t)clamp8((int32_t)__builtin_rintf(v * inv_step));
}
__device__ __forceinline__ float load_one(const void* p, int64_t at, int type) {
    return type == TYPE_BF16 ? (float)static_cast<const __bf16*>(p)[at] : type == TYPE_F16 ? (float)static_cast<const _Float16*>(p)[at]
                                                                                          : static_cast<const float*>(p)[at];
}

__global__ __launch_bounds__(256) void gemm_scaled_kernel(ScaledArgs P, uint32_t tiles_n, uint32_t tiles) {
    const int lane = threadIdx.x & 63, li = lane & 31, lg = lane >> 5;
    const uint32_t tile = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int64_t m = (int64_t)(tile / tiles_n) * 32 + li;
    const int n0 = (int)(tile % tiles_n) * 32, N = P.N, K = P.K;
    const int8_t* xp = P.x + min64(m, P.M - 1) * P.ldx;
    const int8_t* wp = P.w + (int64_t)min(n0 + li, N - 1) * K;
    v16i acc = {};
    for (int k = 16 * lg; k - 16 * lg < K; k += 32) {
        v4i a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
        if (k < K) {
            a = *reinterpret_cast<const v4i*>(wp + k);
            b = *reinterpret_cast<const v4i*>(xp + k);
        }
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
    if (m >= P.M) return;
    const float sx = P.x_scale[P.one_scale ? 0 : m], inv_step = P.y_type == TYPE_I8 ? 1.0f / P.y_step : 0.0f;
    with_activation(P.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int n = n0 + 8 * (e >> 2) + 4 * lg + (e & 3);
            if (n >= N) continue;
            float v = (float)acc[e] * (sx * P.w_scale[n]);
            if (P.bias) v += P.bias[n];
            v = activation<decltype(act)::value>(v);
            if (P.residual) v += load_one(P.residual, m * P.ld_res + n, P.y_type);
            store_one(P.y, m * P.ldy + n, P.y_type, v, inv_step);
        }
    });
}

}  // namespace

hipError_t launch_linear_scaled(hipStream_t s, const ScaledArgs& a) {
    if (a.M == 0) return hipSuccess;
    TraceScope trace(s, KIND_GEMM_SCALED, 2 * a.M * a.N * a.K,
                     a.M * a.K + (int64_t)a.N * a.K + a.M * a.N * element_bytes(a.y_type) * (a.residual ? 2 : 1));
    const int64_t tn = (a.N + 31) / 32, tiles = (a.M + 31) / 32 * tn, grid = (tiles + 3) / 4;
    if (tiles > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(gemm_scaled_kernel, dim3((unsigned)grid), dim3(256), 0, s, a, (uint32_t)tn, (uint32_t)tiles);
    return hipGetLastError();
}

}  // namespace ivit
