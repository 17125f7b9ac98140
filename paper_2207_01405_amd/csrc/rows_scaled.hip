// Rows that leave as int8 values with a scale each: the root-mean-square norm with the residual's addition in front, and the
// (gated) activation of an MLP's hidden rows.
//
//   norm:  h = x + r,  n = h / sqrt(mean(h^2) + eps) gamma        gate:  v = act(g) u  or  act(g)
//   s = max |v| / 127,  q = round(v / s)
//
// A group of TPR threads holds a row in registers, NV pieces of eight elements a thread, so that x is read once; one reduction over the group
// gives the norm its sum of squares and its largest |h gamma| together: the factor 1 / sqrt(..) is the same for a row's elements, so q
// needs h gamma only and s takes the factor once.
//
// Norms are bound by memory, 5 to 7 bytes an element for some 14 instruction slots: 16384 x 4096 bf16 with a residual 85 us (5.5 TB/s), 25216 x 384
// 15.5 (4.4).  Gated by SiLU 8192 x 14336 take 100 (5.9), memory too; GELU alone is bound by vector instructions as well, about 24 slots an element
// for 3 bytes: 20000 x 1536 bf16 23 us, of which 21 are issue and 18 the bytes; 8192 x 14336 gated by it 117.  Results go through the caches, since
// the product after them reads them: stored past the L2 the norm gets faster (when chosen: 16384 x 4096 82 us, 25216 x 768 23.5 for 28.6)
// and what follows slower by more (norm, Dense 768 -> 2048, activation and Dense 2048 -> 768 of 50432 rows 355 for 338).
#include "scaled_common.hpp"

namespace ivit {
namespace {

using namespace scaled;

template <int TPR, int BLOCK> struct Group {
    static constexpr int ROWS = BLOCK / TPR, WAVES = TPR > 64 ? TPR / 64 : 1;
    static_assert(TPR <= 64 || TPR == BLOCK, "a row of several wavefronts is the workgroup's");
    // what all threads of a row agree on and is hardly ever true, as a branch of the wavefront where it has one row only: what is live on the way
    // not taken needs no registers then
    static __device__ __forceinline__ bool agreed(bool b) { return __builtin_expect(TPR >= 64 ? __builtin_amdgcn_readfirstlane(b) : b, 0); }
    // one(a, b) of a value and the largest of the bits over the threads of a row, every one of them getting both.  AGAIN: a call for the same
    // rows was before it.
    template <bool AGAIN, class One> static __device__ __forceinline__ void reduce(float& value, uint32_t& top, One&& one) {
#pragma unroll
        for (int m = (TPR < 64 ? TPR : 64) / 2; m > 0; m >>= 1) {
            value = one(value, __shfl_xor(value, m));
            top = max(top, (uint32_t)__shfl_xor((int)top, m));
        }
        if constexpr (TPR > 64) {
            __shared__ float s[WAVES];
            __shared__ uint32_t t[WAVES];
            if (AGAIN) __syncthreads();
            if ((threadIdx.x & 63) == 0) { s[threadIdx.x >> 6] = value; t[threadIdx.x >> 6] = top; }
            __syncthreads();
            value = s[0]; top = t[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                value = one(value, s[w]); top = max(top, t[w]);
                if (w % 8 == 7) __builtin_amdgcn_sched_barrier(0);      // (sixteen wavefronts' at once would be 32 registers)
            }
        }
    }
    // The largest of the bits alone; and whether a wavefront of the row (for short rows: the row) had a thread whose `wide` is more than eight
    // times the largest there.  If the row's largest is that small against a `wide` of the row, it is so.
    static __device__ __forceinline__ bool largest(uint32_t& top, float wide) {
#pragma unroll
        for (int m = (TPR < 64 ? TPR : 64) / 2; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        uint64_t small = __ballot(8.0f * __uint_as_float(top) < wide);
        if constexpr (TPR < 64) small &= ((1ull << TPR) - 1) << (threadIdx.x & 63 & ~(TPR - 1));
        if constexpr (TPR > 64) {
            __shared__ uint32_t t[WAVES], any[WAVES];
            if ((threadIdx.x & 63) == 0) { t[threadIdx.x >> 6] = top; any[threadIdx.x >> 6] = small != 0; }
            __syncthreads();
            top = t[0];
            uint32_t a = any[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) { top = max(top, t[w]); a |= any[w]; }
            return a != 0;
        }
        return small != 0;
    }
};

// Piece v of thread t starts at element 8 (t + TPR v).  One that would run over the end of the row starts eight elements before the
// end instead: its first `twice` elements are also in the piece before, where they count; results that both hold are stored twice,
// with the same value.  So no load waits for a branch.  (All loads of a row have returned before its first store: behind the
// reduction, and behind the barrier in it.  A row may be written where it was read.)
struct Piece { int at, twice; };
__device__ __forceinline__ Piece piece_of(int i, int C) {
    const int c = 8 * i, at = min(c, C - 8);
    return Piece{at, c - at};
}

struct NormParams {
    const void* x; const void* r; const float* gamma; void* sum; void* y; float* scale;
    int64_t ldx, ldr, ld_sum, ldy, rows; int C; float eps;
};

// A row whose sum of squares, or whose largest |h gamma|, is beyond the range of 32 bits or below the normal numbers, while its n need not be: the
// sum again of h 2^-64, if it is infinite, and products of h factor, which is at most sqrt(C), with gamma.  All threads of the row come here, with the
// same sum, and read it anew, element by element, each its own ones: hardly a row is like this, and the kernel needs no register for it.
template <class T, int TPR, int BLOCK, bool I8>
__device__ __forceinline__ void far_row(const NormParams& P, int64_t row, bool real, float sum) {
    using G = Group<TPR, BLOCK>;
    const int t = threadIdx.x % TPR, C = P.C;
    const T* const x = static_cast<const T*>(P.x) + row * P.ldx;
    const T* const r = static_cast<const T*>(P.r) + row * P.ldr;
    auto input = [&](int c) __attribute__((always_inline)) { return P.r ? (float)x[c] + (float)r[c] : (float)x[c]; };
    auto gamma = [&](int c) __attribute__((always_inline)) { return P.gamma ? P.gamma[c] : 1.0f; };
    auto add = [](float a, float b) __attribute__((always_inline)) { return a + b; };
    uint32_t top = 0;
    float factor = 1.0f / __builtin_sqrtf(sum / (float)C + P.eps);
    if (G::agreed(sum == __builtin_inff())) {
        sum = 0.0f;
#pragma unroll 1
        for (int c = t; c < C; c += TPR) {
            const float h = input(c) * 0x1p-64f;
            sum = __builtin_fmaf(h, h, sum);
        }
        G::template reduce<true>(sum, top, add);
        const float mean = sum / (float)C + P.eps * 0x1p-64f * 0x1p-64f;
        factor = mean < 1.0f ? 0x1p-64f / __builtin_sqrtf(mean) : 0.0f;        // (a mean square beyond the range counts as infinite)
    }
    Quant q = {};
    if (I8) {
        top = 0;
#pragma unroll 1
        for (int c = t; c < C; c += TPR) top = max(top, __float_as_uint(input(c) * factor * gamma(c)) & 0x7fffffffu);
        G::template reduce<true>(sum, top, add);
        q = quant_of(top, 1.0f);
        if (real && t == 0) P.scale[row] = q.scale;
    }
    if (!real) return;
    const double up = q.top > 0.0f ? 127.0 / (double)q.top : 0.0;
#pragma unroll 1
    for (int c = t; c < C; c += TPR) {
        const float h = input(c), n = h * factor * gamma(c);
        if (P.sum) static_cast<T*>(P.sum)[row * P.ld_sum + c] = (T)h;
        if (I8) static_cast<int8_t*>(P.y)[row * P.ldy + c] = q.top > 0.0f ? (int8_t)nearest(n, up) : (int8_t)0;
        else static_cast<T*>(P.y)[row * P.ldy + c] = (T)n;
    }
}

// SHORT: fewer than eight elements a row (TPR = 8, NV = 1): the first thread takes them one by one
template <class T, int NV, int TPR, int BLOCK, bool I8, bool SHORT>
__global__ __launch_bounds__(BLOCK) void rmsnorm_kernel(NormParams P) {
    using G = Group<TPR, BLOCK>;
    const int t = threadIdx.x % TPR, C = P.C;
    const int64_t mine = (int64_t)blockIdx.x * G::ROWS + threadIdx.x / TPR, row = min64(mine, P.rows - 1);
    const T* const x = static_cast<const T*>(P.x) + row * P.ldx;
    const T* const r = static_cast<const T*>(P.r) + row * P.ldr;
    v8f h[NV], g[NV];
    Piece p[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        p[v] = SHORT ? Piece{0, t ? 8 : 0} : piece_of(t + TPR * v, C);
        h[v] = SHORT ? load_some(x, C) : load8(x + p[v].at);
    }
    if (P.r) {
#pragma unroll
        for (int v = 0; v < NV; ++v) h[v] += SHORT ? load_some(r, C) : load8(r + p[v].at);
    }
    if (P.gamma) {
#pragma unroll
        for (int v = 0; v < NV; ++v) g[v] = SHORT ? load_some(P.gamma, C) : load8(P.gamma + p[v].at);
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) g[v] = v8f{1, 1, 1, 1, 1, 1, 1, 1};
    }
    float sum = 0.0f;
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (p[v].twice == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(h[v][e], h[v][e], sum);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= p[v].twice) sum = __builtin_fmaf(h[v][e], h[v][e], sum);
        }
        if (I8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(h[v][e] * g[v][e]) & 0x7fffffffu);
        }
    }
    G::template reduce<false>(sum, top, [](float a, float b) __attribute__((always_inline)) { return a + b; });
    // (rows of zeros go on, and with them rows whose squares and products with gamma are all 0 in 32 bits)
    if (G::agreed(sum == __builtin_inff() || (I8 && top - kNormal >= kInf - kNormal && (top | __float_as_uint(sum)))))
        return far_row<T, TPR, BLOCK, I8>(P, row, mine < P.rows, sum);
    const float factor = 1.0f / __builtin_sqrtf(sum / (float)C + P.eps);
    const Quant q = quant_of(top, factor);
    if (mine >= P.rows) return;
    if (I8 && t == 0) P.scale[row] = q.scale;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (p[v].twice >= 8) continue;
        const int n = SHORT ? C : 8;
        if (P.sum) {
            T* s = static_cast<T*>(P.sum) + row * P.ld_sum + p[v].at;
            if (SHORT) store_some(s, h[v], n); else store8(s, h[v]);
        }
        if (I8) {
            store_q(static_cast<int8_t*>(P.y) + row * P.ldy + p[v].at, h[v] * g[v], q, n);
        } else {                                              // (h factor is at most sqrt(C), a product of h and gamma may be beyond the range)
            T* y = static_cast<T*>(P.y) + row * P.ldy + p[v].at;
            if (SHORT) store_some(y, h[v] * factor * g[v], n); else store8(y, h[v] * factor * g[v]);
        }
    }
}

// (one instruction; of __builtin_fminf and __builtin_fmaxf on values that come from memory the compiler makes two for each)
__device__ __forceinline__ float min3(float a, float b, float c) {
    float m;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
    float m;
    asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

struct GateParams { const void* x; int8_t* y; float* scale; int64_t ldx, ldy, rows; int C, act, once; };

template <class T, int NV, int TPR, int BLOCK, bool GATED, bool SHORT>
__global__ __launch_bounds__(BLOCK) void gated_kernel(GateParams P) {
    using G = Group<TPR, BLOCK>;
    using Raw = typename Eight<T>::at;
    using Mem = typename Eight<T>::mem;
    const int t = threadIdx.x % TPR, C = P.C;
    const int64_t mine = (int64_t)blockIdx.x * G::ROWS + threadIdx.x / TPR, row = min64(mine, P.rows - 1);
    const T* const x = static_cast<const T*>(P.x) + row * P.ldx;
    Raw a[NV], b[NV];
    Piece p[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) p[v] = SHORT ? Piece{0, t ? 8 : 0} : piece_of(t + TPR * v, C);
    if (SHORT) {
        a[0] = __builtin_convertvector(load_some(x, C), Raw);
        if (GATED) b[0] = __builtin_convertvector(load_some(x + C, C), Raw);
    } else if (P.once) {
        keep_apart();
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            a[v] = __builtin_nontemporal_load(reinterpret_cast<const Mem*>(x + p[v].at));
            if (GATED) b[v] = __builtin_nontemporal_load(reinterpret_cast<const Mem*>(x + C + p[v].at));
        }
        keep_apart();
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            a[v] = *reinterpret_cast<const Mem*>(x + p[v].at);
            if (GATED) b[v] = *reinterpret_cast<const Mem*>(x + C + p[v].at);
        }
    }
    v8f h[NV];
    // GELU falls so fast below 0 that a row's largest value can be far smaller than what goes into it.  gelu_erf is within 2^-23 |x|: where the largest
    // is below an eighth of `wide`, the most that |x| |u| with x < 0 can be, the row is formed again by gelu_tail, from x anew (the
    // registers that would hold it until then are worth more).  In all others the values are within 2^-20 of the largest.
    float wide = 0.0f;
    uint32_t top = 0;
    auto form = [&](auto act, auto tail_c) __attribute__((always_inline)) {
        constexpr bool TAIL = decltype(tail_c)::value, WIDE = !TAIL && decltype(act)::value == ACT_GELU;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const v8f f = __builtin_convertvector(a[v], v8f);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[v][e] = activation<decltype(act)::value, TAIL>(f[e]);
            float low = 0.0f, by = GATED ? 0.0f : 1.0f;
            if (WIDE) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) low = min3(low, f[e], f[e + 1]);
            }
            if (GATED) {
                const v8f u = __builtin_convertvector(b[v], v8f);
                h[v] *= u;
                if (WIDE) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) by = max3_abs(by, u[e], u[e + 1]);
                }
            }
            if (WIDE) wide = __builtin_fmaxf(wide, -low * by);
        }
        top = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(h[v][e]) & 0x7fffffffu);
    };
    with_activation(P.act, [&](auto act) __attribute__((always_inline)) { form(act, std::false_type()); });
    if (G::agreed(G::largest(top, wide))) {
        auto more = [](float a, float b) __attribute__((always_inline)) { return __builtin_fmaxf(a, b); };
        G::template reduce<false>(wide, top, more);
        if (G::agreed(8.0f * __uint_as_float(top) < wide)) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                a[v] = SHORT ? __builtin_convertvector(load_some(x, C), Raw) : *reinterpret_cast<const Mem*>(x + p[v].at);
                if (GATED) b[v] = SHORT ? __builtin_convertvector(load_some(x + C, C), Raw) : *reinterpret_cast<const Mem*>(x + C + p[v].at);
            }
            form(std::integral_constant<int, ACT_GELU>(), std::true_type());
            G::template reduce<true>(wide, top, more);
        }
    }
    const Quant q = quant_of(top, 1.0f);
    if (mine >= P.rows) return;
    if (t == 0) P.scale[row] = q.scale;
#pragma unroll
    for (int v = 0; v < NV; ++v)
        if (p[v].twice < 8) store_q(P.y + row * P.ldy + p[v].at, h[v], q, SHORT ? C : 8);
}

// f(NV, TPR, BLOCK, SHORT) for rows of C elements.  Many rows: as few threads a row as hold it in up to three pieces each, so that hardly
// a thread is idle, and a workgroup for every wavefront (bf16 norms with a residual, us: 25216 x 384 15.7, with four wavefronts a
// workgroup 16.5; 25216 x 768 29.3, with 256 threads a row 51.0; 20000 x 1536, activation alone, 24.0 and 34.1); from 1537 to 2048 elements 256 threads
// have one piece each (10000 x 2048 30.6, with 128 threads of two 33.3); up to three pieces of 128 threads then, against two of 256:
// activation alone 10000 x 2304 21.7 and 26.9, x 3000 23.5 and 29.2, gated 22.3 and 26.0, 26.9 and 27.3, norms 36.4 and 35.8, 44.9 and 43.7,
// without a residual, to float16, 5003 x 2049 10.8 and 11.4, 10000 x 3000 26.1 and 26.3.  Few rows, where a launch is a chain of
// latencies: 256 threads from 513 elements on (197 x 1536, activation alone, 3.2 and 3.5; 300 x 2304 3.9, with 128 threads of three pieces 4.4, norms 4.2 and 4.6).
template <class F> hipError_t with_group(int64_t rows, int C, F&& f) {
    const int pieces = (C + 7) / 8;
#define IVIT_GROUP(nv, tpr, block, s) f(std::integral_constant<int, nv>(), std::integral_constant<int, tpr>(), std::integral_constant<int, block>(), std::integral_constant<bool, s>())
    if (C < 8) return IVIT_GROUP(1, 8, 64, true);
    if (pieces <= 8) return IVIT_GROUP(1, 8, 64, false);
    if (pieces <= 16) return IVIT_GROUP(1, 16, 64, false);
    if (pieces <= 32) return IVIT_GROUP(1, 32, 64, false);
    if (pieces <= 64) return IVIT_GROUP(1, 64, 64, false);
    const bool many = rows > 2 * num_cus();
    if (pieces <= 192 && many) {
        if (pieces <= 128) return IVIT_GROUP(2, 64, 64, false);
        return IVIT_GROUP(3, 64, 64, false);
    }
    if (pieces <= 256) return IVIT_GROUP(1, 256, 256, false);
    if (pieces <= 384 && many) return IVIT_GROUP(3, 128, 128, false);
    if (pieces <= 512) return IVIT_GROUP(2, 256, 256, false);
    if (pieces <= 1024) return IVIT_GROUP(4, 256, 256, false);
    if (pieces <= 2048) return IVIT_GROUP(2, 1024, 1024, false);
    return IVIT_GROUP(4, 1024, 1024, false);
#undef IVIT_GROUP
}

// Rows of one launch: a grid may have 2^32 threads.
constexpr int64_t kThreads = (int64_t)1 << 31;

template <class T> hipError_t norm_of(hipStream_t s, const RmsNormArgs& a) {
    return with_group(a.rows, a.C, [&](auto nv, auto tpr, auto block, auto few) {
        constexpr int NV = nv, TPR = tpr, BLOCK = block, ROWS = BLOCK / TPR;
        constexpr bool SHORT = few;
        constexpr int64_t MOST = kThreads / BLOCK * ROWS;
        for (int64_t r = 0; r < a.rows; r += MOST) {
            auto at = [&](const void* p, int64_t ld) { return p ? static_cast<const T*>(p) + r * ld : nullptr; };
            const int64_t rows = min64(a.rows - r, MOST), grid = (rows + ROWS - 1) / ROWS;
            NormParams P{at(a.x, a.ldx), at(a.residual, a.ld_res), a.gamma, const_cast<T*>(at(a.sum, a.ld_sum)), nullptr, nullptr,
                         a.ldx, a.ld_res, a.ld_sum, a.ldy, rows, a.C, a.eps};
            const int64_t e = sizeof(T), n = rows * a.C;
            TraceScope trace(s, KIND_RMSNORM, 0, n * e * (1 + (a.residual != nullptr) + (a.sum != nullptr)) + n * (a.y_scale ? 1 : e));
            if (a.y_scale) {
                P.y = static_cast<int8_t*>(a.y) + r * a.ldy;
                P.scale = a.y_scale + r;
                hipLaunchKernelGGL((rmsnorm_kernel<T, NV, TPR, BLOCK, true, SHORT>), dim3((unsigned)grid), dim3(BLOCK), 0, s, P);
            } else {
                P.y = const_cast<T*>(at(a.y, a.ldy));
                hipLaunchKernelGGL((rmsnorm_kernel<T, NV, TPR, BLOCK, false, SHORT>), dim3((unsigned)grid), dim3(BLOCK), 0, s, P);
            }
            if (hipError_t e = hipGetLastError()) return e;
        }
        return hipSuccess;
    });
}

template <class T> hipError_t gate_of(hipStream_t s, const GatedArgs& a) {
    // x past the caches from 32 MB on (8192 x 14336 gated, 470 MB, 103.6 and 99.7 us, 20000 x 1536, 61 MB, 22.7 and 23.2; 1000 x 4096 gated, 16 MB,
    // 6.4 and 6.0).  The norm's inputs, residual and all, are better left alone (when chosen: 25216 x 384 13.7 and 16.6, 16384 x 4096 82 and 79.5).
    const int once = a.rows * a.C * (int64_t)sizeof(T) * (a.gated ? 2 : 1) >= (int64_t)1 << 25;
    return with_group(a.rows, a.C, [&](auto nv, auto tpr, auto block, auto few) {
        constexpr int NV = nv, TPR = tpr, BLOCK = block, ROWS = BLOCK / TPR;
        constexpr bool SHORT = few;
        constexpr int64_t MOST = kThreads / BLOCK * ROWS;
        for (int64_t r = 0; r < a.rows; r += MOST) {
            const int64_t rows = min64(a.rows - r, MOST), grid = (rows + ROWS - 1) / ROWS;
            const GateParams P{static_cast<const T*>(a.x) + r * a.ldx, a.y + r * a.ldy, a.y_scale + r, a.ldx, a.ldy, rows, a.C, a.act, once};
            TraceScope trace(s, KIND_GATED, 0, rows * a.C * ((int64_t)sizeof(T) * (a.gated ? 2 : 1) + 1));
            if (a.gated) hipLaunchKernelGGL((gated_kernel<T, NV, TPR, BLOCK, true, SHORT>), dim3((unsigned)grid), dim3(BLOCK), 0, s, P);
            else hipLaunchKernelGGL((gated_kernel<T, NV, TPR, BLOCK, false, SHORT>), dim3((unsigned)grid), dim3(BLOCK), 0, s, P);
            if (hipError_t e = hipGetLastError()) return e;
        }
        return hipSuccess;
    });
}

}  // namespace

hipError_t launch_rmsnorm(hipStream_t s, const RmsNormArgs& a) {
    if (a.rows == 0) return hipSuccess;
    if (a.type == TYPE_F16) return norm_of<_Float16>(s, a);
    if (a.type == TYPE_BF16) return norm_of<__bf16>(s, a);
    return norm_of<float>(s, a);
}

hipError_t launch_gated(hipStream_t s, const GatedArgs& a) {
    if (a.rows == 0) return hipSuccess;
    if (a.type == TYPE_F16) return gate_of<_Float16>(s, a);
    if (a.type == TYPE_BF16) return gate_of<__bf16>(s, a);
    return gate_of<float>(s, a);
}

}  // namespace ivit
