// Attention of one token per request over a paged cache, with a prefix that all requests share.
//
//   o_b = softmax over the prefix's keys and the request's own of scale q_b . k, times their values
//
// The keys are cut into parts: the prefix into some for all requests together, whose queries (all requests, the heads of a group) are then rows of one
// product, and each request's own keys into as many for every request.  A workgroup takes 32 query rows against one part; its wavefronts take blocks of
// 32 keys of it in turn, each through LDS of its own, and join what they have at the end.  The parts of a row, its largest score, sum and unscaled output
// each, are joined by a second launch, in a fixed order.
//
// int8 rows come into LDS as they are and are spread to 16 bits on the way to the matrix cores, where whole numbers up to 127 are exact.  The keys' scales
// go to the scores, the values' to the weights.
#include "regst_common.hpp"
#include "float_attention.hpp"

namespace ivit {
namespace {

using namespace regst;
using namespace fatt;

constexpr int W = 4, BK = 32, S = 2;           // wavefronts; keys of a block; blocks of a wavefront in LDS

struct CaParams {
    const void* q; void* o; const int8_t *k, *v; const float *ks, *vs; const int32_t *prefix_pages, *pages, *lens; float *ml, *part;
    int64_t ldq, ldo, ld_pages, ld_page;       // ld_page in bytes
    int prefix_len, max_len, B, H, G, group, page_shift, n_pages, prefix_parts, own_parts, prefix_tiles, own_tiles; float c;
};

template <class T, int D, bool I8> struct CaTile {
    static constexpr int RB = I8 ? D : 2 * D, BYTES = BK * RB, STAGE = 2 * BYTES + (I8 ? 2 * 4 * BK : 0);      // of a key's row; keys or values; a block
    static constexpr int OUT = BK * (D + 4) * 4;                                                              // a wavefront's output on its way to the others
    static constexpr int WAVE = S * STAGE > OUT ? S * STAGE : OUT;
};

// 16-byte pieces of an int8 row: piece ^ mix8(row), for keys (8 bytes of 32 rows at a time) and values (8 bytes of 8 rows, twice) alike
template <int D> __device__ __forceinline__ int mix8(int row) { return D == 128 ? row & 7 : (row >> 1) & 3; }

// 4 bytes per lane from an address of its own into LDS at dst + 4 lane
__device__ __forceinline__ void dma4_at(const float* p, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(p) : "memory", "m0");
}

template <class T> __device__ __forceinline__ typename Elem<T>::v8 spread(v2u b) {
    typename Elem<T>::v8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)(float)(int8_t)(b[e / 4] >> (8 * (e % 4)));
    return v;
}

template <class T, int D, bool I8>
__global__ __launch_bounds__(64 * W) void cached_attention_kernel(CaParams P) {
    using TL = CaTile<T, D, I8>;
    using V8 = typename Elem<T>::v8;
    constexpr int RB = TL::RB, DS = D / 16, DT = D / 32, PC = RB / 16, LR = 64 / PC, LI = BK / LR;      // pieces of a row; rows of a load instruction; loads of a block
    __shared__ __align__(16) int8_t lds[W * TL::WAVE];
    __shared__ float join_m[W][32], join_l[W][32];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, li = lane & 31;

    // which rows, which keys
    const int prefix_items = P.prefix_tiles * P.G * P.prefix_parts;
    int item = blockIdx.x, g, b = 0, r0, rows, len, part, parts;
    const bool prefix = item < prefix_items;
    const int32_t* table;
    if (prefix) {                                          // items of the same keys are a multiple of the heads' and parts' number apart
        part = item % P.prefix_parts; item /= P.prefix_parts;
        g = item % P.G;
        r0 = 32 * (item / P.G);
        rows = P.B * P.group;
        len = P.prefix_len; parts = P.prefix_parts; table = P.prefix_pages;
    } else {
        item -= prefix_items;
        part = item % P.own_parts; item /= P.own_parts;
        g = item % P.G; item /= P.G;
        r0 = 32 * (item % P.own_tiles);
        b = item / P.own_tiles;
        rows = P.group;
        len = P.lens[b]; parts = P.own_parts; table = P.pages + (int64_t)b * P.ld_pages;
        if (len < 0) return;
        len = min(len, P.max_len);
    }
    const int blocks = (len + BK - 1) / BK, each = max((blocks + parts - 1) / parts, W);
    const int b0 = min(part * (int64_t)each, (int64_t)blocks), b1 = min(b0 + each, blocks);
    const int out_part = prefix ? part : P.prefix_parts + part, all_parts = P.prefix_parts + P.own_parts;
    auto row_of = [&](int r, int& rb, int& rh) __attribute__((always_inline)) {        // request and head of row r
        const int x = r0 + r;
        rb = prefix ? x / P.group : b;
        rh = g * P.group + (prefix ? x % P.group : x);
    };

    // loads: instruction i brings rows LR i + lane / PC, physical piece lane % PC
    int8_t* const mine = lds + wv * TL::WAVE;
    const uint32_t lds0 = lds_offset(mine);
    const int mask = (1 << P.page_shift) - 1, lr = lane / PC, lp = lane % PC;
    typedef const int32_t __attribute__((address_space(4)))* scalar_table;
    auto issue = [&](int blk, int buf) __attribute__((always_inline)) {
        const int k0 = blk * BK, last = len - 1;
        int scale_page[2];
#pragma unroll
        for (int a = 0; a < 2; ++a) {                      // 16 keys, which lie in one page (behind the last key: that one again)
            const int first = min(k0 + 16 * a, last);
            const int page = min(max(((scalar_table)table)[first >> P.page_shift], 0), P.n_pages - 1);
            const int64_t at = (int64_t)page * P.ld_page + ((int64_t)g << P.page_shift) * RB;
            const int8_t *const kp = uniform_ptr(P.k + at), *const vp = uniform_ptr(P.v + at);
#pragma unroll
            for (int i = 0; i < LI / 2; ++i) {
                const int r = 16 * a + LR * i + lr, slot = min(k0 + r, last) & mask;
                const int mk = I8 ? mix8<D>(r) : mix_k<D>(r), mv = I8 ? mix8<D>(r) : mix_v<D>(r);
                const uint32_t to = lds0 + buf * TL::STAGE + (a * (LI / 2) + i) * 1024;
                dma16(kp, slot * RB + 16 * (lp ^ mk), to);
                dma16(vp, slot * RB + 16 * (lp ^ mv), to + TL::BYTES);
            }
            if constexpr (I8) scale_page[a] = page;
        }
        if constexpr (I8) {                                // lanes 0 .. 31: the keys' scales, 32 .. 63: the values'
            const int64_t slots = ((int64_t)(li < 16 ? scale_page[0] : scale_page[1]) * P.G + g) << P.page_shift;
            dma4_at((half ? P.vs : P.ks) + slots + (min(k0 + li, last) & mask), lds0 + buf * TL::STAGE + 2 * TL::BYTES);
        }
    };
    int blk = b0 + wv;
    if (blk < b1) issue(blk, 0);

    V8 qf[DS];
    {
        int rb, rh;
        row_of(min(li, rows - 1 - r0), rb, rh);
        const T* const qp = static_cast<const T*>(P.q) + (int64_t)rb * P.ldq + (int64_t)rh * D + 8 * half;
#pragma unroll
        for (int s = 0; s < DS; ++s) qf[s] = *reinterpret_cast<const V8*>(qp + 16 * s);
    }
    v16f acc[DT];
    float m = -__builtin_inff(), l = 0.0f, ref = 0.0f;
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = v16f{};

#pragma unroll 1
    for (int n = 0; blk < b1; ++n, blk += W) {
        const int buf = n & 1;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if (blk + W < b1) issue(blk + W, buf ^ 1);
        const int8_t* const kl = mine + buf * TL::STAGE;
        const int8_t* const vl = kl + TL::BYTES;
        v16f s[1] = {v16f{}};
#pragma unroll
        for (int d = 0; d < DS; ++d) {
            V8 kf;
            if constexpr (I8) kf = spread<T>(*reinterpret_cast<const v2u*>(kl + li * RB + 16 * (d ^ mix8<D>(li)) + 8 * half));
            else kf = *reinterpret_cast<const V8*>(kl + li * RB + 16 * ((2 * d + half) ^ mix_k<D>(li)));
            s[0] = mfma(kf, qf[d], s[0]);
        }
        const float* const scale = reinterpret_cast<const float*>(kl + 2 * TL::BYTES);
        if constexpr (I8) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] *= scale[8 * (r / 4) + 4 * half + r % 4];
        }
        if ((blk + 1) * BK > len) {
            const int rel = len - 1 - blk * BK - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r / 4) + r % 4 > rel) s[0][r] = -__builtin_inff();
        }
        V8 pw[1][2];
        V8 (&p)[2] = pw[0];
        if constexpr (I8) {
            // Weights times the values' scales, over 2^ref: what float16 holds goes by the largest scale so far.
            const float most = scale[BK + li];
            float top = most;
#pragma unroll
            for (int x = 1; x < 32; x *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, x));
            softmax_step_scaled<T, DT>(s, p, m, l, acc, P.c, ref, n == 0, top, scale + BK + 4 * half);
        } else {
            softmax_step<T, 1, DT>(s, pw, m, l, acc, P.c);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                V8 vf;
                if constexpr (I8) {
                    // the transposing read of bytes takes 8 rows x 16 elements from 16 lanes: keys 16 t + 4 half + 0 .. 3 and + 8 .. 11
                    typedef v2i __attribute__((address_space(3)))* at;
                    const int j = (lane & 15) >> 1, row = 16 * t + 4 * half + (j & 3) + 8 * (j >> 2), col = 32 * i + 16 * ((lane >> 4) & 1) + 8 * (lane & 1);
                    vf = spread<T>(__builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr8_b64_v2i32((at)(vl + row * RB + 16 * ((col >> 4) ^ mix8<D>(row)) + (col & 15)))));
                } else {
                    vf = transposed<T, D>(vl + transposed_at<D>(i, lane) + 16 * t * RB);
                }
                acc[i] = mfma(vf, p[t], acc[i]);
            }
    }
    l = add_halves(l);

    // the wavefronts' parts: largest scores and sums, then the outputs
    if (half == 0) { join_m[wv][li] = m; join_l[wv][li] = l; }
    float* const out = reinterpret_cast<float*>(mine);
    const float up = I8 ? __builtin_amdgcn_exp2f(ref) : 1.0f;
    __syncthreads();                                       // (every wavefront has read its last block)
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[li * (D + 4) + 32 * i + 8 * (r / 4) + 4 * half + r % 4] = acc[i][r] * up;
    __syncthreads();
    constexpr int TPR = 256 / 32, E = D / TPR;             // threads of a row; elements of a thread
    const int row = tid / TPR, e0 = tid % TPR * E;
    if (r0 + row >= rows) return;
    float top = join_m[0][row], f[W], sum = 0.0f, val[E] = {};
#pragma unroll
    for (int w = 1; w < W; ++w) top = __builtin_fmaxf(top, join_m[w][row]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        f[w] = join_l[w][row] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((join_m[w][row] - top) * P.c);
        if (join_l[w][row] == 0.0f) continue;              // (no keys)
        sum = __builtin_fmaf(f[w], join_l[w][row], sum);
#pragma unroll
        for (int e = 0; e < E; ++e)
            val[e] = __builtin_fmaf(f[w], reinterpret_cast<const float*>(lds + w * TL::WAVE)[row * (D + 4) + e0 + e], val[e]);
    }
    int rb, rh;
    row_of(row, rb, rh);
    if (all_parts == 1) {
        if (P.lens[rb] < 0) return;
        T* const o = static_cast<T*>(P.o) + (int64_t)rb * P.ldo + (int64_t)rh * D + e0;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = (T)(val[e] * inv);
        return;
    }
    const int64_t at = (int64_t)out_part * P.B * P.H + (int64_t)rb * P.H + rh;
    if (e0 == 0) { P.ml[2 * at] = top; P.ml[2 * at + 1] = sum; }
    if (sum != 0.0f)
#pragma unroll
        for (int e = 0; e < E; ++e) P.part[at * D + e0 + e] = val[e];
}

// One wavefront a row: the parts' outputs, each times 2^(its maximum less the largest).
template <class T, int D> __global__ __launch_bounds__(256) void join_kernel(CaParams P, int parts) {
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)P.B * P.H, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int b = (int)(row / P.H);
    if (P.lens[b] < 0) return;
    float top = -__builtin_inff();
    for (int p = 0; p < parts; ++p)
        if (P.ml[2 * (p * rows + row) + 1] != 0.0f) top = __builtin_fmaxf(top, P.ml[2 * (p * rows + row)]);
    float sum = 0.0f, val[D / 64] = {};
    for (int p = 0; p < parts; ++p) {
        const int64_t at = p * rows + row;
        const float l = P.ml[2 * at + 1];
        if (l == 0.0f) continue;
        const float f = __builtin_amdgcn_exp2f((P.ml[2 * at] - top) * P.c);
        sum = __builtin_fmaf(f, l, sum);
#pragma unroll
        for (int e = 0; e < D / 64; ++e) val[e] = __builtin_fmaf(f, P.part[at * D + lane * (D / 64) + e], val[e]);
    }
    T* const o = static_cast<T*>(P.o) + b * P.ldo + (row % P.H) * D + lane * (D / 64);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) o[e] = (T)(val[e] * inv);
}

struct Plan { int prefix_tiles, own_tiles, prefix_parts, own_parts; };

// Parts: about two workgroups a CU, each of 256 keys at least.
Plan plan_of(const CachedArgs& a) {
    const int group = a.H / a.c.G, goal = 2 * num_cus();
    Plan p{(int)(((int64_t)a.B * group + 31) / 32), (group + 31) / 32, 0, 0};
    auto parts = [&](int64_t items, int64_t keys) {
        const int64_t most = (keys + 255) / 256, want = (goal + items - 1) / items;
        return (int)(want < most ? want : most);
    };
    if (a.prefix_len > 0) p.prefix_parts = parts((int64_t)p.prefix_tiles * a.c.G, a.prefix_len);
    if (a.max_pages > 0) p.own_parts = parts((int64_t)a.B * p.own_tiles * a.c.G, (int64_t)a.max_pages * a.c.page_size);
    return p;
}
size_t ml_bytes(const CachedArgs& a, int parts) { return ((size_t)parts * a.B * a.H * 8 + 255) & ~(size_t)255; }

template <class T, int D, bool I8> hipError_t launch(hipStream_t s, const CachedArgs& a) {
    const Plan p = plan_of(a);
    const int parts = p.prefix_parts + p.own_parts;
    float* const ml = static_cast<float*>(a.workspace);
    const CaParams P{a.q, a.o, static_cast<const int8_t*>(a.c.k), static_cast<const int8_t*>(a.c.v), a.c.k_scale, a.c.v_scale, a.prefix_pages, a.pages, a.lens,
                     ml, reinterpret_cast<float*>(static_cast<int8_t*>(a.workspace) + ml_bytes(a, parts)), a.ldq, a.ldo, a.ld_pages,
                     a.c.ld_page * (I8 ? 1 : 2), a.prefix_len, a.max_pages * a.c.page_size, a.B, a.H, a.c.G, a.H / a.c.G, __builtin_ctz(a.c.page_size), a.c.n_pages,
                     p.prefix_parts, p.own_parts, p.prefix_tiles, p.own_tiles, a.scale * 1.44269504088896341f};
    const int64_t items = (int64_t)p.prefix_tiles * a.c.G * p.prefix_parts + (int64_t)a.B * p.own_tiles * a.c.G * p.own_parts;
    const int64_t keys = a.prefix_len + (int64_t)a.B * a.max_pages * a.c.page_size;
    if (items > 0) {
        TraceScope trace(s, KIND_CACHED_ATTENTION, 4 * (int64_t)D * a.H * a.B * (a.prefix_len + (int64_t)a.max_pages * a.c.page_size),
                         2 * keys * a.c.G * (I8 ? D + 4 : 2 * D) + 4 * (int64_t)a.B * a.H * D);
        cached_attention_kernel<T, D, I8><<<dim3((unsigned)items), 64 * W, 0, s>>>(P);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (parts == 1) return hipSuccess;
    TraceScope trace(s, KIND_CACHED_JOIN, 0, (int64_t)a.B * a.H * (parts * (4 * (int64_t)D + 8) + 2 * D));
    join_kernel<T, D><<<dim3((unsigned)(((int64_t)a.B * a.H + 3) / 4)), 256, 0, s>>>(P, parts);
    return hipGetLastError();
}

}  // namespace

size_t cached_attention_workspace(const CachedArgs& a) {
    const Plan p = plan_of(a);
    const int parts = p.prefix_parts + p.own_parts;
    return ml_bytes(a, parts) + (((size_t)parts * a.B * a.H * a.c.d * 4 + 255) & ~(size_t)255) + 256;
}

hipError_t launch_cached_attention(hipStream_t s, const CachedArgs& a) {
    const bool i8 = a.c.type == TYPE_I8;
    if (a.type == TYPE_F16) {
        if (a.c.d == 64) return i8 ? launch<_Float16, 64, true>(s, a) : launch<_Float16, 64, false>(s, a);
        return i8 ? launch<_Float16, 128, true>(s, a) : launch<_Float16, 128, false>(s, a);
    }
    if (a.c.d == 64) return i8 ? launch<__bf16, 64, true>(s, a) : launch<__bf16, 64, false>(s, a);
    return i8 ? launch<__bf16, 128, true>(s, a) : launch<__bf16, 128, false>(s, a);
}

}  // namespace ivit
