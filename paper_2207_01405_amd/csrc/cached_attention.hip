// Attention of one token per request over a paged cache, with a prefix that all requests share.
//
//   o_b = softmax over the prefix's keys and the request's own of scale q_b . k, times their values
//
// The keys are cut into parts: the prefix into some for all requests together, whose queries (all requests, the heads of a group) are then rows of one
// product, and each request's own keys by their number.  A workgroup takes 32 query rows against one part; its wavefronts take blocks of 32 keys of it in
// turn, each through LDS of its own without a barrier, and join what they have at the end.  The parts of a row, its largest score, sum and unscaled
// output each, are joined by a second launch, in a fixed order.
//
// int8 rows come into LDS as they are and are spread to float16 on the way to the matrix cores, where whole numbers up to 128 are exact: an instruction and a
// quarter an element, which bounds these caches (to bfloat16, which has no place for eight bits under a leading one, they were three, and 48 requests of 8192 keys took
// 177 us for 163).  bfloat16 queries become float16 with a power of two of their own, which their scores get back.  The keys' scales go to the
// scores, the values' to the weights.
#include "cached_form.hpp"
#include "regst_common.hpp"
#include "float_attention.hpp"

namespace ivit {
namespace {

using namespace regst;
using namespace fatt;
using namespace cached;

typedef float v4f __attribute__((ext_vector_type(4)));

struct CaParams {
    const void* q; void* o; const int8_t *k, *v; const float *ks, *vs; const int32_t *prefix_pages, *pages, *lens; float *ml, *part;
    int64_t ldq, ldo, ld_pages, ld_page;       // ld_page in bytes
    int prefix_len, max_len, B, H, G, group, page_shift, n_pages, prefix_parts, own_parts, prefix_least, own_least, prefix_tiles, wide; float c;
    FastDiv by_head, by_prefix_part, by_own_part, by_own_tile, by_group, by_heads;
};

// RB: bytes of a key's row; BYTES: of the keys or values of a block.  A wavefront has S blocks of keys and S of values in LDS or on their way there, some
// 16 KB in all, so that two workgroups fit a CU; keys are asked for again as soon as the scores are formed, values behind their product.  In the end
// the space takes the wavefronts' outputs.
template <int D, bool I8> struct CaTile {
    static constexpr int RB = I8 ? D : 2 * D, BYTES = BK * RB, S = I8 || D == 64 ? 2 : 1, STAGE = 2 * BYTES + (I8 ? 2 * 4 * BK : 0);
    static constexpr int OUT = 64 * 16 * (D / 32) * 4, WAVE = S * STAGE > OUT ? S * STAGE : OUT;
    static constexpr int SHARED = 2 * TK * RB + (I8 ? W * 256 : 0);               // a tile of keys and values that the wavefronts share, two of them
    static_assert(2 * SHARED <= W * WAVE, "room for two");
};

// 16-byte pieces of an int8 row are stored at piece ^ mix8(row).  Keys are read 8 bytes of 16 rows at a time, values 32 bytes of rows 0 .. 3 and 8 .. 11 or 4 .. 7
// and 12 .. 15: either spreads over all banks.
template <int D> __device__ __forceinline__ int mix8(int row) {
    return D == 128 ? (row & 2) | ((row >> 2) & 1) | ((row >> 1) & 4) : ((row >> 2) & 1) | ((row >> 2) & 2);
}

// all loads but the newest N have arrived; all LDS reads have
template <int N> __device__ __forceinline__ void wait_but() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// 4 bytes per lane from an address of its own into LDS at dst + 4 lane
__device__ __forceinline__ void dma4_at(const float* p, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(p) : "memory", "m0");
}

// Eight int8 numbers as float16: 128 + q in the low bits of 1024 is 1152 + q.
__device__ __forceinline__ Elem<_Float16>::v8 spread(v2u b) {
    const uint32_t x = b[0] ^ 0x80808080u, y = b[1] ^ 0x80808080u, up = 0x64646464u;
    const v4u w = {__builtin_amdgcn_perm(up, x, 0x04010400u), __builtin_amdgcn_perm(up, x, 0x04030402u), __builtin_amdgcn_perm(up, y, 0x04010400u),
                   __builtin_amdgcn_perm(up, y, 0x04030402u)};
    return __builtin_bit_cast(Elem<_Float16>::v8, w) - (_Float16)1152.0f;
}

// What the matrix cores multiply: the rows' type, float16 where the cache is int8.
template <class T, bool I8> using Mul = std::conditional_t<I8, _Float16, T>;

// A lane's half of a query row, elements 16 s + 8 half on, as fragments; those of an int8 cache's bfloat16 queries over 2^e, e that of the row's largest: what is
// below 2^-14 of it keeps 24 bits below it.  Returns 2^e, a normal number as its reciprocal is.
template <class T, bool I8, int DS> __device__ __forceinline__ float query(const T* q, typename Elem<Mul<T, I8>>::v8 (&qf)[DS]) {
    if constexpr (!I8 || __is_same(T, _Float16)) {
#pragma unroll
        for (int s = 0; s < DS; ++s) qf[s] = *reinterpret_cast<const typename Elem<T>::v8*>(q + 16 * s);
        return 1.0f;
    } else {
        typename Elem<T>::v8 x[DS];
        float top = 0.0f;
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            x[s] = *reinterpret_cast<const typename Elem<T>::v8*>(q + 16 * s);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = __builtin_fmaxf(top, __builtin_fabsf((float)x[s][e]));
        }
        top = max_halves(top);
        const int e = top > 0.0f && top < 0x1p126f ? max(__builtin_amdgcn_frexp_expf(top), -125) : top > 0.0f ? 120 : 0;
        const float down = __builtin_amdgcn_ldexpf(1.0f, -e);
#pragma unroll
        for (int s = 0; s < DS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) qf[s][i] = (_Float16)((float)x[s][i] * down);
        return __builtin_amdgcn_ldexpf(1.0f, e);
    }
}

// Parts are joined by the exponents of their largest scores: scores of rows of int8 keys, each in units of its own, need not fit 32 bits otherwise.
__device__ __forceinline__ float exponent(float m, float c) { return m == -__builtin_inff() ? m : m * c; }

// The page of a key by its number, as a scalar load.  (Kept 64 at a time in a vector register: no change.)
__device__ __forceinline__ int page_at(const CaParams& P, const int32_t* table, int key) {
    return min(max(((const int32_t __attribute__((address_space(4)))*)table)[key >> P.page_shift], 0), P.n_pages - 1);
}

// Fragments of 32 keys and of 16 keys' values (as transposed has them) from rows in LDS.
template <class T, int D, bool I8> __device__ __forceinline__ typename Elem<Mul<T, I8>>::v8 key_frag(const int8_t* kl, int d, int li, int half) {
    if constexpr (I8) return spread(*reinterpret_cast<const v2u*>(kl + li * D + 16 * (d ^ mix8<D>(li)) + 8 * half));
    else return *reinterpret_cast<const typename Elem<T>::v8*>(kl + li * 2 * D + 16 * ((2 * d + half) ^ mix_k<D>(li)));
}
template <class T, int D, bool I8> __device__ __forceinline__ typename Elem<Mul<T, I8>>::v8 value_frag(const int8_t* vl, int i, int lane) {
    if constexpr (I8) {
        // the transposing read of bytes takes 8 rows x 16 elements from 16 lanes: keys 4 half + 0 .. 3 and + 8 .. 11
        typedef v2i __attribute__((address_space(3)))* at;
        const int j = (lane & 15) >> 1, row = 4 * (lane >> 5) + (j & 3) + 8 * (j >> 2), col = 32 * i + 16 * ((lane >> 4) & 1) + 8 * (lane & 1);
        return spread(__builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr8_b64_v2i32((at)(vl + row * D + 16 * ((col >> 4) ^ mix8<D>(row)) + (col & 15)))));
    } else {
        return transposed<T, D>(vl + transposed_at<D>(i, lane));
    }
}

// The prefix for more than 64 query rows: a wavefront has 32 rows of its own, and all share tiles of 64 keys, of which each brings 16.  Scores are formed
// a tile ahead of the values' product.
template <class T, int D, bool I8, class RowOf>
__device__ __forceinline__ void shared_keys(const CaParams& P, int8_t* lds, int g, int first, int k0, int k1, int part, RowOf&& row_of) {
    using TL = CaTile<D, I8>;
    using V8 = typename Elem<Mul<T, I8>>::v8;
    constexpr int RB = TL::RB, DS = D / 16, DT = D / 32, PC = RB / 16, LR = 64 / PC, LI = 16 / LR, KB = TK / 32;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, li = lane & 31;
    const int rows = P.B * P.group, last = k1 - 1, tiles = (k1 - k0 + TK - 1) / TK, mask = (1 << P.page_shift) - 1;
    const uint32_t lds0 = lds_offset(lds);
    auto issue = [&](int n, auto values) __attribute__((always_inline)) {
        constexpr bool V = decltype(values)::value;
        if (n >= tiles) return;
        const int from = k0 + n * TK + 16 * wv, page = page_at(P, P.prefix_pages, min(from, last));
        const int8_t* const p = uniform_ptr((V ? P.v : P.k) + (int64_t)page * P.ld_page + ((int64_t)g << P.page_shift) * RB);
        const uint32_t to = lds0 + (n & 1) * TL::SHARED + (V ? TK * RB : 0) + 16 * RB * wv;
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            const int r = LR * i + lane / PC, slot = min(from + r, last) & mask;
            const int mix = I8 ? mix8<D>(r) : V ? mix_v<D>(r) : mix_k<D>(r);
            dma16(p, slot * RB + 16 * ((lane % PC) ^ mix), to + i * 1024);
        }
        if constexpr (I8) {                                // the scales of the 16 keys, and 64 bytes behind them, of the values
            const int64_t slots = ((int64_t)page * P.G + g) << P.page_shift;
            if (lane < 16) dma4_at((V ? P.vs : P.ks) + slots + (min(from + lane, last) & mask), lds0 + (n & 1) * TL::SHARED + 2 * TK * RB + 256 * wv + (V ? 64 : 0));
        }
    };
    constexpr std::false_type keys{};
    constexpr std::true_type values{};
    issue(0, keys);
    issue(0, values);
    const int mine = first + 32 * wv;
    V8 qf[DS];
    float c = P.c;                                         // of scores in the row's units, as m is up to the end
    {
        int rb, rh;
        row_of(min(mine + li, rows - 1), rb, rh);
        c *= query<T, I8>(static_cast<const T*>(P.q) + (int64_t)rb * P.ldq + (int64_t)rh * D + 8 * half, qf);
    }
    v16f acc[DT];
    float m = -__builtin_inff(), l = 0.0f, ref = kRefLeast;
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = v16f{};
    auto scale_at = [&](int buf, int b, int r) __attribute__((always_inline)) {        // of the keys; 16 further on: of the values
        return lds + buf * TL::SHARED + 2 * TK * RB + 256 * (2 * b + r / 8) + 4 * (8 * (r / 4 % 2) + 4 * half + r % 4);
    };
    auto scores = [&](int n, int buf, v16f (&s)[KB]) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DS; ++d)
#pragma unroll
            for (int b = 0; b < KB; ++b) s[b] = mfma(key_frag<T, D, I8>(lds + buf * TL::SHARED + 32 * b * RB, d, li, half), qf[d], d ? s[b] : v16f{});
    };
    auto finish = [&](int n, int buf, v16f (&s)[KB]) __attribute__((always_inline)) {  // scales, and keys behind the last one
        if constexpr (I8) {
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] *= *reinterpret_cast<const float*>(scale_at(buf, b, r));
        }
        const int left = last - k0 - n * TK;
        if (left < TK - 1) {
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * b + 8 * (r / 4) + r % 4 > left - 4 * half) s[b][r] = -__builtin_inff();
        }
    };
    arrive<0>();
    issue(1, keys);
    v16f even_s[KB], odd_s[KB];
    scores(0, 0, even_s);
    finish(0, 0, even_s);
    // The values behind the last key, of weight 0, to 0 (with int8 rows, their scales): the last key's are in their place, and may be infinite.
    auto clear = [&](int n, int buf) __attribute__((always_inline)) {
        wait_but<0>();
        const int from = max(last + 1 - (k0 + n * TK + 16 * wv), 0);
        int8_t* const to = lds + buf * TL::SHARED;
        if constexpr (I8) {
            if (lane >= from && lane < 16) *reinterpret_cast<float*>(to + 2 * TK * RB + 256 * wv + 64 + 4 * lane) = 0.0f;
        } else {
#pragma unroll 1
            for (int i = from * PC + lane; i < 16 * PC; i += 64) *reinterpret_cast<v4u*>(to + (TK + 16 * wv) * RB + 16 * i) = v4u{};
        }
    };
    auto step = [&](int n, int buf, v16f (&s)[KB], v16f (&next)[KB]) __attribute__((always_inline)) {
        if (n == tiles - 1 && last - k0 - n * TK < TK - 1) clear(n, buf);
        arrive<0>();
        issue(n + 2, keys);
        issue(n + 1, values);
        V8 p[KB][2];
        if constexpr (I8) {
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                v16f one[1] = {s[b]};
                float vs[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) vs[r] = *reinterpret_cast<const float*>(scale_at(buf, b, r) + 64);
                softmax_step_scaled<DT>(one, p[b], m, l, acc, c, ref, vs);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < DT; ++i) acc[i] = mfma(value_frag<T, D, I8>(lds + buf * TL::SHARED + (TK + 32 * b + 16 * t) * RB, i, lane), p[b][t], acc[i]);
            }
            __builtin_amdgcn_sched_barrier(0);             // (products of both mixed need a register too many)
            scores(n + 1, buf ^ 1, next);                  // (of the last tile: of what that buffer holds, not used)
        } else {
            move_largest<DT>(largest_of(s), m, l, acc, c);
            const float base = base_of<T>(m, c);
            scores(n + 1, buf ^ 1, next);
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; r += 2) weigh<T>(s[b], r, p[b], l, c, base);
#pragma unroll
            for (int t = 0; t < 2 * KB; ++t)
#pragma unroll
                for (int i = 0; i < DT; ++i) acc[i] = mfma(value_frag<T, D, I8>(lds + buf * TL::SHARED + (TK + 16 * t) * RB, i, lane), p[t / 2][t % 2], acc[i]);
        }
        finish(n + 1, buf ^ 1, next);
    };
#pragma unroll 1
    for (int n = 0; n < tiles; n += 2) {
        step(n, 0, even_s, odd_s);
        if (n + 1 < tiles) step(n + 1, 1, odd_s, even_s);
    }
    l = add_halves(l);
    m = exponent(m, c);
    // results as whole lines: a lane's registers into LDS of the wavefront's own, and out of it 4 elements of row lane / 8 + 8 n at 4 (lane % 8)
    __syncthreads();
    float* const out = reinterpret_cast<float*>(lds + wv * TL::WAVE);
    const float up = I8 ? __builtin_amdgcn_exp2f(ref - 15.0f) : 1.0f;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[64 * (16 * i + r) + lane] = acc[i][r] * up;
    int rb, rh;
    if (half == 0 && mine + li < rows) {
        row_of(mine + li, rb, rh);
        const int64_t at = (int64_t)part * P.B * P.H + (int64_t)rb * P.H + rh;
        P.ml[2 * at] = m;
        P.ml[2 * at + 1] = l;
    }
    const int q = lane % 8;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int r = lane / 8 + 8 * n;
        if (mine + r >= rows) continue;
        row_of(mine + r, rb, rh);
        float* const to = P.part + ((int64_t)part * P.B * P.H + (int64_t)rb * P.H + rh) * D + 4 * q;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const float* const x = out + 64 * (16 * i + 4 * (q / 2)) + r + 32 * (q % 2);
            *reinterpret_cast<v4f*>(to + 32 * i) = v4f{x[0], x[64], x[128], x[192]};
        }
    }
}

template <class T, int D, bool I8>
__global__ __launch_bounds__(64 * W, 2) void cached_attention_kernel(CaParams P) {
    using TL = CaTile<D, I8>;
    using V8 = typename Elem<Mul<T, I8>>::v8;
    constexpr int RB = TL::RB, S = TL::S, DS = D / 16, DT = D / 32, PC = RB / 16, LR = 64 / PC, LI = BK / LR;      // pieces of a row; rows of a load instruction; loads
    __shared__ __align__(16) int8_t lds[W * TL::WAVE];
    __shared__ float join_m[W][32], join_l[W][32];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, li = lane & 31;

    // which rows, which keys; a head's workgroups are G apart: on the same XCD, if G is a multiple of 8
    uint32_t g_, part_;
    const uint32_t item = P.by_head.divide(blockIdx.x, g_), prefix_items = (uint32_t)(P.prefix_tiles * P.prefix_parts);
    const int g = (int)g_;
    int b = 0, r0, rows, len, parts, least;
    const bool prefix = item < prefix_items;
    const int32_t* table;
    if (prefix) {
        r0 = (P.wide ? WIDE : 32) * (int)P.by_prefix_part.divide(item, part_);
        rows = P.B * P.group;
        len = P.prefix_len; parts = P.prefix_parts; least = P.prefix_least; table = P.prefix_pages;
    } else {
        uint32_t t;
        b = (int)P.by_own_tile.divide(P.by_own_part.divide(item - prefix_items, part_), t);
        r0 = 32 * (int)t;
        rows = P.group;
        len = P.lens[b]; parts = P.own_parts; least = P.own_least; table = P.pages + (int64_t)b * P.ld_pages;
        if (len < 0) return;
        len = min(len, P.max_len);
    }
    const int part = (int)part_, blocks = (len + BK - 1) / BK, each = max((blocks + parts - 1) / parts, least);
    const int b0 = (int)min64(part * (int64_t)each, blocks), b1 = min(b0 + each, blocks);
    const int out_part = prefix ? part : P.prefix_parts + part, all_parts = P.prefix_parts + P.own_parts;
    auto row_of = [&](int r, int& rb, int& rh) __attribute__((always_inline)) {        // request and head of row r
        uint32_t rest = (uint32_t)(r0 + r);
        rb = prefix ? (int)P.by_group.divide(rest, rest) : b;
        rh = g * P.group + (int)rest;
    };
    const bool sharing = prefix && P.wide;
    if (b0 == b1 && (all_parts > 1 || sharing)) {          // no keys here (the only part writes its rows of zeros itself)
        int rb, rh;
        row_of(tid, rb, rh);
        if (tid < (sharing ? WIDE : 32) && r0 + tid < rows) {
            const int64_t at = (int64_t)out_part * P.B * P.H + (int64_t)rb * P.H + rh;
            P.ml[2 * at] = -__builtin_inff();
            P.ml[2 * at + 1] = 0.0f;
        }
        return;
    }

    if (sharing) {
        shared_keys<T, D, I8>(P, lds, g, r0, b0 * BK, min(b1 * BK, len), part, [&](int r, int& rb, int& rh) __attribute__((always_inline)) { row_of(r - r0, rb, rh); });
        return;
    }

    // loads: instruction i brings rows LR i + lane / PC, physical piece lane % PC
    int8_t* const mine = lds + wv * TL::WAVE;
    const uint32_t lds0 = lds_offset(mine);
    const int mask = (1 << P.page_shift) - 1, lr = lane / PC, lp = lane % PC;
    auto issue = [&](int blk, int buf, auto values) __attribute__((always_inline)) {
        constexpr bool V = decltype(values)::value;
        const int k0 = blk * BK, last = len - 1;
        int page[2];
#pragma unroll
        for (int a = 0; a < 2; ++a)                        // 16 keys lie in one page (behind the last key: that one again)
            page[a] = page_at(P, table, min(k0 + 16 * a, last));
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const int8_t* const p = uniform_ptr((V ? P.v : P.k) + (int64_t)page[a] * P.ld_page + ((int64_t)g << P.page_shift) * RB);
#pragma unroll
            for (int i = 0; i < LI / 2; ++i) {
                const int r = 16 * a + LR * i + lr, slot = min(k0 + r, last) & mask;
                const int mix = I8 ? mix8<D>(r) : V ? mix_v<D>(r) : mix_k<D>(r);
                dma16(p, slot * RB + 16 * (lp ^ mix), lds0 + buf * TL::STAGE + (V ? TL::BYTES : 0) + (a * (LI / 2) + i) * 1024);
            }
        }
        if constexpr (I8 && !V) {                          // lanes 0 .. 31: the keys' scales, 32 .. 63: the values'
            const int64_t slots = ((int64_t)(li < 16 ? page[0] : page[1]) * P.G + g) << P.page_shift;
            dma4_at((half ? P.vs : P.ks) + slots + (min(k0 + li, last) & mask), lds0 + buf * TL::STAGE + 2 * TL::BYTES);
        }
    };
    constexpr std::false_type keys{};
    constexpr std::true_type values{};
    constexpr int KL = LI + (I8 ? 1 : 0), PAIR = KL + LI;  // loads of a block's keys; of its keys and values
    const int own = (b1 - b0 - wv + W - 1) / W;            // the wavefront's blocks: b0 + wv + W n
    auto block = [&](int n) __attribute__((always_inline)) { return b0 + wv + W * n; };
#pragma unroll
    for (int n = 0; n < S; ++n)
        if (n < own) {
            issue(block(n), n, keys);
            issue(block(n), n, values);
        }

    V8 qf[DS];
    float c = P.c;                                         // of scores in the row's units, as m is up to the end
    {
        int rb, rh;
        row_of(min(li, rows - 1 - r0), rb, rh);
        c *= query<T, I8>(static_cast<const T*>(P.q) + (int64_t)rb * P.ldq + (int64_t)rh * D + 8 * half, qf);
    }
    // (here, where all loads so far are waited for: the waits in the loop count its own ones)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    v16f acc[DT];
    float m = -__builtin_inff(), l = 0.0f, ref = kRefLeast;
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = v16f{};

#pragma unroll 1
    for (int n = 0; n < own; ++n) {
        const int blk = block(n), buf = S == 1 ? 0 : n & 1;
        if (n + S - 1 < own) wait_but<LI + (S - 1) * PAIR>();              // behind the block's keys: its values, the next S - 1 blocks
        else wait_but<0>();
        const int8_t* const kl = mine + buf * TL::STAGE;
        const int8_t* const vl = kl + TL::BYTES;
        v16f s[1] = {v16f{}};
#pragma unroll
        for (int d = 0; d < DS; ++d) {
            s[0] = mfma(key_frag<T, D, I8>(kl, d, li, half), qf[d], s[0]);
        }
        float ks[16], vs[16];
        if constexpr (I8) {
            const float* const scale = reinterpret_cast<const float*>(kl + 2 * TL::BYTES);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                ks[r] = scale[8 * (r / 4) + 4 * half + r % 4];
                vs[r] = scale[BK + 8 * (r / 4) + 4 * half + r % 4];
            }
        }
        wait_lds();
        if (n + S < own) issue(block(n + S), buf, keys);
        if constexpr (I8) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] *= ks[r];
        }
        if ((blk + 1) * BK > len) {
            const int rel = len - 1 - blk * BK - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r / 4) + r % 4 > rel) {
                    s[0][r] = -__builtin_inff();
                    vs[r] = 0.0f;                          // (see below)
                }
        }
        V8 p[1][2];
        if constexpr (I8) {
            softmax_step_scaled<DT>(s, p[0], m, l, acc, c, ref, vs);
        } else {
            softmax_step<T, 1, DT>(s, p, m, l, acc, c);
        }
        if (n + S < own) wait_but<(S - 1) * PAIR + KL>();                  // behind its values: the next S - 1 blocks, and the keys behind them
        else wait_but<0>();
        if constexpr (!I8)
            if ((blk + 1) * BK > len) {                    // behind the last key are its values again, which may be infinite, of weight 0
#pragma unroll 1
                for (int i = (len - blk * BK) * PC + lane; i < BK * PC; i += 64) *reinterpret_cast<v4u*>(mine + buf * TL::STAGE + TL::BYTES + 16 * i) = v4u{};
                wait_lds();
            }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] = mfma(value_frag<T, D, I8>(vl + 16 * t * RB, i, lane), p[0][t], acc[i]);
        wait_lds();
        if (n + S < own) issue(block(n + S), buf, values);
    }
    l = add_halves(l);
    m = exponent(m, c);

    // The wavefronts' parts: largest scores and sums, then the outputs, a lane's registers to the same lane; a wavefront joins every fourth tile of 32 elements.
    if (half == 0) { join_m[wv][li] = m; join_l[wv][li] = l; }
    const float up = I8 ? __builtin_amdgcn_exp2f(ref - 15.0f) : 1.0f;
    float* const out = reinterpret_cast<float*>(mine) + lane;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[64 * (16 * i + r)] = acc[i][r] * up;
    __syncthreads();
    float top = join_m[0][li], f[W], sum = 0.0f;
#pragma unroll
    for (int w = 1; w < W; ++w) top = __builtin_fmaxf(top, join_m[w][li]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        f[w] = join_m[w][li] == top ? 1.0f : __builtin_amdgcn_exp2f(join_m[w][li] - top);
        sum = __builtin_fmaf(f[w], join_l[w][li], sum);
    }
    if (r0 + li >= rows) return;
    int rb, rh;
    row_of(li, rb, rh);
    if (all_parts == 1 && P.lens[rb] < 0) return;
    const int64_t at = (int64_t)out_part * P.B * P.H + (int64_t)rb * P.H + rh;
    if (all_parts > 1 && tid < 32) { P.ml[2 * at] = top; P.ml[2 * at + 1] = sum; }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    static_assert(DT <= W, "a tile a wavefront");
    if (wv >= DT) return;
    v16f o[1] = {v16f{}};
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[0][r] = __builtin_fmaf(f[w], reinterpret_cast<const float*>(lds + w * TL::WAVE)[lane + 64 * (16 * wv + r)], o[0][r]);
    if (all_parts == 1) {
        store_rows<T, 1>(static_cast<T*>(P.o) + (int64_t)rb * P.ldo + (int64_t)rh * D + 32 * wv, o, inv, half);
    } else {
        float* const to = P.part + at * D + 32 * wv + 4 * half;
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<v4f*>(to + 8 * q) = v4f{o[0][4 * q], o[0][4 * q + 1], o[0][4 * q + 2], o[0][4 * q + 3]};
    }
}

// One wavefront a row: the parts' outputs, each times 2^(its maximum less the largest).
template <class T, int D, int AT_ONCE> __global__ __launch_bounds__(256) void join_kernel(CaParams P, int parts) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)P.B * P.H, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    uint32_t h;
    const int b = (int)P.by_heads.divide((uint32_t)row, h);
    if (P.lens[b] < 0) return;
    float top = -__builtin_inff(), sum = 0.0f, val[E] = {};
#pragma unroll 1
    for (int p0 = 0; p0 < parts; p0 += 64) {               // 64 parts at once: lane i has part p0 + i
        float m = -__builtin_inff(), l = 0.0f;
        if (p0 + lane < parts) {
            m = P.ml[2 * ((p0 + lane) * rows + row)];
            l = P.ml[2 * ((p0 + lane) * rows + row) + 1];
        }
        float most = l != 0.0f ? m : -__builtin_inff();
#pragma unroll
        for (int x = 1; x < 64; x *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, x));
        const float to = __builtin_fmaxf(top, most), f = to == top ? 1.0f : __builtin_amdgcn_exp2f(top - to);
        sum *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) val[e] *= f;
        top = to;
        const float w = l == 0.0f ? 0.0f : m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        const uint64_t there = __ballot(l != 0.0f);
        // AT_ONCE together: those without keys were not written, and one that was is loaded in their place, for nothing
        const int n = min(64, parts - p0), some = there ? __builtin_ctzll(there) : 0;
        if (there)
#pragma unroll 1
            for (int i0 = 0; i0 < n; i0 += AT_ONCE) {
                float x[AT_ONCE][E], wi[AT_ONCE], li[AT_ONCE];
                bool has[AT_ONCE];
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    const int i = i0 + j;
                    const bool counts = i < n && (there >> i & 1);
                    const int at = counts ? i : some;
                    has[j] = counts;
                    wi[j] = __shfl(w, at);
                    li[j] = __shfl(l, at);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[j][e] = P.part[((p0 + at) * rows + row) * D + lane * E + e];
                }
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    if (!has[j]) continue;                             // (a weight of 0 counts: a sum of NaN stays one)
                    sum = __builtin_fmaf(wi[j], li[j], sum);
#pragma unroll
                    for (int e = 0; e < E; ++e) val[e] = __builtin_fmaf(wi[j], x[j][e], val[e]);
                }
            }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* const o = static_cast<T*>(P.o) + b * P.ldo + (int64_t)h * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = (T)(val[e] * inv);
}

Plan plan_of(const CachedArgs& a) {
    return cached::plan_of(a.B, a.H, a.c.G, a.c.d, a.c.type == TYPE_I8, a.c.page_size, a.max_pages, a.prefix_len, num_cus());
}
size_t ml_bytes(const CachedArgs& a, int parts) { return ((size_t)parts * a.B * a.H * 8 + 255) & ~(size_t)255; }

template <class T, int D, bool I8> hipError_t launch(hipStream_t s, const CachedArgs& a) {
    const Plan p = plan_of(a);
    const int parts = p.prefix_parts + p.own_parts;
    float* const ml = static_cast<float*>(a.workspace);
    auto div = [](int n) { return FastDiv((uint32_t)(n > 0 ? n : 1)); };
    const CaParams P{a.q, a.o, static_cast<const int8_t*>(a.c.k), static_cast<const int8_t*>(a.c.v), a.c.k_scale, a.c.v_scale, a.prefix_pages, a.pages, a.lens,
                     ml, reinterpret_cast<float*>(static_cast<int8_t*>(a.workspace) + ml_bytes(a, parts)), a.ldq, a.ldo, a.ld_pages,
                     a.c.ld_page * (I8 ? 1 : 2), a.prefix_len, a.max_pages * a.c.page_size, a.B, a.H, a.c.G, a.H / a.c.G, __builtin_ctz(a.c.page_size), a.c.n_pages,
                     p.prefix_parts, p.own_parts, p.prefix_least, p.own_least, p.prefix_tiles, p.wide, a.scale * 1.44269504088896341f,
                     div(a.c.G), div(p.prefix_parts), div(p.own_parts), div(p.own_tiles), div(a.H / a.c.G), div(a.H)};
    const int64_t items = ((int64_t)p.prefix_tiles * p.prefix_parts + (int64_t)a.B * p.own_tiles * p.own_parts) * a.c.G;
    const int64_t keys = a.prefix_len + (int64_t)a.B * a.max_pages * a.c.page_size;
    if (items > 0) {
        TraceScope trace(s, KIND_CACHED_ATTENTION, 4 * (int64_t)D * a.H * a.B * (a.prefix_len + (int64_t)a.max_pages * a.c.page_size),
                         2 * keys * a.c.G * (I8 ? D + 4 : 2 * D) + 4 * (int64_t)a.B * a.H * D);
        cached_attention_kernel<T, D, I8><<<dim3((unsigned)items), 64 * W, 0, s>>>(P);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (parts == 1 && !(p.wide && p.prefix_parts)) return hipSuccess;
    TraceScope trace(s, KIND_CACHED_JOIN, 0, (int64_t)a.B * a.H * (parts * (4 * (int64_t)D + 8) + 2 * D));
    auto* const join = parts > 4 ? join_kernel<T, D, 16> : join_kernel<T, D, 4>;
    join<<<dim3((unsigned)(((int64_t)a.B * a.H + 3) / 4)), 256, 0, s>>>(P, parts);
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
