// Attention over whole prompts on the gfx950 matrix cores: packed sequences, grouped heads, causal or not.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c (q_i . k_j - m_i)),   c = scale log2 e,  m_i the largest score so far
//
// One pass over the keys, 64 at a time, with the running maximum and sum of the softmax.  Scores are formed transposed, keys x queries: an MFMA
// result lane then holds scores of ONE query, so that maximum, sum and the rescaling of the output are a lane's own (one exchange between the halves
// of a wavefront joins the maximum), and its registers, rounded and packed, are as they stand the "B" operand of the second product, values x queries:
// that product sums over keys, in any order that both operands agree on, and the values' fragments come by the transposing LDS read in the order
// in which the scores' registers hold the keys.
#include "float_attention.hpp"
#include "prompt_form.hpp"
#include "regst_common.hpp"

namespace ivit {
namespace {

using namespace regst;
using namespace fatt;

struct PaParams {
    const void *q, *k, *v; void* o; const int32_t *q_start, *k_start; int64_t ldq, ldk, ldv, ldo, n_q, n_k;
    int n_seq, H, group, by_xcd, slots; float c; int causal; FastDiv heads;
};

// The sequence of tile slot x: sequence s has the slots q_start[s] / ROWS + s on, which are enough for its rows whatever they begin at.  64 places are
// looked at at once; with up to 64 sequences their bounds come with the same loads.
struct Span { int seq, qa, qb, ka, kb; };
template <int ROWS> __device__ __forceinline__ Span span_of(const int32_t* q_start, const int32_t* k_start, int n_seq, int x, int lane) {
    int lo = 0, n = n_seq;                                          // it is one of lo .. lo + n - 1
    while (n > 64) {
        const int step = (n + 63) / 64, s = lo + lane * step;
        const bool behind = lane * step < n && (max(q_start[s], 0) / ROWS + s) <= x;
        const int at = 63 - __builtin_clzll(__ballot(behind) | 1);
        lo += at * step;
        n = min(step, n - at * step);
    }
    const int s = lo + min(lane, n - 1), qa = q_start[s], qb = q_start[s + 1], ka = k_start[s], kb = k_start[s + 1];
    const int at = 63 - __builtin_clzll(__ballot(lane < n && max(qa, 0) / ROWS + s <= x) | 1);
    return Span{__builtin_amdgcn_readfirstlane(lo + at), __builtin_amdgcn_readlane(qa, at), __builtin_amdgcn_readlane(qb, at), __builtin_amdgcn_readlane(ka, at),
                __builtin_amdgcn_readlane(kb, at)};
}

// RW wavefronts of 32 rows, KG times: group g takes tiles g, g + KG, .. of BK keys, each group through LDS of its own, and the groups join what they have at
// the end.
template <class T, int D, int RW, int KG, int BK>
__global__ __launch_bounds__(64 * RW * KG, 2) void prompt_attention_kernel(PaParams P) {
    constexpr int ROWS = 32 * RW, KB = BK / 32, DS = D / 16, DT = D / 32, RB = 2 * D;                 // RB: bytes of a key's row
    constexpr int TILE = BK * RB, STAGE = 2 * TILE, LI = TILE / (1024 * RW);     // bytes of a tile of keys or values, of both; load instructions of a wavefront
    constexpr int PC = RB / 16, LR = 64 / PC;                                    // pieces of a row; rows of a load instruction
    static_assert(LI >= 1 && TILE % (1024 * RW) == 0, "whole load instructions");
    using V8 = typename Elem<T>::v8;
    constexpr int ROWS_OF = 32 * RB, GROUP = 2 * STAGE;                          // bytes of a wavefront's queries or results; LDS of a group
    static_assert(RW * ROWS_OF <= STAGE, "room for the queries");
    constexpr int OUT = 64 * 4 * (16 * DT + 2);                                  // a wavefront's part on its way to another
    __shared__ __align__(16) int8_t lds[KG * GROUP];
    static_assert(KG == 1 || KG * GROUP >= (KG - 1) * RW * OUT, "room for the groups' parts");
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, li = lane & 31;
    const int rw = wv % RW, g = wv / RW;

    uint32_t hn;
    const int slot = P.slots - 1 - (int)P.heads.divide(blockIdx.x, hn);           // the last rows of a sequence, which see the most keys, come first
    const int head = P.by_xcd ? (int)(hn % NXCD) * (P.H / NXCD) + (int)hn / NXCD : (int)hn;
    const Span span = span_of<ROWS>(P.q_start, P.k_start, P.n_seq, slot, lane);
    const int seq = span.seq, qa = span.qa, qb = span.qb, ka = span.ka, kb = span.kb;
    const int tile = slot - (max(qa, 0) / ROWS + seq), nq = qb - qa, nk = kb - ka;
    if (qa < 0 || qb < qa || qb > P.n_q || ka < 0 || kb < ka || kb > P.n_k || tile < 0 || (int64_t)tile * ROWS >= nq) return;
    const int first = tile * ROWS, mine = first + 32 * rw;                        // first row of the workgroup and of the wavefront
    const int shift = nk - nq;                                                    // query i sees keys up to i + shift
    const int top_row = min(first + ROWS, nq) - 1;
    const int seen = P.causal ? min(nk, top_row + shift + 1) : nk;
    const int tiles = seen > 0 ? (seen + BK - 1) / BK : 0, rounds = (tiles + KG - 1) / KG;

    const T* const kbase = static_cast<const T*>(P.k) + (int64_t)ka * P.ldk + (int64_t)(head / P.group) * D;
    const T* const vbase = static_cast<const T*>(P.v) + (int64_t)ka * P.ldv + (int64_t)(head / P.group) * D;
    // Load instruction i of a wavefront brings rows LR (RW i + rw) + lane / PC, physical piece lane % PC.
    int8_t* const ring = lds + g * GROUP;
    const uint32_t lds0 = lds_offset(ring) + 1024 * rw;
    // rounds with tiles of which not all queries of the workgroup see all keys
    const int all_see = P.causal ? min(first + shift, nk - 1) : nk - 1;
    const int odd = (tiles - max(min((all_see + 1) / BK, tiles), 0) + KG - 1) / KG;
    // The group's tile of round n, the last keys first.  The two buffers of each operand are taken in turn, such that the first round of whole tiles has buffer 0.
    auto issue = [&](int n, auto values) __attribute__((always_inline)) {
        constexpr bool V = decltype(values)::value;
        const int kt = tiles - 1 - (n * KG + g);
        if (kt < 0) return;
        const int lr = LR * rw + lane / PC, lp = lane % PC;
        const int64_t ld = V ? P.ldv : P.ldk;
        const int8_t* const p = uniform_ptr(reinterpret_cast<const int8_t*>((V ? vbase : kbase) + (int64_t)kt * BK * ld));
        const int last = nk - 1 - kt * BK;                                        // (rows behind the sequence: its last row again)
        const uint32_t to = lds0 + (uint32_t)((n + odd) & 1) * STAGE + (V ? TILE : 0);
#pragma unroll
        for (int i = 0; i < LI; ++i) {
            const int r = LR * RW * i + lr;
            dma16(p, (uint32_t)min(r, last) * ((uint32_t)ld * 2) + 16 * (lp ^ (V ? mix_v<D>(r) : mix_k<D>(r))), to + i * 1024 * RW);
        }
    };
    constexpr std::false_type keys{};
    constexpr std::true_type values{};

    // The queries, B operand: query li, elements 16 s + 8 half on.  Their rows come whole through LDS, where the second tile will be: fragments straight from
    // memory are 32 bytes of 32 rows an instruction, and every line is asked for four times (with that of the results 32 sequences of 512, 32 heads 143 -> 128 us,
    // 32 of 128 29.0 -> 22.5).
    const int row = min(mine + li, nq - 1), limit = P.causal ? min(row + shift, nk - 1) : nk - 1;      // the last key that the lane's query sees
    const T* const qbase = static_cast<const T*>(P.q) + (int64_t)qa * P.ldq + (int64_t)head * D;
    int8_t* const rows = ring + ((odd + 1) & 1) * STAGE + rw * ROWS_OF;
    {
        const int from = min(mine, nq - 1);
        const int8_t* const p = uniform_ptr(reinterpret_cast<const int8_t*>(qbase + (int64_t)from * P.ldq));
#pragma unroll
        for (int i = 0; i < 32 / LR; ++i) {
            const int r = LR * i + lane / PC;
            dma16(p, (uint32_t)min(r, nq - 1 - from) * ((uint32_t)P.ldq * 2) + 16 * (lane % PC ^ mix_k<D>(r)), lds_offset(rows) + 1024 * i);
        }
    }
    if (rounds > 0) {
        issue(0, keys);
        issue(0, values);
    }
    if (KG == 1 && tiles > 0) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * LI) : "memory");
    else wait_vm0();                                                              // (a group may be without a tile)
    V8 qf[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s) qf[s] = *reinterpret_cast<const V8*>(rows + li * RB + 16 * ((2 * s + half) ^ mix_k<D>(li)));
    v16f acc[DT];
    float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = v16f{};
    const int sees_any = P.causal ? min(min(mine + 32, nq) - 1 + shift, nk - 1) : nk - 1;      // the last key that one of the wavefront's queries sees
    const bool idle = mine >= nq;
    int at_k[DS], at_v[DT];                                                       // where this lane's fragments lie in a tile
#pragma unroll
    for (int d = 0; d < DS; ++d) at_k[d] = li * RB + 16 * ((2 * d + half) ^ mix_k<D>(li));
#pragma unroll
    for (int i = 0; i < DT; ++i) at_v[i] = TILE + transposed_at<D>(i, lane);
    auto scores = [&](v16f (&s)[KB], int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DS; ++d)
#pragma unroll
            for (int b = 0; b < KB; ++b) s[b] = mfma(*reinterpret_cast<const V8*>(ring + at_k[d] + buf * STAGE + 32 * b * RB), qf[d], d ? s[b] : v16f{});
    };
    auto weighted = [&](const V8 (&p)[KB][2], int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 2 * KB; ++b)
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] = mfma(transposed<T, D>(ring + at_v[i] + buf * STAGE + 16 * b * RB), p[b / 2][b % 2], acc[i]);
    };

#pragma unroll 1
    for (int n = 0; n < odd; ++n) {
        const int kt = tiles - 1 - (n * KG + g), k0 = kt * BK, buf = (n + odd) & 1;
        arrive<0>();
        issue(n + 1, keys);
        issue(n + 1, values);
        if (idle || kt < 0 || k0 > sees_any) continue;
        v16f s[KB];
        scores(s, buf);
        V8 p[KB][2];
        const int rel = limit - k0 - 4 * half;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = 32 * b + 8 * (r / 4) + r % 4 > rel ? -__builtin_inff() : s[b][r];
        softmax_step<T, KB, DT>(s, p, m, l, acc, P.c);
        weighted(p, buf);
    }
    // A key left out has the weight 0, and 0 times an infinite value or NaN is NaN: where these tiles, which come first, leave a value that is not finite, they
    // are done again, key by key, with those that count only.
    if (__builtin_expect(__any(not_finite<DT>(acc)), 0))
        key_by_key<T, D>(qbase + (int64_t)row * P.ldq, kbase, P.ldk, vbase, P.ldv, max(tiles - ((odd - 1) * KG + g) - 1, 0) * BK, limit, P.c, half, m, l, acc,
                         [&](int j) { return (tiles - 1 - j / BK) % KG == g; });
    // The tiles that all queries see.  Scores are formed a tile ahead of the values' product, so that its matrix instructions stand between the vector
    // instructions of the softmax.
    if (odd < rounds) {
        arrive<0>();
        issue(odd + 1, keys);
        v16f even_s[KB], odd_s[KB];
        scores(even_s, 0);
        float top = largest_of(even_s);
        // one tile: its scores in s, the next one's into next; buf: the buffer of its values, the next keys are in the other one
        auto step = [&](int n, int buf, v16f (&s)[KB], v16f (&next)[KB]) __attribute__((always_inline)) {
            arrive<0>();
            issue(n + 2, keys);
            issue(n + 1, values);
            if (idle || (KG > 1 && n * KG + g >= tiles)) return;
            move_largest<DT>(top, m, l, acc, P.c);
            const float base = base_of<T>(m, P.c);
            V8 p[KB][2];
            scores(next, buf ^ 1);                                                // (of the last tile: of what that buffer holds, not used)
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; r += 2) weigh<T>(s[b], r, p[b], l, P.c, base);
            weighted(p, buf);
            top = largest_of(next);
        };
#pragma unroll 1
        for (int n = odd; n < rounds; n += 2) {
            step(n, 0, even_s, odd_s);
            if (n + 1 < rounds) step(n + 1, 1, odd_s, even_s);
        }
    }
    l = add_halves(l);
    if constexpr (KG > 1) {                                                       // the other groups' parts to the first, a lane's to the same lane
        __syncthreads();
        float* const out = reinterpret_cast<float*>(lds + ((g - 1) * RW + rw) * OUT) + lane;
        if (g > 0) {
            out[0] = m;
            out[64] = l;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) out[64 * (2 + 16 * i + r)] = acc[i][r];
        }
        __syncthreads();
        if (g > 0) return;
        const float* in = reinterpret_cast<const float*>(lds + rw * OUT) + lane;
        float to = m;
#pragma unroll
        for (int o = 1; o < KG; ++o) to = __builtin_fmaxf(to, in[(o - 1) * RW * OUT / 4]);
        const float f = m == to ? 1.0f : __builtin_amdgcn_exp2f((m - to) * P.c);
        l *= f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] *= f;
#pragma unroll 1
        for (int o = 1; o < KG; ++o, in += RW * OUT / 4) {
            const float h = in[0] == to ? 1.0f : __builtin_amdgcn_exp2f((in[0] - to) * P.c);
            l = __builtin_fmaf(h, in[64], l);
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] = __builtin_fmaf(h, in[64 * (2 + 16 * i + r)], acc[i][r]);
        }
    }
    // Results leave as whole rows, turned over in LDS of the wavefront's own: as they lie, a store instruction would write 16 bytes of 32 rows.
    if constexpr (KG == 1) __syncthreads();
    int8_t* const mine_l = lds + rw * (KG == 1 ? ROWS_OF : OUT);
    const float inv = l > 0.0f ? 1.0f / l : l != l ? l : 0.0f;
    typedef T v4 __attribute__((ext_vector_type(4)));
    typedef float v4f __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<v4*>(mine_l + li * RB + 16 * ((4 * i + q) ^ mix_k<D>(li)) + 8 * half) =
                __builtin_convertvector((v4f{acc[i][4 * q] * inv, acc[i][4 * q + 1] * inv, acc[i][4 * q + 2] * inv, acc[i][4 * q + 3] * inv}), v4);
    T* const obase = static_cast<T*>(P.o) + (int64_t)(qa + mine) * P.ldo + (int64_t)head * D;
#pragma unroll
    for (int i = 0; i < 32 / LR; ++i) {
        const int r = LR * i + lane / PC;
        if (mine + r < nq) *reinterpret_cast<v4i*>(obase + r * P.ldo + 8 * (lane % PC ^ mix_k<D>(r))) = *reinterpret_cast<const v4i*>(mine_l + 1024 * i + 16 * lane);
    }
}

template <class T, int D, int RW, int KG, int BK> hipError_t launch(hipStream_t s, const PromptArgs& a) {
    constexpr int ROWS = 32 * RW;
    const int64_t units = (a.n_q / ROWS + a.n_seq) * a.H;
    PaParams P{a.q, a.k, a.v, a.o, a.q_start, a.k_start, a.ldq, a.ldk, a.ldv, a.ldo, a.n_q, a.n_k, a.n_seq, a.H, a.H / a.G, a.H % NXCD == 0,
               (int)(units / a.H), a.scale * 1.44269504088896341f, a.causal, FastDiv((uint32_t)a.H)};
    prompt_attention_kernel<T, D, RW, KG, BK><<<dim3((unsigned)units), 64 * RW * KG, 0, s>>>(P);
    return hipGetLastError();
}
template <class T, int D> hipError_t choose(hipStream_t s, const PromptArgs& a) {
    switch (prompt::form_of(a.n_q, a.n_seq, a.H, a.causal, num_cus())) {
        case prompt::R64X4_K32: return launch<T, D, 2, 4, 32>(s, a);
        case prompt::R64_K32: return launch<T, D, 2, 1, 32>(s, a);
        case prompt::R128X2_K64: return launch<T, D, 4, 2, 64>(s, a);
        default: return launch<T, D, 4, 1, 64>(s, a);
    }
}

}  // namespace

hipError_t launch_prompt_attention(hipStream_t s, const PromptArgs& a) {
    // (the sequences' lengths are not known here: all keys for every query of one sequence, half of them where causal)
    const int64_t pairs = a.n_seq ? a.n_q * (a.n_k / a.n_seq) / (a.causal ? 2 : 1) : 0;
    TraceScope trace(s, KIND_PROMPT_ATTENTION, 4 * pairs * a.H * a.d, 4 * a.d * (a.n_q * a.H + a.n_k * a.G));
    if (a.type == TYPE_F16) return a.d == 64 ? choose<_Float16, 64>(s, a) : choose<_Float16, 128>(s, a);
    return a.d == 64 ? choose<__bf16, 64>(s, a) : choose<__bf16, 128>(s, a);
}

}  // namespace ivit
