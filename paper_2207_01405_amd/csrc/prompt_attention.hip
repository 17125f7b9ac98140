// Attention over whole prompts on the gfx950 matrix cores: packed sequences, grouped heads, causal or not.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c (q_i . k_j - m_i)),   c = scale log2 e,  m_i the largest score so far
//
// One pass over the keys, 64 at a time, with the running maximum and sum of the softmax.  Scores are formed transposed, keys x queries: an MFMA
// result lane then holds scores of ONE query, so that maximum, sum and the rescaling of the output are a lane's own (one exchange between the halves
// of a wavefront joins the maximum), and its registers, rounded and packed, are as they stand the "B" operand of the second product, values x queries:
// that product sums over keys, in any order that both operands agree on, and the values' fragments come by the transposing LDS read in the order
// in which the scores' registers hold the keys.
#include "regst_common.hpp"
#include "float_attention.hpp"

namespace ivit {
namespace {

using namespace regst;
using namespace fatt;

struct PaParams {
    const void *q, *k, *v; void* o; const int32_t *q_start, *k_start; int64_t ldq, ldk, ldv, ldo, n_q, n_k;
    int n_seq, H, group, by_xcd, slots; float c; int causal; FastDiv heads;
};

// The sequence of tile slot x: sequence s has the slots q_start[s] / ROWS + s on, which are enough for its rows whatever they begin at.  64 places are
// looked at at once.
template <int ROWS> __device__ __forceinline__ int sequence_of(const int32_t* start, int n_seq, int x, int lane) {
    int lo = 0, n = n_seq;                                          // it is one of lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 63) / 64, s = lo + lane * step;
        const bool behind = lane * step < n && (max(start[s], 0) / ROWS + s) <= x;
        const int at = 63 - __builtin_clzll(__ballot(behind) | 1);
        lo += at * step;
        n = min(step, n - at * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

template <class T, int D, int W, int QT>
__global__ __launch_bounds__(64 * W) void prompt_attention_kernel(PaParams P) {
    constexpr int ROWS = 32 * QT * W, BK = 64, KB = BK / 32, DS = D / 16, DT = D / 32, RB = 2 * D;     // RB: bytes of a key's row
    constexpr int TILE = BK * RB, S = 2, LI = TILE / (1024 * W);                 // bytes of a tile of keys or values; stages; load instructions of a wavefront
    constexpr int PC = RB / 16, LR = 64 / PC;                                    // pieces of a row; rows of a load instruction
    using V8 = typename Elem<T>::v8;
    __shared__ __align__(16) int8_t lds[S * 2 * TILE];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, li = lane & 31;

    uint32_t hn;
    const int slot = P.slots - 1 - (int)P.heads.divide(blockIdx.x, hn);             // the last rows of a sequence, which see the most keys, come first
    const int head = P.by_xcd ? (int)(hn % NXCD) * (P.H / NXCD) + (int)hn / NXCD : (int)hn;
    const int seq = sequence_of<ROWS>(P.q_start, P.n_seq, slot, lane);
    const int qa = P.q_start[seq], qb = P.q_start[seq + 1], ka = P.k_start[seq], kb = P.k_start[seq + 1];
    const int tile = slot - (max(qa, 0) / ROWS + seq), nq = qb - qa, nk = kb - ka;
    if (qa < 0 || qb < qa || qb > P.n_q || ka < 0 || kb < ka || kb > P.n_k || tile < 0 || (int64_t)tile * ROWS >= nq) return;
    const int first = tile * ROWS, mine = first + 32 * QT * wv;                   // first row of the workgroup and of the wavefront
    const int shift = nk - nq;                                                    // query i sees keys up to i + shift
    const int top_row = min(first + ROWS, nq) - 1;
    const int seen = P.causal ? min(nk, top_row + shift + 1) : nk;
    const int tiles = seen > 0 ? (seen + BK - 1) / BK : 0;

    const T* const kbase = static_cast<const T*>(P.k) + (int64_t)ka * P.ldk + (int64_t)(head / P.group) * D;
    const T* const vbase = static_cast<const T*>(P.v) + (int64_t)ka * P.ldv + (int64_t)(head / P.group) * D;
    // Load instruction i of a wavefront brings rows LR (W i + wavefront) + lane / PC, physical piece lane % PC.
    const int lr = LR * wv + lane / PC, lp = lane % PC;
    const uint32_t ldk2 = (uint32_t)P.ldk * 2, ldv2 = (uint32_t)P.ldv * 2;
    const uint32_t kpiece = 16 * (lp ^ mix_k<D>(lr)), vpiece = 16 * (lp ^ mix_v<D>(lr));
    const uint32_t lds0 = lds_offset(lds) + 1024 * wv;
    // tile n of the order in which they are taken, the last keys first; keys into buffer n % 2 of theirs, values likewise
    auto issue = [&](int n, auto values) __attribute__((always_inline)) {
        constexpr bool V = decltype(values)::value;
        const int kt = tiles - 1 - n;
        const int64_t ld = V ? P.ldv : P.ldk;
        const int8_t* const p = uniform_ptr(reinterpret_cast<const int8_t*>((V ? vbase : kbase) + (int64_t)kt * BK * ld));
        const int last = nk - 1 - kt * BK;                                        // (rows behind the sequence: its last row again)
        const uint32_t to = lds0 + (n & 1) * 2 * TILE + (V ? TILE : 0);
#pragma unroll
        for (int i = 0; i < LI; ++i) dma16(p, (uint32_t)min(LR * W * i + lr, last) * (V ? ldv2 : ldk2) + (V ? vpiece : kpiece), to + i * 1024 * W);
    };
    constexpr std::false_type keys{};
    constexpr std::true_type values{};
    if (tiles > 0) {
        issue(0, keys);
        issue(0, values);
    }

    // the queries: B operand, query li, elements 16 s + 8 half on
    V8 qf[QT][DS];
    int limit[QT];                                                                // the last key that the lane's query sees
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int row = min(mine + 32 * t + li, nq - 1);
        limit[t] = P.causal ? min(row + shift, nk - 1) : nk - 1;
        const T* const qp = static_cast<const T*>(P.q) + (int64_t)(qa + row) * P.ldq + (int64_t)head * D + 8 * half;
#pragma unroll
        for (int s = 0; s < DS; ++s) qf[t][s] = *reinterpret_cast<const V8*>(qp + 16 * s);
    }
    v16f acc[QT][DT];
    float m[QT], l[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = -__builtin_inff();
        l[t] = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[t][i] = v16f{};
    }
    const int sees_any = P.causal ? min(min(mine + 32 * QT, nq) - 1 + shift, nk - 1) : nk - 1;
    const bool idle = mine >= nq;
    // tiles of which not all queries of the workgroup see all keys
    const int all_see = P.causal ? min(first + shift, nk - 1) : nk - 1;
    const int odd = tiles - max(min((all_see + 1) / BK, tiles), 0);

    int at_k[DS], at_v[DT];                                                       // where this lane's fragments lie in a tile
#pragma unroll
    for (int d = 0; d < DS; ++d) at_k[d] = li * RB + 16 * ((2 * d + half) ^ mix_k<D>(li));
#pragma unroll
    for (int i = 0; i < DT; ++i) at_v[i] = TILE + transposed_at<D>(i, lane);
    auto key_frag = [&](int buf, int b, int d) __attribute__((always_inline)) {
        return *reinterpret_cast<const V8*>(lds + at_k[d] + buf * 2 * TILE + 32 * b * RB);
    };
    auto value_frag = [&](int buf, int b, int i) __attribute__((always_inline)) { return transposed<T, D>(lds + at_v[i] + buf * 2 * TILE + 16 * b * RB); };
    auto scores = [&](v16f (&s)[QT][KB], int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DS; ++d)
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const V8 kf = key_frag(buf, b, d);
#pragma unroll
                for (int t = 0; t < QT; ++t) s[t][b] = mfma(kf, qf[t][d], d ? s[t][b] : v16f{});
            }
    };

#pragma unroll 1
    for (int n = 0; n < odd; ++n) {
        const int k0 = (tiles - 1 - n) * BK, buf = n & 1;
        arrive<0>();
        if (n + 1 < tiles) {
            issue(n + 1, keys);
            issue(n + 1, values);
        }
        if (idle || k0 > sees_any) continue;
        v16f s[QT][KB];
        scores(s, buf);
        V8 p[QT][KB][2];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int rel = limit[t] - k0 - 4 * half;
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][b][r] = 32 * b + 8 * (r / 4) + r % 4 > rel ? -__builtin_inff() : s[t][b][r];
            softmax_step<T, KB, DT>(s[t], p[t], m[t], l[t], acc[t], P.c);
        }
#pragma unroll
        for (int b = 0; b < 2 * KB; ++b)
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const V8 vf = value_frag(buf, b, i);
#pragma unroll
                for (int t = 0; t < QT; ++t) acc[t][i] = mfma(vf, p[t][b / 2][b % 2], acc[t][i]);
            }
        // A key left out has the weight 0, and 0 times an infinite value or NaN is NaN: where these tiles, which come first, leave a value that is
        // not finite, they are done again, key by key, with those that count only.
#pragma unroll
        for (int t = 0; t < QT; ++t)
            if (__builtin_expect(__any(not_finite<DT>(acc[t])), 0)) {
                const int row = min(mine + 32 * t + li, nq - 1);
                key_by_key<T, D>(static_cast<const T*>(P.q) + (int64_t)(qa + row) * P.ldq + (int64_t)head * D, kbase, P.ldk, vbase, P.ldv, k0, limit[t],
                                 P.c, half, m[t], l[t], acc[t]);
            }
    }
    // The tiles that all queries see.  Scores are formed a tile ahead of the values' product, so that its matrix instructions stand between the vector
    // instructions of the softmax.
    if (odd < tiles) {
        arrive<0>();
        if (odd + 1 < tiles) issue(odd + 1, keys);
        v16f even_s[QT][KB], odd_s[QT][KB];
        float top[QT];
        // one tile: its scores in s, the next one's into next; buf: the buffer of its values, the next keys are in the other one
        auto step = [&](int n, auto buf_c, v16f (&s)[QT][KB], v16f (&next)[QT][KB]) __attribute__((always_inline)) {
            constexpr int buf = decltype(buf_c)::value;
            arrive<0>();
            if (n + 2 < tiles) issue(n + 2, keys);
            if (n + 1 < tiles) issue(n + 1, values);
            float base[QT];
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                move_largest<DT>(top[t], m[t], l[t], acc[t], P.c);
                base[t] = base_of<T>(m[t], P.c);
            }
            V8 p[QT][KB][2];
            scores(next, buf ^ 1);                                                // (of the last tile: of what the other buffer holds, not used)
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int r = 0; r < 16; r += 2) weigh<T>(s[t][b], r, p[t][b], l[t], P.c, base[t]);
#pragma unroll
            for (int b = 0; b < 2 * KB; ++b)
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const V8 vf = value_frag(buf, b, i);
#pragma unroll
                    for (int t = 0; t < QT; ++t) acc[t][i] = mfma(vf, p[t][b / 2][b % 2], acc[t][i]);
                }
#pragma unroll
            for (int t = 0; t < QT; ++t) top[t] = largest_of(next[t]);
#ifdef SCHED
            SCHED
#endif
        };
        constexpr std::integral_constant<int, 0> b0{};
        constexpr std::integral_constant<int, 1> b1{};
        int n = odd;
        if (n & 1) {
            scores(odd_s, 1);
#pragma unroll
            for (int t = 0; t < QT; ++t) top[t] = largest_of(odd_s[t]);
            step(n, b1, odd_s, even_s);
            ++n;
        } else {
            scores(even_s, 0);
#pragma unroll
            for (int t = 0; t < QT; ++t) top[t] = largest_of(even_s[t]);
        }
#pragma unroll 1
        for (; n + 1 < tiles; n += 2) {
            step(n, b0, even_s, odd_s);
            step(n + 1, b1, odd_s, even_s);
        }
        if (n < tiles) step(n, b0, even_s, odd_s);
    }
    if (idle) return;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const float total = add_halves(l[t]), inv = total > 0.0f ? 1.0f / total : total != total ? total : 0.0f;
        const int row = mine + 32 * t + li;
        if (row < nq) store_rows<T, DT>(static_cast<T*>(P.o) + (int64_t)(qa + row) * P.ldo + (int64_t)head * D, acc[t], inv, half);
    }
}

template <class T, int D> hipError_t launch(hipStream_t s, const PromptArgs& a) {
    constexpr int W = 4, QT = 1, ROWS = 32 * QT * W;
    const int64_t units = (a.n_q / ROWS + a.n_seq) * a.H;
    PaParams P{a.q, a.k, a.v, a.o, a.q_start, a.k_start, a.ldq, a.ldk, a.ldv, a.ldo, a.n_q, a.n_k, a.n_seq, a.H, a.H / a.G, a.H % NXCD == 0,
               (int)(units / a.H), a.scale * 1.44269504088896341f, a.causal, FastDiv((uint32_t)a.H)};
    prompt_attention_kernel<T, D, W, QT><<<dim3((unsigned)units), 64 * W, 0, s>>>(P);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attention(hipStream_t s, const PromptArgs& a) {
    // (the sequences' lengths are not known here: all keys for every query of one sequence, half of them where causal)
    const int64_t pairs = a.n_seq ? a.n_q * (a.n_k / a.n_seq) / (a.causal ? 2 : 1) : 0;
    TraceScope trace(s, KIND_PROMPT_ATTENTION, 4 * pairs * a.H * a.d, 4 * a.d * (a.n_q * a.H + a.n_k * a.G));
    if (a.type == TYPE_F16) return a.d == 64 ? launch<_Float16, 64>(s, a) : launch<_Float16, 128>(s, a);
    return a.d == 64 ? launch<__bf16, 64>(s, a) : launch<__bf16, 128>(s, a);
}

}  // namespace ivit
