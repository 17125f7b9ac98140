// int8 x int8 -> int32 Dense on the gfx950 matrix cores with real scales and the epilogue of a float layer:
//   y[m][n] = act(s_x[m] s_w[n] sum_k x[m][k] w[n][k] + bias[n]) + r[m][n]
//
// A workgroup of GM x GN wavefronts computes tiles of 32 MT GM tokens x 32 NT GN channels.  Both operands stream through S LDS
// stages of 128 bytes of K, filled by LDS-direct loads (no register pass, one barrier per stage); the 16-byte pieces of a row are
// permuted by an XOR with bits of the row number, so that the fragment reads are spread over the banks.  The weights are the MFMA "A"
// operand and the loads put the channel rows in such an order that a lane ends up with 16 NT consecutive channels of one token.
//
// What bounds the tiles is LDS, 128 bytes a cycle and CU for fragment reads and arriving loads alike: a stage of two 128 x 128 tiles a CU is
// 1536 cycles of it for 1024 of products and takes 0.99 us, one of 256 x 256 (eight wavefronts of 128 x 64) 2048 for 2048 and 1.57 us at the
// 1.7 GHz that this card keeps up then.  8192 x 8192 x 4096 with bf16 results 224 to 229 us, 2.4 POP/s (a product alone from registers runs at 3.2
// to 3.3 on random data); with the residual 249 to 252.  Tried for 256 x 256 and taken back: four wavefronts of 128 x 128,
// a quarter less LDS (497 against 465 us at K = 8192, then 461 against 451); stages of 64 bytes, four of them (473 against 451: half lines);
// the residual's lines requested into L2 during the last stages (286 against 281) or a pass ahead (290 against 286); wave priorities (no change).
#include "linear_rows.hpp"
#include "regst_common.hpp"
#include "scaled_common.hpp"
#include "scaled_form.hpp"

namespace ivit {
namespace {

using namespace regst;
using namespace scaled;

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int BK = 128, LR = 1024 / BK, PC = BK / 16;      // bytes of K per stage; rows a load instruction fills; 16-byte pieces of a row

// Tiles in bands of `height` rows of tiles, column by column within a band; each XCD takes a contiguous range of that order.  What
// an XCD works on at one time is then a patch of the result about as high as wide, and its L2 takes in the fewest rows of either operand.
struct TileOrder {
    FastDiv band, full, last;                  // tiles of a band; its height; that of the last one
    uint32_t tiles, per_xcd, last_band;
    __device__ __forceinline__ void tile(uint32_t t, uint32_t& tm, uint32_t& tn) const {
        uint32_t in, row;
        const uint32_t b = band.divide(t, in);
        tn = b == last_band ? last.divide(in, row) : full.divide(in, row);
        tm = b * full.d + row;
    }
    TileOrder() = default;
    TileOrder(uint32_t rows, uint32_t cols, uint32_t height)
        : band(height * cols), full(height), last((rows - 1) % height + 1), tiles(rows * cols), per_xcd((rows * cols + NXCD - 1) / NXCD),
          last_band((rows - 1) / height) {}
};

struct GsParams {
    const int8_t* x; const float* x_scale; const int8_t* w; const float* w_scale; const float* bias; const void* residual; void* y;
    int64_t ldx, ld_res, ldy, M; int N, K, act, one_scale, once; float inv_step;
    TileOrder order;
};

template <int TYPE> using Stored = std::conditional_t<TYPE == TYPE_F32, float, std::conditional_t<TYPE == TYPE_F16, _Float16,
                                   std::conditional_t<TYPE == TYPE_BF16, __bf16, int8_t>>>;

// A chunk: the 16 bytes of 16, 8 or 4 consecutive results of a row.
template <int TYPE> struct Chunk {
    using T = Stored<TYPE>;
    static constexpr int E = 16 / (int)sizeof(T);
    typedef float vf __attribute__((ext_vector_type(E)));
    typedef T vt __attribute__((ext_vector_type(E)));
    typedef T mem __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    static __device__ __forceinline__ v4i pack(vf v, float inv_step) {
        if constexpr (TYPE == TYPE_I8) {
            v4i o;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint32_t q[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) q[e] = (uint32_t)clamp8((int32_t)__builtin_rintf(v[4 * d + e] * inv_step));     // (NaN: 0)
                o[d] = (int)pack4(q[0], q[1], q[2], q[3]);
            }
            return o;
        } else {
            return __builtin_bit_cast(v4i, __builtin_convertvector(v, vt));
        }
    }
    static __device__ __forceinline__ vf unpack(v4i v) { return __builtin_convertvector(__builtin_bit_cast(vt, v), vf); }
    // a chunk past the L2, and one stored there
    static __device__ __forceinline__ v4i load_once(const T* p) { return __builtin_bit_cast(v4i, (vt)__builtin_nontemporal_load(reinterpret_cast<const mem*>(p))); }
    // the chunk at p, which may have the alignment of one element; of it n elements count, and `there` exist
    static __device__ __forceinline__ v4i load(const T* p, int n, int64_t there) {
        if (n >= E || there >= E) return __builtin_bit_cast(v4i, (vt)*reinterpret_cast<const mem*>(p));
        vt v = {};
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
            if (e < n) v[e] = p[e];
        return __builtin_bit_cast(v4i, v);
    }
    static __device__ __forceinline__ void store_once(T* p, v4i w) { __builtin_nontemporal_store(__builtin_bit_cast(vt, w), reinterpret_cast<mem*>(p)); }
    static __device__ __forceinline__ void store(T* p, v4i w, int n) {
        const vt v = __builtin_bit_cast(vt, w);
        if (n >= E) { *reinterpret_cast<mem*>(p) = v; return; }
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
            if (e < n) p[e] = v[e];
    }
};

template <int MT, int NT, int GM, int GN> struct GsTile {
    static constexpr int W = GM * GN, TM = 32 * MT * GM, TN = 32 * NT * GN;
    static_assert(TM % (LR * W) == 0 && TN % (LR * W) == 0, "a load instruction of all wavefronts fills rows of one operand");
    static_assert(TN % 64 == 0 && TN / 64 <= W && TM % 64 == 0 && TM / 64 <= W, "the constants of 64 channels or rows a wavefront");
};

template <int TYPE, int MT, int NT, int GM, int GN, int S>
__global__ __launch_bounds__((64 * GM * GN), 2) void gemm_scaled_kernel(GsParams P) {
    using TL = GsTile<MT, NT, GM, GN>;
    using T = Stored<TYPE>;
    constexpr int W = TL::W, TM = TL::TM, TN = TL::TN, XI = TM / (LR * W), WI = TN / (LR * W), DP = XI + WI, STG = (TM + TN) * BK;
    // PIPE: the tiles of four products a k-step and more; PERSIST: a workgroup goes on to its next tile, whose first stage comes in
    // under the epilogue of the present one
    constexpr bool PIPE = MT * NT >= 4, PERSIST = PIPE && S == 2;
    __shared__ __align__(16) int8_t lds[S * STG];
    __shared__ __align__(16) float ws_s[PERSIST ? 2 : 1][TN], bias_s[PERSIST ? 2 : 1][TN], xs_s[PERSIST ? 2 : 1][TM];

    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wv / GN, wn = wv % GN;

    // each XCD takes a contiguous range of tiles, each of its workgroups every `slots`th of them
    const uint32_t slots = gridDim.x / NXCD, end = min((blockIdx.x % NXCD + 1) * P.order.per_xcd, P.order.tiles);
    uint32_t tile = (blockIdx.x % NXCD) * P.order.per_xcd + blockIdx.x / NXCD;
    if (tile >= end) return;
    const int K = P.K, N = P.N;
    struct Place { int64_t m0; int n0, rows; };
    auto place = [&](uint32_t t) __attribute__((always_inline)) {
        uint32_t tm, tn;
        P.order.tile(t, tm, tn);
        const int64_t m0 = (int64_t)tm * TM;
        return Place{m0, (int)tn * TN, (int)min64(P.M - m0, TM)};
    };

    // (32-bit offsets from the tile's first row: 255 rows of at most 2^22 bytes)
    // Load instruction i of a wavefront fills LDS rows LR (W i + wavefront) + lane / PC, PC lanes a row; the lane lands in physical
    // piece p = lane % PC of row r and fetches piece p ^ mix(r).  Rows past the last token or channel repeat it (never stored),
    // pieces past the end of a row its last piece (never multiplied, see below).
    auto mix = [](int r) __attribute__((always_inline)) { return (r >> 1) & (PC - 1); };
    // a copy of the lane's number that the compiler takes for another one at every use: what is formed from it anew for every tile would
    // else be kept in registers all along
    auto lane_now = [&]() __attribute__((always_inline)) {
        int l = lane;
        if (PERSIST) asm volatile("" : "+v"(l));
        return l;
    };
    const int ld_col = 16 * ((lane % PC) ^ mix(LR * wv + lane / PC));
    const int stages = (K + BK - 1) / BK, k_last = K - (stages - 1) * BK;      // bytes of K in the last stage: 16 .. BK
    uint32_t off[DP];
    bool off_whole = false;
    v4i x_buf, w_buf;
    int is = 0;
    uint32_t k_off = 0;
    auto buffer = [](const int8_t* p) __attribute__((always_inline)) {
        const uint64_t a = (uint64_t)uniform_ptr(p);
        return v4i{(int)(uint32_t)a, (int)(uint32_t)(a >> 32), (int)kTileBytes, 0x00020000};
    };
    // where the loads of a tile find their rows; the constants of its channels and rows, 64 a wavefront
    auto aim = [&](const Place& at, int par) __attribute__((always_inline)) {
        const int lane = lane_now(), ld_r = LR * wv + lane / PC, ld_col = 16 * ((lane % PC) ^ mix(ld_r));
        if (wv < TN / 64) {
            const uint32_t o = 4u * min(at.n0 + 64 * wv + lane, N - 1);
            dma4(uniform_ptr(reinterpret_cast<const int8_t*>(P.w_scale)), o, lds_offset(reinterpret_cast<const int8_t*>(ws_s[par] + 64 * wv)));
            if (P.bias) dma4(uniform_ptr(reinterpret_cast<const int8_t*>(P.bias)), o, lds_offset(reinterpret_cast<const int8_t*>(bias_s[par] + 64 * wv)));
            else bias_s[par][64 * wv + lane] = 0.0f;
        }
        if (wv < TM / 64)
            dma4(uniform_ptr(reinterpret_cast<const int8_t*>(P.x_scale + (P.one_scale ? 0 : at.m0))), P.one_scale ? 0u : 4u * min(64 * wv + lane, at.rows - 1),
                 lds_offset(reinterpret_cast<const int8_t*>(xs_s[par] + 64 * wv)));
        // (whole tiles have the same offsets from their first rows)
        const bool whole = at.rows == TM && at.n0 + TN <= N && k_last == BK;
        if (!(whole && off_whole))
#pragma unroll
        for (int i = 0; i < DP; ++i) {
            if (i < XI) {
                off[i] = (uint32_t)min(LR * W * i + ld_r, at.rows - 1) * (uint32_t)P.ldx + ld_col;
            } else {
                // row 8 q + 4 g + r of MFMA tile ct holds channel 16 NT g + 16 ct + 4 q + r of the wavefront's 32 NT: that is
                // accumulator register 4 q + r of lane group g
                const int R = LR * W * (i - XI) + ld_r, ct = (R >> 5) % NT, rr = R & 31;
                const int ch = (R / (32 * NT)) * 32 * NT + 16 * NT * ((rr >> 2) & 1) + 16 * ct + 4 * (rr >> 3) + (rr & 3);
                off[i] = (uint32_t)min(ch, N - 1 - at.n0) * (uint32_t)K + ld_col;
            }
        }
        off_whole = whole;
        x_buf = buffer(P.x + at.m0 * P.ldx);
        w_buf = buffer(P.w + (int64_t)at.n0 * K);
        is = 0;
        k_off = 0;
    };
    const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds_offset(lds) + wv * 1024));
    // A stage's loads: stage `is` goes to buffer is % S, known where the loads stand.  A lane whose piece lies past the end of
    // the rows moves back to the last one (the last stage only).  One scalar offset serves both operands.
    const int back = max(ld_col - (k_last - 16), 0), moves = k_last < BK ? stages - 1 : -1;
    auto issue = [&](auto buf_c) __attribute__((always_inline)) {
        if (is == moves) {
#pragma unroll
            for (int i = 0; i < DP; ++i) off[i] -= back;
        }
        static_for<DP>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value;
            load_lds<decltype(buf_c)::value * STG + i * W * 1024>(i < XI ? x_buf : w_buf, off[i], k_off, lds0);
        });
        ++is;
        k_off += BK;
    };
    Place at = place(tile);
    aim(at, 0);
    if constexpr (PERSIST) {
        issue(std::integral_constant<int, 0>());
        wait_vm0();
    }
    v16i acc[NT][MT];
    constexpr int KS = BK / 32, AHEAD = MT * NT == 1 ? KS : 2;      // fragments are read AHEAD - 1 k-steps before their use
    int fx[KS], fw[KS];                                   // where this lane's fragments of k-step kk lie (buffer 0)
    struct Frag { v4i a[NT], b[MT]; };
    // fragment i of k-step kk, in the order of their use: the first of the weights, those of the tokens, the other ones
    auto read_one = [&](Frag& f, int i, int kk, int buf) __attribute__((always_inline)) {
        if (i >= 1 && i <= MT) f.b[i - 1] = *reinterpret_cast<const v4i*>(lds + fx[kk] + buf * STG + (i - 1) * 32 * BK);
        else f.a[i ? i - MT : 0] = *reinterpret_cast<const v4i*>(lds + fw[kk] + buf * STG + (i ? i - MT : 0) * 32 * BK);
    };
    auto read_frag = [&](Frag& f, int kk, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NT + MT; ++i) read_one(f, i, kk, buf);
    };
    auto multiply = [&](const Frag& f) __attribute__((always_inline)) {
#pragma unroll
        for (int ct = 0; ct < NT; ++ct)
#pragma unroll
            for (int tt = 0; tt < MT; ++tt) acc[ct][tt] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.a[ct], f.b[tt], acc[ct][tt], 0, 0, 0);
    };
    static_assert(S >= 2 && S <= 4 && (S - 1) * DP + 2 <= 63, "wait counts");
    const int full = k_last == BK ? stages : stages - 1;  // a last stage of less than 128 bytes comes after the loop
    // all loads but those of the `left` stages requested last have arrived, and LDS reads returned, for everybody
    auto arrive_but = [&](int left) __attribute__((always_inline)) {
        if (left <= 0) arrive<0>();
        else if (left == 1) arrive<DP>();
        else arrive<2 * DP>();
    };
    // The epilogue turns results over in LDS (see there), SLOTS times 32 tokens at once.
    using CK = Chunk<TYPE>;
    constexpr int RB = 32 * NT * (int)sizeof(T), CH = RB / 16, MINE = NT * (int)sizeof(T);     // bytes and chunks of a row; a lane's chunks
    constexpr int REGION = (PERSIST ? STG : S * STG) / W / 1024 * 1024, FIT = REGION / (32 * RB);
    constexpr int SLOTS = FIT >= MT && MT * RB <= 512 ? MT : FIT >= 2 && MT % 2 == 0 && RB <= 128 ? 2 : 1;     // (registers for a residual's chunks)
    constexpr int MOVES = RB / 32;                        // instructions of 64 chunks that move a slot
    static_assert(FIT >= 1 && MT % SLOTS == 0, "room for 32 rows");
    // chunk i of a lane when rows move: row MV_ROWS i + lane / CH of the slots, channels from E (lane % CH) on
    constexpr int MV_ROWS = 64 / CH;
#pragma unroll 1
    for (int par = 0;; par ^= PERSIST) {
        constexpr bool EARLY = !PIPE && TYPE != TYPE_I8;      // a residual is requested first: such launches are a chain of latencies
        v4i early[EARLY ? MT / SLOTS : 1][EARLY ? SLOTS * MOVES : 1];
        // Where the last channels are not a whole chunk, what follows them, the next row's, is loaded with them; only behind the last row of all
        // there may be nothing: (rows behind this one) ld + (channels from the chunk on) elements follow.
        if constexpr (EARLY) {
            if (P.residual) {
                const int c = at.n0 + wn * 32 * NT + CK::E * (lane % CH);
                const T* const res = static_cast<const T*>(P.residual) + at.m0 * P.ld_res + c;
#pragma unroll
                for (int p = 0; p < MT / SLOTS; ++p)
#pragma unroll
                    for (int i = 0; i < SLOTS * MOVES; ++i) {
                        const int row = min(wm * 32 * MT + 32 * SLOTS * p + MV_ROWS * i + lane / CH, at.rows - 1);
                        early[p][i] = v4i{0, 0, 0, 0};
                        if (c < N) early[p][i] = CK::load(res + row * P.ld_res, N - c, (P.M - 1 - at.m0 - row) * P.ld_res + N - c);
                    }
            }
        }
        if constexpr (PERSIST) {                              // stage 0 has arrived; the other buffer served the last epilogue
            __syncthreads();
            if (1 < stages) issue(std::integral_constant<int, 1>());
        } else {
            static_for<PIPE ? S : S - 1>([&](auto buf) __attribute__((always_inline)) {
                if (decltype(buf)::value < stages) issue(buf);
            });
        }
#pragma unroll
        for (int ct = 0; ct < NT; ++ct)
#pragma unroll
            for (int tt = 0; tt < MT; ++tt) acc[ct][tt] = sums_from(0);
        int s = 0;
        {
            const int ln = lane_now(), li = ln & 31, lg = ln >> 5;
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
                const int col = 16 * ((2 * kk + lg) ^ mix(li));
                fx[kk] = (wm * 32 * MT + li) * BK + col;
                fw[kk] = (TM + wn * 32 * NT + li) * BK + col;
            }
        }
        if constexpr (PIPE) {
            // All S buffers are filled to begin with.  In front of the last k-step of stage s, whose fragments are in registers then, stage
            // s + 1 has to have arrived; behind the barrier there nobody reads stage s any more: its buffer takes stage s + S, and the first
            // fragments of stage s + 1 come under the products of that last k-step.  So no stage begins with a wait.  Reads and requests stand
            // one by one between the products: a wavefront issues in order, and eight reads at a stretch hold it for longer than a product takes.
            Frag f[2];
            if constexpr (!PERSIST) arrive_but(stages >= S ? S - 1 : 0);
            read_frag(f[0], 0, 0);
            auto body = [&](auto buf_c, auto more_c) __attribute__((always_inline)) {
                constexpr int buf = decltype(buf_c)::value, nb = (buf + 1) % S;
                constexpr bool MORE = decltype(more_c)::value;            // there is a stage s + S (false: maybe)
                static_for<KS>([&](auto kk_c) __attribute__((always_inline)) {
                    constexpr int kk = decltype(kk_c)::value;
                    constexpr bool last = kk == KS - 1;
                    if constexpr (last) {
                        if constexpr (MORE) {
                            arrive<(S - 2) * DP>();
                            if (is == moves) {
#pragma unroll
                                for (int i = 0; i < DP; ++i) off[i] -= back;
                            }
                        } else if (s + 1 < stages) {
                            arrive_but(min(stages - 2 - s, S - 2));
                            if (is < stages) issue(buf_c);
                        }
                    }
                    constexpr int READS = NT + MT, DO = READS + (last && MORE ? DP : 0), N_MUL = NT * MT;
                    static_for<N_MUL>([&](auto i_c) __attribute__((always_inline)) {
                        constexpr int i = decltype(i_c)::value, ct = i / MT, tt = i % MT;
                        acc[ct][tt] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f[kk & 1].a[ct], f[kk & 1].b[tt], acc[ct][tt], 0, 0, 0);
                        constexpr int from = i * DO / N_MUL, to = (i + 1) * DO / N_MUL;
                        static_for<to - from>([&](auto d_c) __attribute__((always_inline)) {
                            constexpr int d = from + decltype(d_c)::value;
                            if constexpr (d < READS) read_one(f[(kk + 1) & 1], d, last ? 0 : kk + 1, last ? nb : buf);
                            else load_lds<buf * STG + (d - READS) * W * 1024>(d - READS < XI ? x_buf : w_buf, off[d - READS], k_off, lds0);
                        });
                        __builtin_amdgcn_sched_barrier(0);
                    });
                    if constexpr (last && MORE) { ++is; k_off += BK; }
                });
                ++s;
            };
            static_assert(KS % 2 == 0, "the first fragments of every stage go to the same registers");
#pragma unroll 1
            while (s + 2 * S <= stages)
                static_for<S>([&](auto buf) __attribute__((always_inline)) { body(buf, std::true_type()); });
#pragma unroll 1
            while (s < full)
                static_for<S>([&](auto buf) __attribute__((always_inline)) { if (s < full) body(buf, std::false_type()); });
        } else {
            // Stage s: its loads have arrived when at most those of the later stages requested so far (S - 2, fewer at the end)
            // are outstanding; behind the barrier nobody reads stage s - 1 any more and its buffer takes stage s + S - 1.  Those
            // loads go out behind the first fragment reads.
            auto body = [&](auto buf_c) __attribute__((always_inline)) {
                constexpr int buf = decltype(buf_c)::value;
                arrive_but(min(stages - 1 - s, S - 2));
                Frag f[AHEAD];
                static_for<AHEAD - 1>([&](auto kk) __attribute__((always_inline)) { read_frag(f[decltype(kk)::value], decltype(kk)::value, buf); });
                if (is < stages) issue(std::integral_constant<int, (buf + S - 1) % S>());
                static_for<KS>([&](auto kk_c) __attribute__((always_inline)) {
                    constexpr int kk = decltype(kk_c)::value;
                    if constexpr (kk + AHEAD - 1 < KS) read_frag(f[(kk + AHEAD - 1) % AHEAD], kk + AHEAD - 1, buf);
                    multiply(f[kk % AHEAD]);
                });
                ++s;
            };
#pragma unroll 1
            while (s < full)
                static_for<S>([&](auto buf) __attribute__((always_inline)) { if (s < full) body(buf); });
        }
        if (full < stages) {                                  // what is left of K; of its last 32 bytes maybe the first half only
            arrive<0>();
            const int buf = s % S;
            static_for<KS>([&](auto kk_c) __attribute__((always_inline)) {
                constexpr int kk = decltype(kk_c)::value;
                if (32 * kk >= k_last) return;
                Frag f;
                read_frag(f, kk, buf);
                if (32 * kk + 16 >= k_last && lane >= 32) {
#pragma unroll
                    for (int ct = 0; ct < NT; ++ct) f.a[ct] = v4i{0, 0, 0, 0};
                }
                multiply(f);
            });
        }

        // ---- epilogue.  A lane has 16 NT consecutive channels of a token, and its neighbour those of the next one: stored from there, every
        // instruction would touch 64 lines and fill none.  So a wavefront turns its results over in LDS that it has for itself
        // (REGION bytes), SLOTS times 32 tokens at once, and lines leave whole; a residual comes in the same way.  Chunk c of a row
        // stands at c ^ swz(row), which spreads rows over the banks.
        auto swz = [](int r) __attribute__((always_inline)) { return (CH >= 8 ? r : r / (CH < 8 ? 8 / CH : 1)) & (CH - 1); };
        __syncthreads();                                      // (nobody reads operands any more)
        const bool more_tiles = PERSIST && tile + slots < end;
        Place next = at;
        if constexpr (PERSIST) {
            if (more_tiles) {
                next = place(tile + slots);
                aim(next, par ^ 1);
                issue(std::integral_constant<int, 0>());
            }
        }
        const int64_t m0 = at.m0;
        const int n0 = at.n0, rows = at.rows;
        int8_t* const own = lds + (PERSIST ? STG : 0) + wv * REGION;
        // this lane's results: tokens 32 MT wm + 32 tt + li, channels from cl on
        const int lane_e = lane_now(), li = lane_e & 31, lg = lane_e >> 5, cl = wn * 32 * NT + 16 * NT * lg;
        float xs[MT];
#pragma unroll
        for (int tt = 0; tt < MT; ++tt) xs[tt] = xs_s[par][wm * 32 * MT + li + 32 * tt];
        const int mv_row = lane_e / CH, c_mv = n0 + wn * 32 * NT + CK::E * (lane_e % CH);
        const bool whole = n0 + (wn + 1) * 32 * NT <= N;      // (of all lanes) no channel of the wavefront's is past the last
        auto at_mv = [&](int i) __attribute__((always_inline)) {
            const int row = MV_ROWS * i + mv_row;
            return own + row * RB + 16 * ((lane_e % CH) ^ swz(row));
        };
        auto pass = [&](auto t0_c) __attribute__((always_inline)) -> bool {      // false: no tokens from there on
            constexpr int t0 = decltype(t0_c)::value;
            const int64_t mw = m0 + wm * 32 * MT + 32 * t0;   // the first token of the slots
            const int left = rows - (wm * 32 * MT + 32 * t0); // tokens from there on
            if (left <= 0) {
                if (PERSIST && t0 == 0) wait_vm0();
                return false;
            }
            if constexpr (TYPE != TYPE_I8) {
                if (P.residual) {
                    if constexpr (EARLY) {
#pragma unroll
                        for (int i = 0; i < SLOTS * MOVES; ++i) *reinterpret_cast<v4i*>(at_mv(i)) = early[EARLY ? t0 / SLOTS : 0][EARLY ? i : 0];
                    } else {
                        const T* const res = static_cast<const T*>(P.residual) + mw * P.ld_res + c_mv;
                        if (whole) {
                            v4i r[SLOTS * MOVES];
                            if (P.once) {
                                keep_apart();
#pragma unroll
                                for (int i = 0; i < SLOTS * MOVES; ++i) r[i] = CK::load_once(res + min(MV_ROWS * i + mv_row, left - 1) * P.ld_res);
                                keep_apart();
                            } else {
#pragma unroll
                                for (int i = 0; i < SLOTS * MOVES; ++i) r[i] = CK::load(res + min(MV_ROWS * i + mv_row, left - 1) * P.ld_res, CK::E, CK::E);
                            }
#pragma unroll
                            for (int i = 0; i < SLOTS * MOVES; ++i) *reinterpret_cast<v4i*>(at_mv(i)) = r[i];
                        } else if (c_mv < N) {
#pragma unroll 1
                            for (int i = 0; i < SLOTS * MOVES; ++i) {
                                const int row = min(MV_ROWS * i + mv_row, left - 1);
                                *reinterpret_cast<v4i*>(at_mv(i)) = CK::load(res + row * P.ld_res, N - c_mv, (P.M - 1 - mw - row) * P.ld_res + N - c_mv);
                            }
                        }
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                }
            }
            with_activation(P.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < MINE; ++j) {
                    const int c = cl + CK::E * j;             // first channel of the chunk in the tile
                    typename CK::vf ws, bi;
#pragma unroll
                    for (int e = 0; e < CK::E; e += 4) {
                        const v4f a = *reinterpret_cast<const v4f*>(&ws_s[par][c + e]), b = *reinterpret_cast<const v4f*>(&bias_s[par][c + e]);
#pragma unroll
                        for (int k = 0; k < 4; ++k) { ws[e + k] = a[k]; bi[e + k] = b[k]; }
                    }
                    static_for<SLOTS>([&](auto tt_c) __attribute__((always_inline)) {
                        constexpr int tt = t0 + decltype(tt_c)::value;
                        int8_t* const at = own + (32 * (tt % SLOTS) + li) * RB + 16 * ((MINE * lg + j) ^ swz(li));
                        typename CK::vf v;
#pragma unroll
                        for (int e = 0; e < CK::E; ++e) {
                            constexpr int PER = 16 / CK::E;   // chunks of the 16 results of an MFMA tile
                            v[e] = activation<decltype(act)::value, TYPE == TYPE_F32>(__builtin_fmaf((float)acc[j / PER][tt][CK::E * (j % PER) + e] * ws[e], xs[tt], bi[e]));
                        }
                        if constexpr (TYPE != TYPE_I8) {
                            if (P.residual) v += CK::unpack(*reinterpret_cast<const v4i*>(at));
                        }
                        *reinterpret_cast<v4i*>(at) = CK::pack(v, P.inv_step);
                    });
                    __builtin_amdgcn_sched_barrier(0);        // keep the register footprint of the epilogue small
                }
            });
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (PERSIST && t0 == 0) wait_vm0();               // the next tile's first stage, before stores stand in line behind it
            T* const y = static_cast<T*>(P.y) + mw * P.ldy + c_mv;
            if (whole && P.once) {
                keep_apart();
#pragma unroll
                for (int i = 0; i < SLOTS * MOVES; ++i) {
                    const v4i v = *reinterpret_cast<const v4i*>(at_mv(i));
                    if (MV_ROWS * i + mv_row < left) CK::store_once(y + (MV_ROWS * i + mv_row) * P.ldy, v);
                }
                keep_apart();
            } else if (whole) {
#pragma unroll
                for (int i = 0; i < SLOTS * MOVES; ++i) {
                    const v4i v = *reinterpret_cast<const v4i*>(at_mv(i));
                    if (MV_ROWS * i + mv_row < left) CK::store(y + (MV_ROWS * i + mv_row) * P.ldy, v, CK::E);
                }
            } else {
#pragma unroll 1
                for (int i = 0; i < SLOTS * MOVES; ++i) {
                    const v4i v = *reinterpret_cast<const v4i*>(at_mv(i));
                    if (MV_ROWS * i + mv_row < left) CK::store(y + (MV_ROWS * i + mv_row) * P.ldy, v, N - c_mv);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            return true;
        };
        bool on = true;
        static_for<MT / SLOTS>([&](auto p) __attribute__((always_inline)) { if (on) on = pass(std::integral_constant<int, decltype(p)::value * SLOTS>()); });
        if (!more_tiles) break;
        at = next;
        tile += slots;
    }
}

constexpr int64_t kBand = 4;                   // rows of tiles in a band
template <int TYPE, int MT, int NT, int GM, int GN, int S> hipError_t launch_tile(hipStream_t s, const ScaledArgs& a) {
    using TL = GsTile<MT, NT, GM, GN>;
    GsParams P;
    P.x = a.x; P.x_scale = a.x_scale; P.w = a.w; P.w_scale = a.w_scale; P.bias = a.bias; P.residual = a.residual; P.y = a.y;
    P.ldx = a.ldx; P.ld_res = a.ld_res; P.ldy = a.ldy; P.M = a.M; P.N = a.N; P.K = a.K; P.act = a.act; P.one_scale = a.one_scale;
    P.inv_step = a.inv_step;
    // From 64 MB on, results are stored past the L2, which has the operands to keep and would write them back at the launch's end
    // (8192 x 8192 x 4096 239 and 229 us, 50432 x 768 x 768 53 and 44.5), and a residual is loaded past it (both: 8192 x 8192 x 4096 278 and 252,
    // 50432 x 768 x 768 64 and 57.5).  Smaller ones stay in the caches for whoever reads them next (25216 x 1152 x 384 with int8 results and a
    // pass over them 67 us for 76; residuals: 25216 x 384 x 1536 28.2 and 29.4, 4096 x 4096 x 4096, 34 MB, 67.4 and 66.6).
    P.once = a.M * a.N * (int64_t)sizeof(Stored<TYPE>) >= (int64_t)1 << 26;
    const int64_t tm = (a.M + TL::TM - 1) / TL::TM, tn = (a.N + TL::TN - 1) / TL::TN;
    int64_t grid = (tm * tn + NXCD - 1) / NXCD * NXCD;
    P.order = TileOrder((uint32_t)tm, (uint32_t)tn, (uint32_t)(tm < kBand ? tm : kBand));
    if (MT * NT >= 4 && S == 2) grid = min64(grid, (int64_t)num_cus() * (TL::W == 4 ? 2 : 1) / NXCD * NXCD);     // (PERSIST)
    hipLaunchKernelGGL((gemm_scaled_kernel<TYPE, MT, NT, GM, GN, S>), dim3((unsigned)grid), dim3(64 * TL::W), 0, s, P);
    return hipGetLastError();
}

template <int TYPE> hipError_t launch_type(hipStream_t s, const ScaledArgs& a, Form form) {
    switch (form) {
        case T64: return launch_tile<TYPE, 1, 1, 2, 2, 3>(s, a);
        case T128X64: return launch_tile<TYPE, 1, 1, 4, 2, 4>(s, a);
        case T128X8: return launch_tile<TYPE, 2, 1, 2, 4, 3>(s, a);
        case T256X128: return launch_tile<TYPE, 2, 2, 4, 2, 3>(s, a);
        case T256: return launch_tile<TYPE, 4, 2, 2, 4, 2>(s, a);
        default: return launch_tile<TYPE, 2, 2, 2, 2, 2>(s, a);
    }
}

}  // namespace

hipError_t launch_linear_scaled(hipStream_t s, const ScaledArgs& a) {
    if (a.M == 0) return hipSuccess;
    const Form form = form_of(a.M, a.N, a.K, num_cus());
    const int64_t e = element_bytes(a.y_type);
    auto ops = [&](int64_t M) { return 2 * M * a.N * a.K; };
    auto bytes = [&](int64_t M) { return M * a.K + (int64_t)a.N * a.K + M * a.N * e * (a.residual ? 2 : 1); };
    if (form == ROWS) {
        TraceScope trace(s, KIND_GEMM_SCALED, ops(a.M), bytes(a.M));
        return launch_linear_scaled_rows(s, a);
    }
    // (a grid may have 2^32 threads; N is at most 2^24)
    const int64_t most = 64 * (((int64_t)1 << 22) / ((a.N + 63) / 64));
    for (int64_t m = 0; m < a.M; m += most) {
        ScaledArgs b = a;
        b.x += m * a.ldx; b.M = min64(a.M - m, most);
        if (!a.one_scale) b.x_scale += m;
        if (a.residual) b.residual = static_cast<const int8_t*>(a.residual) + m * a.ld_res * e;
        b.y = static_cast<int8_t*>(a.y) + m * a.ldy * e;
        TraceScope trace(s, KIND_GEMM_SCALED, ops(b.M), bytes(b.M));
        hipError_t st;
        switch (a.y_type) {
            case TYPE_F16: st = launch_type<TYPE_F16>(s, b, form); break;
            case TYPE_BF16: st = launch_type<TYPE_BF16>(s, b, form); break;
            case TYPE_I8: st = launch_type<TYPE_I8>(s, b, form); break;
            default: st = launch_type<TYPE_F32>(s, b, form);
        }
        if (st != hipSuccess) return st;
    }
    return hipSuccess;
}

}  // namespace ivit
