// Rotary positions on the heads of float rows, and the same on the way of keys and values into a paged cache.
//
//   phi = positions[axis[i]][row] freq[i];   (x1, x2) -> (x1 cos phi - x2 sin phi, x2 cos phi + x1 sin phi)
//
// A workgroup takes a few rows.  It forms their sines and cosines first, once for all heads, into LDS: the angle in 64 bits and brought to one turn
// there, for at position 10^6 an angle of 32 bits is 0.03 off.  Then every thread turns pieces of eight elements.
#include <utility>

#include "scaled_common.hpp"

namespace ivit {
namespace {

using namespace scaled;

constexpr int BLOCK = 256;

struct Turn { const int32_t* positions; const double* freq; const int32_t* axis; int64_t ld; int axes, half; bool split; FastDiv by_half; };

// sines and cosines of rows first .. first + n - 1, pair i of row t at [t half + i]; or, where lanes read eight of them each from multiples of eight on, the first
// four of every eight and then the others, so that lanes read side by side
__device__ __forceinline__ void angles(const Turn& r, int64_t first, int n, float* cs, float* sn) {
    for (int i = threadIdx.x; i < n * r.half; i += BLOCK) {
        uint32_t p;
        const uint32_t t = r.by_half.divide((uint32_t)i, p);
        const int a = r.axis ? min(max(r.axis[p], 0), r.axes - 1) : 0;
        const double turns = (double)r.positions[a * r.ld + first + t] * r.freq[p] * 0.15915494309189535;     // / (2 pi)
        float s, c;
        sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &c);
        const int at = r.split ? (int)t * r.half + (p & 4 ? r.half / 2 : 0) + (int)(p / 8) * 4 + (int)(p & 3) : i;
        cs[at] = c;
        sn[at] = s;
    }
}

typedef float v4f __attribute__((ext_vector_type(4)));
// pairs e .. e + 7 of a row's, split as above
__device__ __forceinline__ v8f split8(const float* row, int half, int e) {
    const v4f a = *reinterpret_cast<const v4f*>(row + e / 2), b = *reinterpret_cast<const v4f*>(row + half / 2 + e / 2);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ float first_of(float x1, float x2, float c, float s) { return __builtin_fmaf(x1, c, -(x2 * s)); }
__device__ __forceinline__ float second_of(float x1, float x2, float c, float s) { return __builtin_fmaf(x2, c, x1 * s); }

struct RotaryParams {
    const void* x; void* y; int64_t ldx, ldy, rows; int d, rows_each, pair_pieces, pieces_each; bool adjacent, in_place; Turn r; FastDiv per_row, per_head;
};

// Items: the pieces of pairs of every head (eight pairs (i, i + half), or four adjacent ones), then those of the elements that stay.  A last piece that is not
// whole starts earlier and does some pairs again, with the same result; in place, where they may be turned by then, it goes element by element
// (5003 x 17 heads of 80 of which 60 are turned, float32: 18.5 us element by element, 12.4 so).
template <class T> __global__ __launch_bounds__(BLOCK) void rotary_kernel(RotaryParams P) {
    extern __shared__ __align__(16) float lds[];
    const int64_t first = (int64_t)blockIdx.x * P.rows_each;
    const int n = (int)min64(P.rows - first, P.rows_each), half = P.r.half;
    float *const cs = lds, *const sn = lds + P.rows_each * half;
    angles(P.r, first, n, cs, sn);
    __syncthreads();
    const bool again = !P.in_place;
    const uint32_t end = min(n * P.per_row.d, (blockIdx.y + 1) * P.pieces_each);
    for (uint32_t i = blockIdx.y * P.pieces_each + threadIdx.x; i < end; i += BLOCK) {
        uint32_t rest, piece;
        const uint32_t t = P.per_row.divide(i, rest), h = P.per_head.divide(rest, piece);
        const T* const x = static_cast<const T*>(P.x) + (first + t) * P.ldx + (int64_t)h * P.d;
        T* const y = static_cast<T*>(P.y) + (first + t) * P.ldy + (int64_t)h * P.d;
        if ((int)piece >= P.pair_pieces) {
            int e = 2 * half + 8 * ((int)piece - P.pair_pieces);
            if (P.d - 2 * half >= 8) e = min(e, P.d - 8);
            const int m = P.d - e;
            if (m >= 8) store8(y + e, load8(x + e));
            else store_some(y + e, load_some(x + e, m), m);
            continue;
        }
        if (P.adjacent) {
            int e = 8 * (int)piece;
            if (again && half >= 4) e = min(e, 2 * half - 8);
            const int m = 2 * half - e;
            const float *const c = cs + t * half + e / 2, *const s = sn + t * half + e / 2;
            v8f v = m >= 8 ? load8(x + e) : load_some(x + e, m), w = {};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (2 * j < m) {
                    w[2 * j] = first_of(v[2 * j], v[2 * j + 1], c[j], s[j]);
                    w[2 * j + 1] = second_of(v[2 * j], v[2 * j + 1], c[j], s[j]);
                }
            if (m >= 8) store8(y + e, w);
            else store_some(y + e, w, m);
            continue;
        }
        int e = 8 * (int)piece;
        if (again && half >= 8) e = min(e, half - 8);
        if (P.r.split) {
            const v8f c = split8(cs + t * half, half, e), s = split8(sn + t * half, half, e), v1 = load8(x + e), v2 = load8(x + half + e);
            v8f w1, w2;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w1[j] = first_of(v1[j], v2[j], c[j], s[j]);
                w2[j] = second_of(v1[j], v2[j], c[j], s[j]);
            }
            store8(y + e, w1);
            store8(y + half + e, w2);
            continue;
        }
        const int m = half - e;
        const float *const c = cs + t * half + e, *const s = sn + t * half + e;
        const v8f v1 = m >= 8 ? load8(x + e) : load_some(x + e, m), v2 = m >= 8 ? load8(x + half + e) : load_some(x + half + e, m);
        v8f w1 = {}, w2 = {};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < m) {
                w1[j] = first_of(v1[j], v2[j], c[j], s[j]);
                w2[j] = second_of(v1[j], v2[j], c[j], s[j]);
            }
        if (m >= 8) {
            store8(y + e, w1);
            store8(y + half + e, w2);
        } else {
            store_some(y + e, w1, m);
            store_some(y + half + e, w2, m);
        }
    }
}

struct AppendParams {
    const void *q, *k, *v; void *q_out, *kc, *vc; float *ks, *vs; const int32_t* slots;
    int64_t ldq, ldk, ldv, ldqo, ld_page, rows; int H, G, page_shift, rows_each, pieces_each, n_slots; bool adjacent; Turn r; FastDiv per_row;
};

// Lanes 0 .. D / 8 of a head hold eight elements each, as they lie; a lane reads its elements' partners beside them.  The heads of a row: queries, keys,
// values.  int8: the largest of a head over its lanes.
template <class T, int D, bool I8> __global__ __launch_bounds__(BLOCK) void append_kernel(AppendParams P) {
    constexpr int L = D / 8;
    extern __shared__ __align__(16) float lds[];
    const int64_t first = (int64_t)blockIdx.x * P.rows_each;
    const int n = (int)min64(P.rows - first, P.rows_each), half = P.r.half;
    float *const cs = lds, *const sn = lds + P.rows_each * half;
    if (half) {
        angles(P.r, first, n, cs, sn);
        __syncthreads();
    }
    const uint32_t end = min(n * P.per_row.d, (blockIdx.y + 1) * P.pieces_each);
    for (uint32_t i = blockIdx.y * P.pieces_each + threadIdx.x; i < end; i += BLOCK) {
        uint32_t rest;
        const uint32_t t = P.per_row.divide(i, rest);
        int h = (int)(rest / L);
        const int e = 8 * (int)(rest % L);
        const int slot = P.slots[first + t];
        if ((uint32_t)slot >= (uint32_t)P.n_slots) continue;            // (all lanes of a head)
        const bool query = h < P.H, value = h >= P.H + P.G;
        h -= query ? 0 : value ? P.H + P.G : P.H;
        const T* const x = query ? static_cast<const T*>(P.q) + (first + t) * P.ldq + (int64_t)h * D
                                 : static_cast<const T*>(value ? P.v : P.k) + (first + t) * (value ? P.ldv : P.ldk) + (int64_t)h * D;
        v8f v = load8(x + e);
        if (!value && e < 2 * half) {
            if (P.adjacent) {
                const float *const c = cs + t * half + e / 2, *const s = sn + t * half + e / 2;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (e / 2 + j < half) {
                        const float a = v[2 * j], b = v[2 * j + 1];
                        v[2 * j] = first_of(a, b, c[j], s[j]);
                        v[2 * j + 1] = second_of(a, b, c[j], s[j]);
                    }
            } else if (P.r.split) {
                const bool lower = e < half;
                const int at = lower ? e : e - half;
                const v8f w = load8(x + (lower ? e + half : at));
                const v8f c = split8(cs + t * half, half, at), s = split8(sn + t * half, half, at);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = lower ? first_of(v[j], w[j], c[j], s[j]) : second_of(w[j], v[j], c[j], s[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool lower = e + j < half;
                    const int at = lower ? e + j : e + j - half;
                    if (at < half) {
                        const float w = (float)x[lower ? at + half : at], c = cs[t * half + at], s = sn[t * half + at];
                        v[j] = lower ? first_of(v[j], w, c, s) : second_of(w, v[j], c, s);
                    }
                }
            }
        }
        if (query) {
            store8(static_cast<T*>(P.q_out) + (first + t) * P.ldqo + (int64_t)h * D + e, v);
            continue;
        }
        const int page = slot >> P.page_shift, in = (h << P.page_shift) + (slot & ((1 << P.page_shift) - 1));
        const int64_t at = page * P.ld_page + (int64_t)in * D + e;
        void* const cache = value ? P.vc : P.kc;
        if constexpr (I8) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
#pragma unroll
            for (int m = L / 2; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
            const Quant q = quant_of(top, 1.0f);
            if (e == 0) (value ? P.vs : P.ks)[(((int64_t)page * P.G) << P.page_shift) + in] = q.scale;
            store_q(static_cast<int8_t*>(cache) + at, v, q, 8);
        } else {
            store8(static_cast<T*>(cache) + at, v);
        }
    }
}

Turn turn_of(const RotaryArgs& r) {
    return Turn{r.positions, r.freq, r.axis, r.ld_positions, r.n_axes, r.half, !r.adjacent && r.half % 8 == 0, FastDiv((uint32_t)(r.half > 0 ? r.half : 1))};
}

// Rows of a workgroup: some 1024 pieces, as long as there are four workgroups a CU; sines and cosines of at most 32 KB.  Few rows: the pieces of one go to
// several workgroups, 256 each at least, which form the row's angles again.
struct Shape { int rows_each, pieces_each; dim3 grid; };
Shape shape_of(int64_t rows, int64_t pieces, int half) {
    const int64_t wanted = 4 * num_cus();
    int64_t n = min64((1024 + pieces - 1) / pieces, (rows + wanted - 1) / wanted);
    n = n < 1 ? 1 : half && n > 4096 / half ? 4096 / half : n;
    int64_t split = n > 1 ? 1 : min64((pieces + BLOCK - 1) / BLOCK, (wanted + rows - 1) / rows);
    int64_t each = (pieces * n + split - 1) / split;
    each = (each + BLOCK - 1) / BLOCK * BLOCK;
    split = (pieces * n + each - 1) / each;
    return Shape{(int)n, (int)each, dim3((unsigned)((rows + n - 1) / n), (unsigned)split)};
}

}  // namespace

hipError_t launch_rotary(hipStream_t s, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int heads, int d, int type, const RotaryArgs& r) {
    const int pairs = r.adjacent ? (2 * r.half + 7) / 8 : (r.half + 7) / 8;
    const int stay = x == y ? 0 : (d - 2 * r.half + 7) / 8;                  // (in place they are there)
    const int64_t pieces = (int64_t)heads * (pairs + stay);
    const Shape sh = shape_of(rows, pieces, r.half);
    RotaryParams P{x, y, ldx, ldy, rows, d, sh.rows_each, pairs, sh.pieces_each, r.adjacent, x == y, turn_of(r), FastDiv((uint32_t)pieces), FastDiv((uint32_t)(pairs + stay))};
    TraceScope trace(s, KIND_ROTARY, 0, 2 * element_bytes(type) * rows * heads * d + 4 * rows * r.n_axes);
    const dim3 grid = sh.grid;
    const size_t lds = (size_t)sh.rows_each * r.half * 2 * sizeof(float);
    if (type == TYPE_F32) rotary_kernel<float><<<grid, BLOCK, lds, s>>>(P);
    else if (type == TYPE_F16) rotary_kernel<_Float16><<<grid, BLOCK, lds, s>>>(P);
    else rotary_kernel<__bf16><<<grid, BLOCK, lds, s>>>(P);
    return hipGetLastError();
}

hipError_t launch_cache_append(hipStream_t s, const AppendArgs& a) {
    const CacheArgs& c = a.c;
    const int64_t pieces = (int64_t)(a.H + 2 * c.G) * (c.d / 8);
    const Shape sh = shape_of(a.rows, pieces, a.r.half);
    AppendParams P{a.q, a.k, a.v, a.q_out, c.k, c.v, c.k_scale, c.v_scale, a.slots, a.ldq, a.ldk, a.ldv, a.ldq_out, c.ld_page, a.rows, a.H, c.G,
                   __builtin_ctz(c.page_size), sh.rows_each, sh.pieces_each, c.n_pages * c.page_size, a.r.adjacent, turn_of(a.r), FastDiv((uint32_t)pieces)};
    const bool i8 = c.type == TYPE_I8;
    TraceScope trace(s, KIND_CACHE_APPEND, 0, a.rows * (2 * (int64_t)(2 * a.H + 2 * c.G) * c.d + 2 * (int64_t)c.G * (i8 ? c.d + 4 : 2 * c.d)));
    const dim3 grid = sh.grid;
    const size_t lds = (size_t)sh.rows_each * a.r.half * 2 * sizeof(float);
    auto with = [&](auto t, auto d) {
        using T = decltype(t);
        if (i8) append_kernel<T, decltype(d)::value, true><<<grid, BLOCK, lds, s>>>(P);
        else append_kernel<T, decltype(d)::value, false><<<grid, BLOCK, lds, s>>>(P);
    };
    auto of_type = [&](auto t) { c.d == 64 ? with(t, std::integral_constant<int, 64>()) : with(t, std::integral_constant<int, 128>()); };
    a.type == TYPE_F16 ? of_type(_Float16()) : of_type(__bf16());
    return hipGetLastError();
}

}  // namespace ivit
