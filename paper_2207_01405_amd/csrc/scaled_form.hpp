// Which form of the Dense layer with real scales a shape takes (host arithmetic only).  us measured on 256 CUs, bf16 results, inputs in turn.
#pragma once
#include <stdint.h>

namespace ivit {
namespace scaled {

enum Form { ROWS, T64, T128X64, T128X8, T256X128, T256, T128 };
constexpr Form form_of(int64_t M, int64_t N, int64_t K, int64_t cus) {
    auto tiles = [&](int64_t m, int64_t n) { return ((M + m - 1) / m) * ((N + n - 1) / n); };
    auto rounds = [&](int64_t m, int64_t n, int64_t per_cu) { return (tiles(m, n) + per_cu * cus - 1) / (per_cu * cus); };
    // Few rows: the kernel whose wavefronts split K, while two of its 32 x 32 tiles a CU take the shape (that kernel's and 64 x 64:
    // 64 x 4096 x 4096 6.4 and 11.0, 128 x 4096 x 4096 9.2 and 11.1, 394 x 384 x 384 3.0 and 3.4, 788 x 384 x 1536 5.3 and 5.1; three a CU:
    // 64 x 11008 x 4096 14.5 and 11.9, 394 x 1536 x 384 4.7 and 3.6), and for up to 32 rows always (16 x 32000 x 4096 27.1 and 33.1).
    if (M <= 32 || rounds(32, 32, 2) <= 1) return ROWS;
    // Rows of 768 bytes and more: the smallest tile that gives every CU at most one workgroup (64 x 64, 128 x 64, 128 x 128, 256 x 128,
    // 256 x 256: 1024 x 1024 x 1024 4.7, 5.6, 6.9, 10.0, 15.0; 512 x 4096 x 4096 16.7, 15.5, 19.0, 24.5, 40.9; 1024 x 4096 x 4096 37, 27, 23.0, 27.4, 42;
    // 512 x 11008 x 4096 42, 38, 38, 29.1, 43; 1024 x 11008 x 4096 77, 74, 60, 58, 49.6).  Shorter rows gain nothing by it (1576 x 1536 x 384
    // 5.2, 7.1).
    if (K >= 768) {
        if (tiles(64, 64) <= cus) return T64;
        if (tiles(128, 64) <= cus) return T128X64;
        if (tiles(128, 128) <= cus) return T128X8;
        if (tiles(256, 128) <= cus) return T256X128;
        // Rounds of 256 x 256, one a CU, against those of 128 x 128, two a CU, which do half the work.  Time with 128 x 128 over 256 x 256, in turn, at
        // K = 768, 1024, 1536 and 2048.  Half as many rounds: 4096 x 4096 1.06, 1.08, 1.09, 1.10, 8192 x 8192 1.08, 1.09, 1.14, 1.16, 4096 x 8192
        // 0.92, 0.95, 1.01, 1.08.  More than half, what the last round leaves idle counts, and the epilogue, which nothing runs beside: 4 of 7
        // (25216 x 2304) 0.98, 0.99, 1.06, 1.08, with a residual 0.94, 0.97, 1.02, 1.05; 3 of 5 (50432 x 768) 0.93, 0.95, 1.01, 1.04, with
        // a residual 0.89, 0.91, 0.95, 0.99, with GELU 0.89, 0.90, 0.93, 0.99.
        const int64_t most = K < 1536 ? 50 : K < 2048 ? 58 : 60;      // in a hundred
        if (rounds(256, 256, 1) * 100 <= rounds(128, 128, 2) * most) return T256;
        return T128;
    }
    // up to three 64 x 64 tiles a CU, and where 128 channels would be half padding: 64 x 64 (1576 x 1536 x 384 5.2 and 6.3 with 128 x 128, 3152 x
    // 1536 x 384, 4.7 tiles a CU, 8.3 and 8.3; 300000 x 64 x 64 16.5 and 23.7)
    if (rounds(64, 64, 3) <= 1 || N <= 64) return T64;
    return T128;
}

}  // namespace scaled
}  // namespace ivit
