// Which workgroups prompt_attention.hip takes for a call (host arithmetic only).
#pragma once
#include <stdint.h>

namespace ivit {
namespace prompt {

// Rows of queries and groups of wavefronts that share out the keys of a workgroup, keys of a tile.
enum Form { R64X4_K32, R64_K32, R128X2_K64, R128_K64 };

// Where 128 rows a workgroup leave CUs without one (taking the sequences for equally long), the keys are shared out inside a workgroup: 500 queries after 7500
// keys, 32 heads of 128, are 128 such workgroups, 128 us; two groups of 128 rows 106, four of 64 rows 88.  1000 after 7000: 140, 130, 155; 1500 after
// 7000: 213, 226, 237.
// Short sequences: 64 rows and tiles of 32 keys, four workgroups a CU, leave fewer rows empty and more loads in flight.  16384 rows, 32 heads of 128 on 8, causal, in
// sequences of 16, 49, 64, 100, 160, 197, 300, 512: 155, 83, 75, 90, 92, 107, 104, 129 us (128 rows 310, 120, 101, 93, 111, 109, 115, 123); not causal 64, 100, 128, 160, 197:
// 77, 102, 90, 106, 131 (103, 98, 88, 123, 127); 12 heads of 64, causal, 49, 160, 300: 21, 27, 34 (30, 28, 30), not causal 64, 100, 128, 160, 197, 300, 512:
// 26, 28, 27, 30, 33, 36, 46 (27, 26, 29, 32, 33, 35, 40).  Of different lengths, 55, 106, 199, 261, 358 on average:
// 57, 54, 59, 67, 74 (74, 62, 61, 68, 72), not causal 59, 61, 76, 93, 103 (70, 67, 73, 89, 97).
// The host knows the mean length only: a long sequence among many short ones goes in 64 rows too, which costs it a twentieth (512: 129 for 123).
inline Form form_of(int64_t n_q, int64_t n_seq, int H, bool causal, int cus) {
    const int64_t blocks = n_seq * ((n_q + 128 * n_seq - 1) / (128 * n_seq)) * H;
    if (2 * blocks <= cus) return R64X4_K32;
    if (n_q <= (causal ? 200 : 128) * n_seq) return R64_K32;
    return blocks <= cus ? R128X2_K64 : R128_K64;
}

}  // namespace prompt
}  // namespace ivit
