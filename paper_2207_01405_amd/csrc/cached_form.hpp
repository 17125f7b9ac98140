// Into how many parts cached_attention.hip cuts the keys of a call (host arithmetic only).
#pragma once
#include <stdint.h>

#include <cmath>

namespace ivit {
namespace cached {

constexpr int W = 4, BK = 32, LEAST = 2 * W;   // wavefronts of a workgroup; keys of a block; blocks of the smallest part
constexpr int WIDE = 32 * W, TK = 16 * W;      // rows of a workgroup that shares its keys, keys of its tiles

// Parts.  Requests: of the greatest length, four workgroups a CU and 1536 keys a part at most (64 parts are enough where CUs have work), so that requests of different
// lengths leave no CU waiting (48 of up to 16384 int8 keys 172 us, in parts of 5461 keys 195); shorter ones in as many, of `least` keys at least, which are fewer where
// there are few requests.  Without a prefix twice as many are one part, which is one launch (1 request of 500, 32 heads of 128 on 8: 9.0 -> 8.7 us, with the host
// 11.5 -> 9.0; 32 of 1000 30.6 -> 27.9).
// The prefix: n parts take about  max(own, chain / n + own / 2) + n part  us.  chain: all its keys by one workgroup, 9 ns a key, or 17 for elements of 128 (34 of int8
// rows) where a wavefront has rows of its own; own: the requests' own keys from memory, beside which a workgroup of the prefix gets on half as fast; part: writing
// and reading the rows of a part.  `own` is known for the greatest length only, and counts up to 40 us.  Where the prefix's workgroups take more than three
// quarters of the CUs, the requests' take a quarter longer.  Heads of 128, 32 on 8, in us with one part / these / the best number: 64 requests behind 1000 keys
// 28.9 / 17.4 / 17.4, behind 8000 with up to 600 of their own 155 / 42 / 41, 256 behind 16000 291 / 97 / 97, 128 behind 8000 with 1200 of their own 207 / 136 / 125.
// Its smallest part is a block a wavefront where these share tiles, else two: against two, 20 requests behind 257 keys 13.1 -> 11.1, behind 1000 15.3 -> 13.6, 24 of 16
// heads on 4 behind 1000 int8 keys 20.3 -> 15.6; 24 behind 2000 16.1 -> 16.6.
struct Plan { int prefix_tiles, own_tiles, prefix_parts, own_parts, prefix_least, own_least; bool wide; };

inline Plan plan_of(int B, int H, int G, int d, bool i8, int page_size, int max_pages, int prefix_len, int cus) {
    const int group = H / G;
    const int64_t keys = (int64_t)max_pages * page_size, rows = (int64_t)B * group;
    auto over = [](int64_t n, int64_t by) { return (n + by - 1) / by; };
    auto less = [](int64_t a, int64_t b) { return a < b ? a : b; };
    auto more = [](int64_t a, int64_t b) { return a > b ? a : b; };
    // of n parts, those that hold keys where parts are of whole blocks, `least` at the least
    auto with_keys = [&](int64_t n, int64_t blocks, int least) { return (int)over(blocks, more(over(blocks, n), least)); };
    const bool wide = rows > 64;
    Plan p{0, (group + 31) / 32, 0, 0, wide ? W : LEAST, LEAST, wide};
    p.prefix_tiles = (int)over(rows, wide ? WIDE : 32);
    const int64_t items = (int64_t)B * p.own_tiles * G;
    if (prefix_len > 0 && rows > 0) {
        const int full = (int)over(cus, (int64_t)p.prefix_tiles * G);                                        // parts that are a workgroup a CU
        const float chain = prefix_len * (wide ? d * (i8 ? 2.66e-4f : 1.33e-4f) : 9e-3f), part = (float)B * H * d * (wide ? 3.5e-6f : 7e-6f);
        const float own = std::fmin((float)B * keys * G * d * (i8 ? 4e-7f : 8e-7f), 40.0f), root = std::sqrt(chain / part);
        auto takes = [&](int n) { return std::fmax(own, chain / n + own / 2) + part * n; };
        const float best = std::fmax(own * root > 2 * chain ? 2 * chain / own : root, 1.0f);               // where it is least
        const int most_parts = (int)less(full, over(prefix_len, BK * p.prefix_least)), fewer = (int)more(3 * full / 4, 1);
        int n = best < most_parts ? (int)best : most_parts;
        if (n < most_parts && takes(n + 1) < takes(n)) ++n;
        p.prefix_parts = with_keys(n > fewer && takes(fewer) < takes(n) + own / 4 ? fewer : n, over(prefix_len, BK), p.prefix_least);
    }
    if (keys > 0 && items > 0) {
        p.own_least = items >= 2 * cus ? 4 * LEAST : 2 * items >= cus ? 2 * LEAST : LEAST;
        const int64_t fill = over(4 * cus, items), even = less(over(keys, 1536), 64);
        p.own_parts = prefix_len == 0 && keys <= 2 * BK * p.own_least ? 1 : (int)less(more(fill, even), over(keys, BK * p.own_least));
        // (a launch has less than 2^32 threads; B H <= 2^23 leaves room for one part of both)
        p.own_parts = (int)more(less(p.own_parts, ((1 << 24) - 1 - (int64_t)p.prefix_tiles * p.prefix_parts * G) / items), 1);
        p.own_parts = with_keys(p.own_parts, over(keys, BK), p.own_least);
    }
    return p;
}

}  // namespace cached
}  // namespace ivit
