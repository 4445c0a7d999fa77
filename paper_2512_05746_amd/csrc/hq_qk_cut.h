// How a head's channels are dealt to lanes (hq_qk_norm_rope.hip): host and device arithmetic without memory accesses.
#pragma once

#include "hq.h"

namespace hq {

// Pairs to a lane and lanes to a head, a power of two (g = 0: a wave for a head).  As many pairs as divide both parts of the head, for a
// lane's channels have to be neighbours: 20000 tokens of 32 heads of 72 in bf16 with 36 of them turned, two pairs, 87 us (137 with
// gradients), with 18, one pair, 124 (207), where a wave for each head takes 368 and 364 (702, 691).  Eight pairs are two loads of 16
// bytes for floats of 16 bits.  For 32 bits four are, and forwards that is faster: 36918 tokens of 36 heads of 96 258 -> 216 us, 30000 of
// 128 219 -> 217; backwards where eight would leave lanes without a pair (heads of 96 358 -> 315 us, of 80 208 -> 198), else eight are
// (heads of 128 332 us, with four 339).
// (Lanes that are no power of two, 60 of 64 busy instead of 40 .. 48: 3 to 6 % less for many tokens of 80 or 96 channels, up to 10 % more
// for a thousand, since their sums take five exchanges through LDS.)
struct QkCut {
    int c, g;
};
inline QkCut qk_cut_of(int d, int rotary, hq_dtype dt, bool back) {
    const bool full = d % 16 == 0 && ((d >> 4) & ((d >> 4) - 1)) == 0;
    for (const int c : {8, 4, 2, 1}) {
        if ((rotary >> 1) % c || (d >> 1) % c) continue;
        const int lanes = (d >> 1) / c;
        if (lanes > 64 || (c == 8 && dt == HQ_F32 && d <= 256 && !(back && full))) continue;
        int g = 2;
        while (g < lanes) g *= 2;
        return {c, g};
    }
    return {0, 0};
}

// The channels of a lane that owns c pairs from pair p on: c from `first`, c from `second`.  Interleaved: 2 c neighbours, and pair i is
// their (2i, 2i + 1).  Channels that are not rotated are dealt in the same way.
struct QkPlace {
    int first, second;
    bool rotated;   // its pairs are elements p .. p + c - 1 of a token's row of the tables
};
__host__ __device__ __forceinline__ QkPlace qk_place_of(int d, int rotary, bool interleaved, int c, int p) {
    const int r = rotary >> 1;
    if (interleaved) return {2 * p, 2 * p + c, p < r};
    return p < r ? QkPlace{p, p + r, true} : QkPlace{r + p, r + p + (d >> 1) - r, false};
}

// Lane `in` of the lanes of a head.  One beyond the last pair has the first lane's, channels and table alike: what it loads has to lie
// inside them.
struct QkLane {
    bool live;   // it has pairs of its own; otherwise it stores nothing
    int p;       // its first pair
    QkPlace at;
};
__host__ __device__ __forceinline__ QkLane qk_lane_of(int d, int rotary, bool interleaved, int c, int in) {
    const bool live = in * c < d >> 1;
    const int p = live ? in * c : 0;
    return {live, p, qk_place_of(d, rotary, interleaved, c, p)};
}

}  // namespace hq
