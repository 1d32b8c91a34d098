// Which tiles of dw each XCD takes: arithmetic alone, for the device and for a host's compiler.
#pragma once

namespace moe {

constexpr int kDwStart = 96;  // rows of reduction that the start and end of a tile of dw are counted as (1 to 384: the same times within 1 %)
constexpr int kDwLists = 8;   // one per XCD

// The first tile of list `x` of kDwLists (x = kDwLists: behind the last tile): stretches of about the same work, where each of an expert's `per` tiles is
// worth its used[e] rows and kDwStart.  first[e]: what the experts before e come to, `total`: all of them.  Rows are up to 2^30, so that eight
// times their number, and that times `per` (up to 2^30 / E), are products in 64 bits.
constexpr int dw_edge(int x, int E, int per, int total, const int *first, const int *used) {
    typedef unsigned long long u64;
    if (x == kDwLists) return E * per;
    const u64 at = (u64)x * (u64)total;
    int e = 0;
    for (int step = 128; step; step >>= 1)
        if (e + step < E && first[e + step] <= (int)(at / kDwLists)) e += step;
    return e * per + (int)((at - (u64)kDwLists * (u64)first[e]) * (u64)per / ((u64)kDwLists * (u64)(used[e] + kDwStart)));
}

}  // namespace moe
