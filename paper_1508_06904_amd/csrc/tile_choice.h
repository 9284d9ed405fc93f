// Which tile a product of codes runs on (matmul_tokens.hip, matmul_mx4.hip).  Plain C++.
#pragma once

#include <cstdint>

namespace dss {

constexpr int kStep = 128;               // bytes of K that a tile takes at a time

// The tile whose launch should take the least time.  A unit (of 256) with q tiles of
// one kind at once, `most` of them at the most, takes first + (q - 1) * more
// microseconds for the steps that its groups take at once, and `ends` for the tiles'
// beginnings and outputs; measured.
struct TileTime {
    int b, groups, most;
    double first, more, ends;
};
constexpr TileTime kTiles[] = {{256, 1, 1, 1.95, 0, 6.0}, {128, 1, 2, 0.95, 0.20, 4.0}, {64, 1, 4, 0.40, 0.17, 2.5},
                               {64, 4, 1, 1.05, 0, 3.0}};

// The index in `tiles_of` for I x J outputs of K bytes of products each.
inline int pick_tile(const TileTime* tiles_of, int n, int64_t I, int64_t J, int K) {
    int best = 0;
    double least = 0;
    for (int t = 0; t < n; ++t) {
        const TileTime& c = tiles_of[t];
        const int steps = (K + c.groups * kStep - 1) / (c.groups * kStep);
        const int64_t tiles = ((I + c.b - 1) / c.b) * ((J + c.b - 1) / c.b), full = tiles / (256 * c.most);
        const int64_t left = (tiles - full * 256 * c.most + 255) / 256;
        double time = full * (steps * (c.first + (c.most - 1) * c.more) + c.ends);
        if (left) time += steps * (c.first + (left - 1) * c.more) + c.ends;
        if (t == 0 || time < least) best = t, least = time;
    }
    return best;
}

// The index in kTiles for I x J outputs of K products each.
inline int pick_tile(int64_t I, int64_t J, int K) { return pick_tile(kTiles, 4, I, J, K); }

// The tiles of the 4-bit products, whose step of kStep bytes has twice the channels, and the index of the one for I x J
// outputs of B blocks.  Microseconds on 256, 128 and 64, a few calls after a pause (the first one 300 in long runs):
// 8192 x 8192 x 8192 346, 465, 853;
// 4096 x 4096 x 4096 47, 56, 83; 2048 x 4096 x 4096 39, 30, 45; 512 x 4096 x 4096 37, 24, 12.7; 1777 x 1003 x 2305 32, 19,
// 11.2; 300 x 300 x 2304 23, 12, 7.0; 100000 x 512 x 256 44, 43, 54; 128 x 8192 x 9216 70, 46, 19.
constexpr TileTime kMx4Tiles[] = {{256, 1, 1, 2.4, 0, 7.0}, {128, 1, 2, 1.2, 0.4, 4.5}, {64, 1, 3, 0.42, 0.13, 3.0}};
// (the small tiles hold their scales in LDS beside three buffers, of up to 28672 channels)
constexpr int kMostSmallBlocks = 896;

inline int pick_mx4_tile(int64_t I, int64_t J, int B) {
    return pick_tile(kMx4Tiles, B <= kMostSmallBlocks ? 3 : 2, I, J, B * 16);
}

}  // namespace dss
