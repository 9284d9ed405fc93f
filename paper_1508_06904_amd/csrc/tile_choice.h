// Which tile a product of 8-bit codes runs on (matmul_tokens.hip).  Plain C++.
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

// The index in kTiles for I x J outputs of K products each.
inline int pick_tile(int64_t I, int64_t J, int K) {
    int best = 0;
    double least = 0;
    for (int t = 0; t < 4; ++t) {
        const TileTime& c = kTiles[t];
        const int steps = (K + c.groups * kStep - 1) / (c.groups * kStep);
        const int64_t tiles = ((I + c.b - 1) / c.b) * ((J + c.b - 1) / c.b), full = tiles / (256 * c.most);
        const int64_t left = (tiles - full * 256 * c.most + 255) / 256;
        double time = full * (steps * (c.first + (c.most - 1) * c.more) + c.ends);
        if (left) time += steps * (c.first + (left - 1) * c.more) + c.ends;
        if (t == 0 || time < least) best = t, least = time;
    }
    return best;
}

}  // namespace dss
