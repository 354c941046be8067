// Tiles of the gated projection's products.  No more than arithmetic: the host's compilers take it too.
#pragma once
#include <algorithm>

namespace ucd {
namespace gated {

inline long round_up(long n, long to) { return (n + to - 1) / to * to; }

constexpr int kStep = 64;              // of a reduction
constexpr int kFewTokens = 64;
constexpr int kUnits = 256;            // compute units

// Tiles of 256 by 256 or 192 by 256, one to a unit, or of 128 by 128, two to a unit, whichever take least time in whole rounds; the reduction in parts of 8
// steps at least where small ones are too few.  A round of the second has 3/4 of the first one's work, a round of small ones half of it at about 0.7 of the
// rate (forward of 4096 x 1024 x 2816: two rounds of 256 by 256 65 us, two of 192 by 256 56 us).  Tiles of 192 are of operands along their rows alone.
struct Shape {
    int side;      // rows of a tile
    int tiles_m, tiles_n, splits;
};

inline Shape shape_of(long m, long n, long steps, bool along)
{
    auto tiles = [&](long rows, long cols) { return ((m + rows - 1) / rows) * ((n + cols - 1) / cols); };
    auto rounds = [](long t, long each) { return (double)((t + each - 1) / each); };
    const double large = rounds(tiles(256, 256), kUnits), mid = rounds(tiles(192, 256), kUnits) * 0.75 / 0.95,
                 small = rounds(tiles(128, 128), 2 * kUnits) * 0.5 / 0.7;
    Shape s;
    s.side = along && mid < large && mid <= small ? 192 : large <= small ? 256 : 128;
    s.tiles_m = (int)((m + s.side - 1) / s.side);
    const int cols = s.side == 128 ? 128 : 256;
    s.tiles_n = (int)((n + cols - 1) / cols);
    s.splits = s.side != 128 ? 1 : (int)std::max(1l, std::min(2 * kUnits / tiles(128, 128), steps / 8));
    return s;
}

// One row of tiles of 64 by 128, three to a unit, and parts of 8 steps at least: 2048 -> 8192, 64 tokens, four parts 20.3 us, two 21.1, six 24.2.
inline Shape low_shape(long n, long steps)
{
    const long tiles = (n + 127) / 128;
    return Shape{64, 1, (int)tiles, (int)std::max(1l, std::min(3 * kUnits / tiles, steps / 8))};
}

// The three products of M tokens, D -> F; fp32 operands go over the reduction `phases` times.
inline Shape forward_shape(long M, long D, long F, int phases)
{
    const long steps = (round_up(D, 8) + kStep - 1) / kStep * phases;
    return M <= kFewTokens ? low_shape(2 * F, steps) : shape_of(M, 2 * F, steps, true);
}
inline Shape dx_shape(long M, long D, long F, int phases) { return shape_of(M, D, 2 * round_up(F, kStep) / kStep * phases, true); }
inline Shape dw_shape(long M, long D, long F, int phases) { return shape_of(2 * round_up(F, kStep), D, (M + kStep - 1) / kStep * phases, false); }

}  // namespace gated
}  // namespace ucd
