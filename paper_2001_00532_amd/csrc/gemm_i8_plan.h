// How a product of 8-bit integers is cut up, from its sizes alone, in plain C++: host code and tests on a machine without a GPU share it.
#pragma once
#include <cstdint>

namespace psk {

constexpr int STEP = 128;                                  // columns, and bytes of a row of a stage

// Tiles by their tokens and channels, and how long a step of 128 columns of one takes, in 10 ns: of the first 256 tiles (a compute unit has one), and
// of each 256 more, which overlap where a compute unit has room for several.  Measured with 4096 columns and channels; the least sum is within a tenth of the
// best shape for 1024 to 32768 channels, 2048 to 8192 columns and 5 to 2048 tokens, but for a sixth at one of 55 places.
struct Shape { int tokens, channels, first, more; };
constexpr Shape SHAPES[] = {{16, 16, 19, 6}, {16, 32, 19, 9}, {32, 32, 22, 11}, {32, 64, 23, 16}, {64, 32, 25, 15}, {64, 64, 28, 21}, {128, 64, 36, 42}, {128, 128, 46, 58},
                            {256, 128, 78, 80}, {256, 256, 118, 118}};
constexpr int SHAPE_COUNT = sizeof(SHAPES) / sizeof(SHAPES[0]);

// Few tiles of many columns: the columns in 2 to 16 parts, whose sums another launch adds up.  That takes 4.5 us and writing and reading the sums at 4 TB/s; they
// have SUM_ROOM at most.  300 channels, 16384 columns, 7 tokens, quantised on the way: 18.7 us, 33 in one part; 1024 x 8192 with 64 tokens 11.0 and 14.3.  (With 3 us
// instead, 4096 x 4096 and 5 tokens went in two parts and took 11.6 us for 9.1.)
constexpr int MOST_PARTS = 16;
constexpr int64_t SUM_ROOM = 16 << 20;
struct Choice { int shape, parts, part_cols; };
inline int64_t pitch_of(int rows) { return ((int64_t)rows + 3) / 4 * 4; }
inline Choice choose(int rows, int cols, int n)
{
    const int steps = (cols + STEP - 1) / STEP;
    Choice best = {0, 1, cols};
    int64_t least = INT64_MAX;
    for (int parts = 1; parts <= MOST_PARTS; parts *= 2) {
        const int64_t bytes = parts * (int64_t)n * pitch_of(rows) * 4;
        const int each = (steps + parts - 1) / parts;
        if (parts > 1 && (bytes > SUM_ROOM || (int64_t)each * (parts - 1) >= steps)) break;
        const int64_t join = parts > 1 ? 4500 + bytes * 2 / 4000 : 0;            // ns
        for (int i = 0; i < (parts > 1 ? SHAPE_COUNT - 1 : SHAPE_COUNT); ++i) {        // SUM_ROOM is 64 of the largest tiles: smaller ones are faster, and it has no form for parts
            const int64_t all = (int64_t)((n + SHAPES[i].tokens - 1) / SHAPES[i].tokens) * ((rows + SHAPES[i].channels - 1) / SHAPES[i].channels) * parts;
            const int64_t cost = join + (SHAPES[i].first + (all - 1) / 256 * SHAPES[i].more) * 10 * (each > 0 ? each : 1);
            if (cost < least) {
                least = cost;
                best = {i, parts, each * STEP};
            }
        }
    }
    return best;
}

}  // namespace psk
