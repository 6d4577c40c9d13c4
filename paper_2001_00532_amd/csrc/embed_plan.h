// What the gradient of the embedding lookup decides from sizes and tokens alone, in plain C++: kernels, host code and tests on a machine without a GPU share it.
#pragma once
#include <algorithm>
#include <cstdint>

namespace psk {

// A token's place among the `count` rows from `first` on, if it is less than count.  Unsigned: a token may be any 32-bit number, and those before `first` and
// below 0 have places from 2^31 - 2^28 on, behind any rows that there are.
constexpr unsigned place_from(int id, int first) { return (unsigned)id - (unsigned)first; }

// ------------------------------------------------------------------ how tokens are sorted
constexpr int SORT = 2048;                                 // positions per workgroup where several sort
constexpr int BASES = 128;                                 // workgroups whose counts every one of them adds up by itself
constexpr int NEAR = 65536, RANGES = 1024, MOST_ROWS = 512;      // tokens that every workgroup reads; workgroups that own rows, and how many each
constexpr int SMALL = 1024;                                // tokens, of 4 MB in all, whose sums are in the sort's launch
enum Way { NO_TOKENS, ONE_LAUNCH, BY_RANGES, BY_DIGITS, BY_SCANNED_DIGITS };
// `bytes`: of an element of dY
inline Way way_of(int n, int rows, int dim, int bytes)
{
    if (n == 0) return NO_TOKENS;
    if (n <= NEAR && rows <= RANGES * MOST_ROWS) return n <= SMALL && dim >= 4 && (int64_t)n * dim * bytes <= 4 << 20 ? ONE_LAUNCH : BY_RANGES;
    return (n + SORT - 1) / SORT > BASES ? BY_SCANNED_DIGITS : BY_DIGITS;
}

// ------------------------------------------------------------------ how their rows are added up
constexpr int MAX_TILE = 64;                               // positions per tile, at most one to a lane

// 256 J columns to a wave: a wave's work is about J + 1 for each position.
inline int quads_per_lane(int64_t dim)
{
    int best = 1;
    int64_t least = INT64_MAX;
    for (int j = 1; j <= 3; ++j) {
        const int64_t cost = (dim + 256 * j - 1) / (256 * j) * (j + 1);
        if (cost < least) {
            least = cost;
            best = j;
        }
    }
    return best;
}
// Positions to a tile: as many as leave 4096 waves, but 16 to 64 (up to FEW tokens 8): a row of many tokens has
// as many parts to join.  16000 tokens of 512 columns, nine tenths of them one: tiles of 8 joined in 34 us and added up in 10, of 16 in 18 and 11 (256 columns to a workgroup that joins).
constexpr int FEW = 2048;
inline int tile_of(int64_t n, int64_t dim)
{
    const int64_t j = 256 * quads_per_lane(dim), chunks = (dim + j - 1) / j;
    int tile = MAX_TILE;
    while (tile > (n <= FEW ? 8 : 16) && n * chunks < (int64_t)tile * 4096) tile /= 2;
    return tile;
}
// As many tiles as n or fewer tokens are cut into at most, so that a workspace for n is one for fewer.
inline int64_t most_tiles(int64_t n, int64_t dim)
{
    const int64_t j = 256 * quads_per_lane(dim), chunks = (dim + j - 1) / j, few = std::max((std::min(n, (int64_t)FEW) + 7) / 8, std::min((n + 15) / 16, 8192 / std::max(chunks, (int64_t)1) + 1));
    return std::max((n + MAX_TILE - 1) / MAX_TILE, few);
}

}  // namespace psk
