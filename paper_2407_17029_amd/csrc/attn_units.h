// How the work of a batch of paged attention is shared out, in whole numbers, host and device: a request's rows make tiles, a
// tile's positions blocks, and a tile that is longer than a unit is cut into parts of about a unit.
#pragma once
#include <cstdint>

namespace qblora {

constexpr int kUnitsBound = 1 << 26;           // above any number of units of a grid

constexpr int smaller(int a, int b) { return a < b ? a : b; }
constexpr int larger_of(int a, int b) { return a > b ? a : b; }

constexpr int kAttnBlock = 32;                 // positions of a block

// A request's positions are counted in 32 bits: at most 2^30 new tokens behind at most 2^30 - 1 positions, which is as good as any larger
// number, as a row of the table lists at most 2^30.
constexpr int context_of(int context) { return smaller(larger_of(context, 0), (1 << 30) - 1); }

// Blocks that hold what the new tokens see of the first `limit` positions
constexpr int blocks_of(int context, int fresh, int limit, int window) {
    const int hi = smaller(context + fresh, limit), lo = window ? larger_of(context + 1 - window, 0) : 0;
    return hi > lo ? (hi + kAttnBlock - 1) / kAttnBlock - lo / kAttnBlock : 1;
}

// The same for one tile, whose rows are of at most `behind` tokens behind its first: with a window it sees fewer.
constexpr int blocks_of_tile(int context, int fresh, int limit, int window, int behind) {
    const int blocks = blocks_of(context, fresh, limit, window);
    return window ? smaller(blocks, (window + behind + 2 * kAttnBlock - 2) / kAttnBlock) : blocks;
}

struct Cost { int tiles, blocks; };            // of a request: its tiles, and the blocks of each

// Blocks of a unit, from the blocks of all tiles.  A tile is at most 2^25 + 1 blocks: a unit of kLongUnit is never cut, and no larger
// one is told from it.  (The sum of all tiles may pass 2^32 times the target, where starts count tokens more than once.)
constexpr int kLongUnit = 1 << 30;
constexpr int blocks_per_unit(int64_t all, int target, int least) {
    const int64_t per = all >> 31 ? (all + target - 1) / target : ((uint32_t)all + (uint32_t)target - 1) / (uint32_t)target;
    return per >= kLongUnit ? kLongUnit : larger_of((int)per, least);
}

// The blocks of one request more, from 2^50 on as good as any larger number
constexpr int64_t add_blocks(int64_t all, const Cost& c) {
    const int64_t sum = all + (int64_t)c.tiles * c.blocks;
    return sum < (int64_t)1 << 50 ? sum : (int64_t)1 << 50;
}

struct Units { int tiles, splits, count, cuts; };                      // cuts: parts, and cut tiles in the upper half
constexpr Units units_of(const Cost& c, int per, int slack) {
    const int splits = larger_of(1, (int)(((uint32_t)c.blocks + (uint32_t)(slack ? per / 2 : per - 1)) / (uint32_t)per));
    const int count = c.tiles * splits;
    return {c.tiles, splits, count, splits > 1 ? count + (c.tiles << 16) : 0};
}

// Units of a grid that is to hold those of `tiles` tiles whose blocks are at most `blocks_of_row`: a unit more than what the target
// makes for every tile, and no more than the longest row of the table allows.
constexpr int64_t units_of_grid(int64_t tiles, int64_t blocks_of_row, int target, int least) {
    const int64_t most = tiles * ((blocks_of_row + least - 1) / least), by_target = tiles + target, units = most < by_target ? most : by_target;
    return units > 1 ? units : 1;
}

// The grid is made for requests that do not share tokens.  `starts` that do not ascend may count tokens more than once, and
// then there can be more units than the grid has: some never run, and a tile of theirs may not be joined.  So requests' units are
// added up as far as it takes to see that, and no further (the sum stays within 32 bits).
constexpr int units_within(int count, int grid_units) { return smaller(count, grid_units + 1); }
constexpr int add_units(int before, int more) { return smaller(before + more, kUnitsBound); }
constexpr int cut_tiles(int cuts, int units, int grid_units) { return units <= grid_units ? cuts >> 16 : 0; }

}  // namespace qblora
