// Which tile of channels and which chunk along the sequence a workgroup of the gated recurrence (gated_scan.hip) works on.  Plain C++ without device
// types: which places a launch hands out can be walked through on the host.
#pragma once
#include <stdint.h>

namespace ssdk {

// The tile (of `side` = tiles of a sequence times sequences) of workgroup `block`.  Workgroups go to the eight XCDs in turn.  Each takes tiles side
// by side, which share lines where rows are no whole number of them (8 x 22844 tokens of 3672 channels, forward and backward: 3.80 ms, the tiles in
// turn as well 4.35; 30000 of 2561 506 us and 552), and goes on by as many from chunk to chunk: with the same ones for good it asks its L2 for
// an eighth of the lines' slots (65536 tokens of 5120 channels: 1.87 ms, going on 1.58).
constexpr uint32_t tile_of(uint32_t block, uint32_t side) {
    const uint32_t each = side >> 3, rest = side & 7, turn = block / side, pos = block - turn * side, xcd = pos & 7;
    return (xcd * each + (xcd < rest ? xcd : rest) + (pos >> 3) + turn * (each + 1)) % side;
}
// Whether the chunk that a tile's counter gave is one of the launch's.  Alone on its workspace a launch draws 0 .. chunks - 1 from each counter.  Beside
// another call, which clears the counters, draws from them or lays other words in their place, it may draw any number: what is no chunk of
// its own it leaves alone, so that such calls stay inside their tensors.
constexpr bool chunk_there(uint32_t drawn, uint32_t chunks) { return drawn < chunks; }

// A launch takes fewer than 2^32 threads, of 256 a workgroup, along a dimension.  More workgroups than that lie in rows of ROW, the last of them with
// some to spare, which draw no chunk of the launch's.  Its number is a workgroup's place in the grid alone: an argument that says where a launch begins
// is waited for in front of everything else (3 x 2001 tokens of 2048 channels, packed, forward and backward: 80.1 us, without 78.1).
constexpr uint32_t ROW = 1u << 16, MOST_IN_LINE = (1u << 24) - 1;
struct Grid {
    uint32_t x, y;
};
constexpr Grid grid_of(uint32_t workgroups) { return workgroups <= MOST_IN_LINE ? Grid{workgroups, 1} : Grid{ROW, (workgroups - 1) / ROW + 1}; }
constexpr uint32_t number_of(uint32_t x, uint32_t y) { return y * ROW + x; }

}  // namespace ssdk
