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

// Workgroups of 256 threads that one launch takes: fewer than 2^32 threads.  More go out in launches one after another, workgroup `block` of the next being
// number `first` + block of all; they go on with the counters, so that what a workgroup waits for still runs already or has run.
constexpr uint32_t MOST_WORKGROUPS = (1u << 24) - 8;
constexpr uint32_t workgroups_from(uint32_t first, uint32_t all) { return all - first < MOST_WORKGROUPS ? all - first : MOST_WORKGROUPS; }

}  // namespace ssdk
