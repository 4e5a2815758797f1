// How the narrow products of the adapters (adapters.hip) walk k, and which row of a factor with k as the row index a lane asks for.  Plain
// C++ without device types: what a launch asks for can be walked through on the host.
#pragma once

namespace ssdk {

constexpr int SHORT_UNIT = 32;              // rows of a unit
constexpr int LWAVES = 8, LSTEP = 64;       // waves of a workgroup, which take steps of 64 k in turn

// Steps of a wave that are asked for together, by ranks (16 rt) and rows (16 mt) of a workgroup; the distance in k from the first of them
// to the wave's next ones; and whether all k of those from k0 on exist.
constexpr int low_group(int rt, int mt) { return rt == 4 ? 2 : mt == 1 ? 6 : 4; }
constexpr int low_advance(int group) { return LSTEP * LWAVES * group; }
constexpr bool low_whole(int k0, int group, int K) { return k0 + LSTEP * (LWAVES * (group - 1) + 1) <= K; }

// A factor stored as [K][rank]: the lanes of a wave take the 16-byte pieces of a step's rows one after another, `per_row` of them to a
// row, in accesses of 64.  Where the workgroup has fewer than its 16 rt ranks the last accesses have more pieces than the 64 rows: there a lane
// is to ask for a row that the step has (and keep nothing of it).
constexpr int low_piece_row(int piece, int per_row) { return piece / per_row; }
constexpr bool low_piece_there(int row) { return row < LSTEP; }
constexpr int low_piece_asked(int row) { return row < LSTEP ? row : 0; }
// The row of the factor that is asked for in the step from ks on; `whole`: all of the step's rows exist.  Always one of 0 .. K - 1.
constexpr int low_row_asked(int ks, int asked, bool whole, int K) { return whole || ks + asked < K ? ks + asked : 0; }

}  // namespace ssdk
