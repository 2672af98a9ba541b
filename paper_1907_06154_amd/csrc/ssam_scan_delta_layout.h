// Which rows and elements of q and k a thread of the scan with matrix states reads: plain arithmetic, so that a program on the host can go
// through all of it.
#pragma once

#include "../../include/ssam_sequence.h"

namespace ssam {

// Element from which eight of a row of dim >= 8 are read that are to be 8 e ..: a vector that would pass the last element starts further left.
constexpr unsigned eights_at(int e, int dim) { return (unsigned)(8 * e + 8 <= dim ? 8 * e : dim - 8); }
// Row that is read in the place of `row`, of rows >= 1: copies of the last one behind it.
constexpr int eights_row(int row, int rows) { return row < rows ? row : rows - 1; }

// How the threads of a block share 64 rows of 32 KT elements, eight elements a lane: rows row(thread), row(thread) + kAtOnce ..
template <int KT, int kThreads>
struct RowLanes {
    static constexpr int kLanes = 4 * KT, kAtOnce = kThreads / kLanes, kPasses = SSAM_DELTA_ROWS > kAtOnce ? SSAM_DELTA_ROWS / kAtOnce : 1;      // lanes of a row, rows
    static constexpr int place(int thread) { return thread / kLanes; }
    // The first row that a thread reads, also where the block is whole and rows are not looked at one by one: threads that are more than
    // there are places read the last row.
    static constexpr int row(int thread) { return kAtOnce > SSAM_DELTA_ROWS && place(thread) >= SSAM_DELTA_ROWS ? SSAM_DELTA_ROWS - 1 : place(thread); }
};

// How the threads share the squares of 8 rows x 8 elements of a block's k, and then of its q.  A wave's are of one of them, also where 32 squares
// are half of it: the distance from row to row is one value for all lanes (load_eights), and those of q need not be k's.
template <int KT>
struct StageLanes {
    static constexpr int kAcross = 4 * KT, kSquares = 8 * kAcross;
    static constexpr int kSide = kSquares < 64 ? 64 : kSquares, kJobs = 2 * kSide;
    static constexpr bool has(int job) { return job < kJobs && job % kSide < kSquares; }
    static constexpr bool query(int job) { return job >= kSide; }
    static constexpr int rows(int job) { return (job % kSide) / kAcross; }      // 8 of them
    static constexpr int elements(int job) { return job % kAcross; }
};

}  // namespace ssam
