"""Which rows and elements of q and k the kernels of the scan with matrix states read, thread by thread: the header that they take them from,
in a program on the host.  Nothing outside of a block's rows may be read, whatever is done with it."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1907_06154_amd", "csrc")

ROWS = r"""
#include "ssam_scan_delta_layout.h"
#include <cstdio>
using namespace ssam;

static int bad;
static void refuse(const char* what, int kt, int threads, int thread, int row)
{
    if (bad++ < 3) std::printf("%s: keys to %d, %d threads: thread %d, row %d\n", what, 32 * kt, threads, thread, row);
}
template <int KT, int kThreads> void rows()
{
    typedef RowLanes<KT, kThreads> L;
    bool seen[SSAM_DELTA_ROWS][4 * KT] = {};
    for (int thread = 0; thread < kThreads; ++thread)
        for (int i = 0; i < L::kPasses; ++i) {
            // a whole block: no row is held back
            const int row = L::row(thread) + i * L::kAtOnce, place = L::place(thread) + i * L::kAtOnce;
            if (row < 0 || row >= SSAM_DELTA_ROWS) refuse("read behind the block", KT, kThreads, thread, row);
            if (place < SSAM_DELTA_ROWS) {
                if (row != place) refuse("not the row of its place", KT, kThreads, thread, row);
                bool& there = seen[place][thread % L::kLanes];
                if (there) refuse("twice", KT, kThreads, thread, row);
                there = true;
            }
        }
    for (auto& r : seen)
        for (bool there : r)
            if (!there) refuse("missing", KT, kThreads, -1, -1);
}

int main()
{
    rows<1, 256>(), rows<2, 256>(), rows<4, 256>(), rows<8, 256>();
    rows<1, 512>(), rows<2, 512>(), rows<4, 512>(), rows<8, 512>();
    for (int rows = 1; rows <= SSAM_DELTA_ROWS; ++rows)
        for (int row = 0; row < 2 * SSAM_DELTA_ROWS; ++row)
            if (eights_row(row, rows) < 0 || eights_row(row, rows) >= rows || (row < rows && eights_row(row, rows) != row)) refuse("of fewer rows", 0, 0, row, rows);
    for (int dim = 8; dim <= SSAM_MAX_KEY; ++dim)
        for (int e = 0; e < SSAM_MAX_KEY / 8; ++e) {
            const unsigned at = eights_at(e, dim);
            if (at + 8 > (unsigned)dim || (8 * e + 8 <= dim && at != 8u * e)) refuse("elements", 0, dim, e, (int)at);
        }
    return bad != 0;
}
"""

SQUARES = r"""
#include "ssam_scan_delta_layout.h"
#include <cstdio>
using namespace ssam;

static int bad;
template <int KT> void squares()
{
    typedef StageLanes<KT> L;
    bool seen[2][8][4 * KT] = {};
    for (int wave = 0; wave < (L::kJobs + 63) / 64; ++wave) {
        int side = -1;      // a wave reads k or q: their rows' distance is one value for all of its lanes
        for (int job = 64 * wave; job < 64 * wave + 64; ++job) {
            if (!L::has(job)) continue;
            if (side < 0) side = L::query(64 * wave);
            if (L::query(job) != (side != 0) && bad++ < 3) std::printf("keys to %d: thread %d reads q, the wave's first %s\n", 32 * KT, job, side ? "q" : "k");
            if (L::rows(job) < 0 || L::rows(job) >= 8 || L::elements(job) < 0 || L::elements(job) >= 4 * KT) {
                if (bad++ < 3) std::printf("keys to %d: thread %d is outside\n", 32 * KT, job);
                continue;
            }
            bool& there = seen[L::query(job)][L::rows(job)][L::elements(job)];
            if (there && bad++ < 3) std::printf("keys to %d: thread %d again\n", 32 * KT, job);
            there = true;
        }
    }
    for (auto& s : seen)
        for (auto& r : s)
            for (bool there : r)
                if (!there && bad++ < 3) std::printf("keys to %d: a square is missing\n", 32 * KT);
}

int main()
{
    squares<1>(), squares<2>(), squares<4>(), squares<8>();
    return bad != 0;
}
"""


@pytest.mark.parametrize("program", [ROWS, SQUARES], ids=["rows", "squares"])
def test_what_the_threads_read(program, tmp_path):
    (tmp_path / "p.cpp").write_text(program)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "p"), str(tmp_path / "p.cpp")], check=True)
    r = subprocess.run([str(tmp_path / "p")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
