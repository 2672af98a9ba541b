"""What the scans' workspaces take, on the host."""
import pytest

import paper_1907_06154_amd.sequence as seq
from test_sequence_abi import Scan, ScanBack, Seq, at, size


@pytest.fixture(scope="module")
def L():
    return seq._load()


def forward(L, D, N, s):
    return size(L, "ssam_scan_selective_workspace_bytes", Scan(dtype=3, channels=D, states=N, groups=1, seq=s))


def back(L, D, N, s, **want):
    return size(L, "ssam_scan_selective_backward_workspace_bytes", ScanBack(dtype=3, channels=D, states=N, groups=1, seq=s, **want))


def test_many_short_sequences_take_no_more_than_long_ones(L):
    """Only pieces that another follows keep states: rows / piece of them, and as many sequences' first ones."""
    D, N, rows = 4096, 16, 32768
    plane, line = D * N * 4, D * 4
    for S in (4096, 8192, 30000):
        s = Seq(S, rows, at(0), at(1))
        assert forward(L, D, N, s) == 2 * 16 * (plane + line)          # pieces of 2048 rows
        assert back(L, D, N, s) == 16 * (plane + line)
        # the parameters' gradients: 512 slots of 64 channel tiles are 2^15 blocks
        assert back(L, D, N, s, grad_a=at(2)) == 16 * (plane + line) + 512 * (plane + 2 * line)
        assert back(L, D, N, Seq(S, 8, None, None), grad_skip=at(2)) == 512 * (plane + 2 * line)
    # a batch has what its sequences are cut into
    assert forward(L, D, N, Seq(1, 4096, None, None)) == 16 * (plane + line)
    assert back(L, D, N, Seq(1, 4096, None, None)) == 16 * (plane + line)
