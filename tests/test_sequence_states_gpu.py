"""Every number of states that the scans take: how they lie over the lanes changes with it."""
import pytest

import test_sequence_gpu as base

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


@pytest.mark.parametrize("states", range(1, 65))
def test_every_number_of_states(states):
    dt, form = TYPES[states % 3], "wide" if states % 2 else "dense"
    spec = ("padded", dt, 6, states, 2, True, states % 4 < 2, True, True, form)
    base.test_scan_selective(spec)
    base.test_scan_selective_backward(spec)
    base.test_scan_selective_step(dt, 6, states, 2, True)


@pytest.mark.parametrize("states", [2, 3, 6, 10, 15, 19, 31, 35, 61])
def test_odd_numbers_of_states_in_pieces(states):
    spec = ("packed_pieces", TYPES[states % 3], 9, states, 1, True, True, False, True, "dense")
    base.test_scan_selective(spec)
    base.test_scan_selective_backward(spec)
