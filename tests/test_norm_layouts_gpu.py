"""The norm where its layouts of lanes and vectors meet: from 2048 units on one wave a unit, wide units over 512 and 1024 lanes."""
import pytest

import test_norm_gpu as base

pytestmark = pytest.mark.gpu

CASES = [((2100,), 1, 900, "bfloat16", True, True, "wide"), ((2047,), 1, 900, "bfloat16", False, False, "dense"), ((1025,), 2, 2048, "float16", True, False, "dense"),
         ((2048,), 1, 513, "float32", True, True, "wide"), ((3,), 1, 6001, "float32", True, True, "wide"), ((5,), 1, 12000, "bfloat16", True, False, "dense"),
         ((2,), 2, 9000, "float16", False, True, "dense"), ((7,), 1, 4097, "float32", False, False, "dense")]


@pytest.mark.parametrize("lead,groups,width,dtype,residual,gate,form", CASES)
def test_layouts(lead, groups, width, dtype, residual, gate, form):
    case = lead, groups, width, dtype, residual, gate, form
    base.test_norm(*case, "own")
    base.test_norm_e4m3(*case)
    base.test_norm_gradients(*case, "float32")
