"""The weight's gradient of the norm where it is exact: elements of magnitude 1, whose root is 1, and whole numbers as gradients, so that every sum of
fp32 is one of whole numbers below 2^24.  A unit that is lost, or counted twice, in any of the sums' stages is seen."""
import pytest

from test_norm_gpu import TYPES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402

# one round of the blocks and several, every number of lanes, several units of a block, odd widths, units that do not fill the last round
CASES = [(1, 1, 40), (17, 1, 100), (1024, 1, 64), (16384, 1, 40), (16385, 1, 128), (20000, 2, 40), (70001, 1, 16), (4096, 1, 512), (5000, 1, 1000), (9001, 3, 333),
         (2047, 1, 2048), (3000, 1, 4096), (2500, 1, 6001), (1500, 1, 8192), (1030, 1, 16384), (1100, 1, 30000)]


@pytest.mark.parametrize("rows,groups,width", CASES)
@pytest.mark.parametrize("dtype", TYPES)
def test_every_unit_is_summed_once(rows, groups, width, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + width)
    t, D = TYPES[dtype], groups * width
    whole = lambda lo, hi: torch.randint(lo, hi, (rows, D), generator=g, device="cuda")  # noqa: E731
    s, d = 2 * whole(0, 2) - 1, 2 * whole(-4, 4) + 1         # +-1; -7, -5 .. 7
    w = torch.ones(width, device="cuda")
    want = (s * d).reshape(-1, width).sum(0)
    assert (s * d).abs().reshape(-1, width).sum(0).max() < 1 << 24
    got = ssam.ssam_rms_norm_backward(d.to(t), s.to(t), w, groups=groups, eps=0.0)
    assert torch.equal(got.weight.double(), want.double()), int((got.weight.double() != want.double()).sum())
    own = ssam.ssam_rms_norm_backward(d.to(t), s.to(t), w.to(t), groups=groups, eps=0.0)
    assert torch.equal(own.weight, want.to(t))
    # a gate of 64, of which the sigmoid is 1 in fp32; as much of it as keeps the sums below 2^24
    if rows * groups < 1 << 15:
        gate = torch.full((rows, D), 64.0, dtype=t, device="cuda")
        gated = ssam.ssam_rms_norm_backward(d.to(t), s.to(t), w, gate=gate, groups=groups, eps=0.0)
        assert torch.equal(gated.weight.double(), 64.0 * want.double())
