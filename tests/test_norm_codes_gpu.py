"""The norm's 8-bit output where y / scale lies halfway between two codes: what a block's values have in common, the root, cancels, so
that the quotient is one of the inputs' own products and goes to the even code, whatever the roundings of y and of the scale."""
import numpy as np
import pytest

from test_norm_gpu import TYPES, f64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402


def e4m3(q):
    """Nearest code's value, halves to the even one: steps of 2^-3 of a value's power of two, 2^-9 at least."""
    power = np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6)))
    step = 2.0 ** (power - 3)
    return np.rint(q / step) * step


# lanes of a block, a block that is the unit, blocks that end inside vectors, odd widths, every number of lanes
CASES = [(3000, 1, 256, 128), (2100, 2, 512, 16), (40, 1, 8192, 128), (300, 3, 100, 100), (130, 1, 4099, 4099), (64, 2, 144, 48), (50, 1, 1000, 20),
         (9, 1, 20032, 64), (2, 1, 32768, 32768), (3, 1, 30000, 1000)]


@pytest.mark.parametrize("rows,groups,width,block", CASES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated", [False, True])
def test_halves_go_to_the_even_code(rows, groups, width, block, dtype, gated):
    """Whole numbers to 224 times weights 1, 2 and 7 / 4 and gates that are powers of two from 32 on, of which the sigmoid is 1 in fp32: products of at
    most 14 bits.  The quotient 448 z / max|z| is exact in 64 bits where it is a half, h 2^e with h below 32, and otherwise off it by 1 / (h max|z|) of it at
    least, 2^-19, since the numerators are whole numbers: far more than what fp32's rounding of the quotient moves it by."""
    g = torch.Generator().manual_seed(width + block)
    t = TYPES[dtype]
    s = torch.randint(-224, 225, (rows, groups * width), generator=g).to(t).cuda()
    w = torch.tensor([1.0, 2.0, 1.75])[torch.randint(0, 3, (width,), generator=g)].to(t).cuda()
    gate = (2.0 ** torch.randint(5, 8, (rows, groups * width), generator=g)).to(t).cuda() if gated else None
    got = ssam.ssam_rms_norm_e4m3(s, w, gate=gate, groups=groups, eps=1e-5, block=block)
    z = f64(s).reshape(rows, groups, width) * f64(w) * (f64(gate).reshape(rows, groups, width) if gated else 1.0)
    r = 1.0 / np.sqrt((f64(s).reshape(rows, groups, width) ** 2).mean(-1) + 1e-5)
    z = z.reshape(rows, -1, block)
    most = np.abs(z).max(-1)
    q = z * 448 / np.where(most > 0, most, 1.0)[..., None]
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6))) - 3)
    halves = (np.abs(q / step - np.floor(q / step) - 0.5) == 0).sum()
    assert halves > 0
    want = e4m3(q).reshape(rows, -1)
    bad = f64(got.values.float()) != want
    assert not bad.any(), (int(bad.sum()), int(halves), np.argwhere(bad)[:3])
    scales = np.where(most > 0, most * np.repeat(r, width // block, -1) / 448, 1.0)
    assert (np.abs(f64(got.scales) - scales) <= scales * (48 + 8) * 2.0 ** -24).all()      # the root's error and six roundings


def test_codes_at_the_ends_of_the_range():
    """Weights from 2^-100 to 2^100, scales that are held at 2^-126, a weight that is infinite: its block's other values are zeros."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(8, 1024, generator=g).cuda()
    r = 1.0 / np.sqrt((f64(x) ** 2).mean(-1, keepdims=True) + 1e-6)
    for power in (-140, -125, -120, -100, -80, 0, 80, 100, 120):
        w = torch.full((1024,), 2.0 ** power, dtype=torch.float64).float().cuda()
        for block in (64, 1024, 128):
            got = ssam.ssam_rms_norm_e4m3(x, w, block=block)
            y = (f64(x) * r * 2.0 ** power).reshape(8, -1, block)
            scale = np.maximum(np.abs(y).max(-1) / 448, 2.0 ** -126)
            assert (np.abs(f64(got.scales) - scale) <= scale * 64 * 2.0 ** -24).all(), (power, block)
            q = y / scale[..., None]
            off = np.abs(f64(got.values.float()).reshape(y.shape) - q)
            # half a step, and what the root's error, or that of a value of few bits, moves it by
            assert (off <= np.maximum(np.abs(q) * 2.0 ** -4, 2.0 ** -10) * (1 + 1e-5) + 2.0 ** -148 / scale.min()).all(), (power, block)
    w = torch.ones(1024, device="cuda")
    w[70] = float("inf")
    got = ssam.ssam_rms_norm_e4m3(x, w, block=64)
    plain = ssam.ssam_rms_norm_e4m3(x, block=64)
    codes, others = got.values.float().reshape(8, 16, 64), plain.values.float().reshape(8, 16, 64)
    assert torch.isnan(codes[:, 1, 6]).all() and (got.scales[:, 1] == float("inf")).all()
    assert (torch.cat([codes[:, 1, :6], codes[:, 1, 7:]], -1) == 0).all()
    assert torch.equal(codes[:, 0], others[:, 0]) and torch.equal(codes[:, 2:], others[:, 2:]) and torch.equal(got.scales[:, 2:], plain.scales[:, 2:])
