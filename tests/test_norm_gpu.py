"""Root-mean-square norm of rows, its output in 8 bits and its gradients, against their definitions in 64 bits."""
import numpy as np
import pytest

import delta_reference as ref
from test_sequence_gpu import NAME, TYPES, check, f64, randn

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402


def rows_of(g, lead, channels, dtype, form, scale=1.0):
    if form == "dense":
        return randn(g, *lead, channels, dtype=dtype, scale=scale)
    return randn(g, *lead, channels + 5, dtype=dtype, scale=scale)[..., 3:3 + channels]


# every layout of lanes and vectors, their last places, one row and many, whole and odd widths
CASES = [((1,), 1, 4096, "bfloat16", True, False, "dense"), ((1,), 1, 1, "float32", True, True, "dense"), ((5,), 1, 7, "float16", False, True, "wide"),
         ((3, 4), 1, 129, "bfloat16", True, True, "wide"), ((130,), 3, 100, "float16", False, True, "wide"), ((2, 33), 8, 64, "float32", True, False, "dense"),
         ((1500,), 1, 333, "bfloat16", True, False, "wide"), ((1100,), 2, 1000, "float32", False, False, "dense"), ((1030,), 1, 2048, "float16", True, False, "dense"),
         ((40,), 1, 2049, "bfloat16", True, True, "wide"), ((9,), 1, 8191, "float16", True, False, "dense"), ((3,), 1, 16384, "float32", True, False, "dense"),
         ((2,), 1, 16400, "bfloat16", True, True, "dense"), ((2,), 1, 32768, "float32", False, False, "dense"), ((2,), 1, 32767, "float16", True, False, "wide")]


def make(lead, groups, width, dtype, residual, gate, form, seed=1):
    g = torch.Generator().manual_seed(seed)
    t, D = TYPES[dtype], groups * width
    v = {"x": rows_of(g, lead, D, t, form), "w": (1 + randn(g, width, scale=0.2)).to(t)}
    v["residual"] = rows_of(g, lead, D, t, form, 2.0) if residual else None
    v["gate"] = rows_of(g, lead, D, t, form, 2.0) if gate else None
    return v


def summed(v):
    return v["x"] if v["residual"] is None else (v["x"].float() + v["residual"].float()).to(v["x"].dtype)


def flat(t):
    return None if t is None else f64(t).reshape(-1, t.shape[-1])


@pytest.mark.parametrize("lead,groups,width,dtype,residual,gate,form", CASES)
@pytest.mark.parametrize("weight", ["own", "float32", "none"])
def test_norm(lead, groups, width, dtype, residual, gate, form, weight):
    v = make(lead, groups, width, dtype, residual, gate, form)
    w = None if weight == "none" else v["w"].float() if weight == "float32" else v["w"]
    s = summed(v)
    want, kappa = ref.norm(flat(s), 1.0 if w is None else f64(w), flat(v["gate"]), groups, 1e-5)
    total = torch.full_like(s, 7.0) if residual else None
    out = ssam.ssam_rms_norm(v["x"], w, d_residual=v["residual"], d_sum=total, gate=v["gate"], groups=groups, eps=1e-5)
    assert out.shape == v["x"].shape and out.dtype == v["x"].dtype and not out.requires_grad
    if residual:
        assert torch.equal(total, s)
    check("out", out.reshape(-1, groups * width), want, ref.rounded(want, np.abs(want), kappa, dtype))
    if residual:                      # in place, and with no place for the sum
        again = v["residual"].clone()
        got = ssam.ssam_rms_norm(v["x"], w, d_residual=again, d_sum=again, gate=v["gate"], groups=groups, eps=1e-5)
        assert torch.equal(again, s) and torch.equal(got, out)
        assert torch.equal(ssam.ssam_rms_norm(v["x"], w, d_residual=v["residual"], gate=v["gate"], groups=groups, eps=1e-5), out)


@pytest.mark.parametrize("lead,groups,width,dtype,residual,gate,form", CASES)
def test_norm_e4m3(lead, groups, width, dtype, residual, gate, form):
    """A value is held within half a step, 2^-4 of it or, below the least normal number, 2^-10 of the scale; a scale is the largest magnitude's
    and two roundings off, and so is the reciprocal that a value is multiplied by."""
    v = make(lead, groups, width, dtype, residual, gate, form)
    want, kappa = ref.norm(flat(summed(v)), f64(v["w"]), flat(v["gate"]), groups, 1e-6)
    for block in {width} | {b for b in (16, 20, 32, 64, 100, 128, 333, 512) if width % b == 0}:
        total = torch.full_like(v["x"], 7.0) if residual else None
        got = ssam.ssam_rms_norm_e4m3(v["x"], v["w"], d_residual=v["residual"], d_sum=total, gate=v["gate"], groups=groups, block=block)
        assert got.values.dtype == torch.float8_e4m3fn and got.values.shape == v["x"].shape
        assert got.scales.dtype == torch.float32 and got.scales.shape == (*lead, groups * width // block)
        if residual:
            assert torch.equal(total, summed(v))
        parts = want.reshape(want.shape[0], -1, block)
        most = np.abs(parts).max(-1)
        scales = np.where(most > 0, np.maximum(most / 448, 2.0 ** -126), 1.0)
        check("scales", got.scales.reshape(scales.shape), scales, scales * (kappa.max() + 3 * ref.U))
        held = f64(got.values.float()).reshape(parts.shape) * f64(got.scales).reshape(scales.shape)[..., None]
        tol = np.maximum(np.abs(parts) * 2.0 ** -4, scales[..., None] * 2.0 ** -10) * (1 + 1e-5) + np.abs(parts) * (kappa.max() + 8 * ref.U)
        bad = np.abs(held - parts) > tol
        assert not bad.any(), (block, np.argwhere(bad)[:3], held[bad][:3], parts[bad][:3])
    assert ssam.ssam_rms_norm_e4m3(v["x"], v["w"], groups=groups).scales.shape == (*lead, groups)


def test_norm_e4m3_of_zeros_and_infinities():
    x = torch.zeros(4, 256, device="cuda")
    x[1], x[2, 5], x[3, 200] = 1e-38, float("inf"), float("nan")
    got = ssam.ssam_rms_norm_e4m3(x, eps=0.0, block=128)
    assert torch.isnan(got.values[0].float()).all()          # 0 / 0 with no eps
    got = ssam.ssam_rms_norm_e4m3(x, eps=1.0, block=128)
    assert got.scales[0].tolist() == [1.0, 1.0] and (got.values[0].float() == 0).all()
    assert got.scales[1].tolist() == [2.0 ** -126] * 2 and (got.values[1].float() - 1e-38 * 2.0 ** 126).abs().max() <= 2.0 ** -4
    assert torch.isnan(got.scales[2, 0]) and got.scales[2, 1] == 1.0
    assert torch.isnan(got.scales[3]).all() and torch.isnan(got.values[3].float()).all()


@pytest.mark.parametrize("lead,groups,width,dtype,residual,gate,form", CASES)
@pytest.mark.parametrize("weight", ["own", "float32", "none"])
def test_norm_gradients(lead, groups, width, dtype, residual, gate, form, weight):
    v = make(lead, groups, width, dtype, residual, gate, form)
    w = None if weight == "none" else v["w"].float() if weight == "float32" else v["w"]
    g = torch.Generator().manual_seed(2)
    dout = rows_of(g, lead, groups * width, TYPES[dtype], form)
    dsum = rows_of(g, lead, groups * width, TYPES[dtype], form) if residual else None
    s = summed(v)
    dx, dw, dgate, xsize, wsize, gsize, kappa = ref.norm_back(flat(dout), flat(s), 1.0 if w is None else f64(w), flat(v["gate"]), flat(dsum), groups, 1e-6)
    got = ssam.ssam_rms_norm_backward(dout, s, w, d_grad_sum=dsum, gate=v["gate"], groups=groups)
    check("x", got.x.reshape(dx.shape), dx, ref.rounded(dx, xsize, kappa, dtype))
    assert (got.weight is None) == (w is None) and (got.gate is None) == (not gate)
    if gate:
        check("gate", got.gate.reshape(dx.shape), dgate, ref.rounded(dgate, gsize, kappa, dtype))
    if w is not None:                 # sums over the rows: an addition each
        assert got.weight.dtype == w.dtype
        units = dx.shape[0] * groups
        check("weight", got.weight, dw, ref.rounded(dw, wsize, kappa + units * ref.U, NAME[w.dtype]))
    again = ssam.ssam_rms_norm_backward(dout, s, w, d_grad_sum=dsum, gate=v["gate"], groups=groups)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))


def test_norm_gradients_of_many_rows():
    """More units than the blocks take at a time, and widths that several units of a block share."""
    g = torch.Generator().manual_seed(3)
    for rows, groups, width in ((20000, 2, 40), (5000, 1, 1000)):
        x, dout, w = randn(g, rows, groups * width), randn(g, rows, groups * width), randn(g, width)
        dx, dw, _, xsize, wsize, _, kappa = ref.norm_back(f64(dout), f64(x), f64(w), None, None, groups, 1e-6)
        got = ssam.ssam_rms_norm_backward(dout, x, w, groups=groups)
        check("x", got.x, dx, ref.rounded(dx, xsize, kappa, "float32"))
        check("weight", got.weight, dw, ref.rounded(dw, wsize, kappa + rows * groups * ref.U, "float32"))


def test_norm_of_nothing():
    x, w = torch.zeros(0, 64, device="cuda"), torch.ones(64, device="cuda")
    assert ssam.ssam_rms_norm(x, w).shape == (0, 64) and ssam.ssam_rms_norm_e4m3(x, w).scales.shape == (0, 1)
    got = ssam.ssam_rms_norm_backward(x, x, w)
    assert got.x.shape == (0, 64) and (got.weight == 0).all()


def test_norm_keeps_what_lies_beside_its_rows():
    """Columns of a wider buffer, rows and sequences apart: nothing else is written."""
    buf = torch.full((3, 5, 50), 7.0, device="cuda", dtype=torch.bfloat16)
    x = randn(torch.Generator().manual_seed(4), 3, 5, 33, dtype=torch.bfloat16)
    out = buf[..., 10:43]
    assert ssam.ssam_rms_norm(x, d_out=out) is out
    assert (buf[..., :10] == 7).all() and (buf[..., 43:] == 7).all()
    turned = x.transpose(0, 1)          # the sequences' rows in turn
    assert torch.equal(ssam.ssam_rms_norm(turned), ssam.ssam_rms_norm(x).transpose(0, 1))
