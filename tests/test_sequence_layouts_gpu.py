"""Layouts of the sequence operators' tensors: the same numbers wherever they lie."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402


def test_halves_of_a_time_major_buffer():
    """[rows, sequences, 2 channels]: inputs are one half, results the other."""
    T, S, D, N = 200, 3, 96, 16
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    one, two = rand(T, S, 2 * D).transpose(0, 1), rand(T, S, 2 * D).transpose(0, 1)
    w, a, b, c = rand(D, 4), -rand(D, N).abs() - 0.1, rand(S, T, 1, N), rand(S, T, 1, N)
    x, dt = one[..., :D], two[..., :D]
    want = ssam.ssam_conv1d(x.contiguous(), w, silu=True)
    out = one[..., D:]
    kept = x.clone()
    assert ssam.ssam_conv1d(x, w, silu=True, d_out=out) is out
    assert torch.equal(out, want) and torch.equal(x, kept)
    want = ssam.ssam_scan_selective(x.contiguous(), dt.contiguous(), a, b, c, softplus=True)
    out = two[..., D:]
    assert ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True, d_out=out) is out
    assert torch.equal(out, want) and torch.equal(x, kept)
