"""Layouts of the sequence operators' tensors: the same numbers wherever they lie."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402
import test_sequence_gpu as base  # noqa: E402


def among_short_ones(longs, each):
    """Offsets of packed sequences: `each` of 0 .. 4 rows before every long one and behind the last."""
    starts = [3]
    for n in [*longs, None]:
        for i in range(each):
            starts.append(starts[-1] + i * 7 % 5)
        if n is not None:
            starts.append(starts[-1] + n)
    return starts


# sequences of more pieces than one among several hundred that are shorter: more sequences than pieces that another follows
MIXED = among_short_ones([500, 33, 700, 64, 32, 65, 96], 52)
base.LAYOUTS["mixed"] = ((MIXED[-1] + 2,), MIXED, None)


@pytest.mark.parametrize("spec", [("mixed", "float32", 70, 16, 1, True, True, True, True, "wide"), ("mixed", "bfloat16", 9, 4, 3, True, True, True, True, "dense"),
                                  ("mixed", "float16", 12, 40, 1, True, False, True, False, "dense")], ids=lambda s: "-".join(map(str, s)))
def test_long_sequences_among_many_short_ones(spec):
    k = base.ScanCase(*spec)
    pieces = k.rows // 32
    assert len(k.spans) > pieces                        # (pieces of 32 rows)
    assert ssam.ssam_scan_selective_workspace_bytes(k.x, k.a, spec[4], **k.seq) == 2 * pieces * (k.D * k.N + k.D) * 4
    base.test_scan_selective(spec)
    base.test_scan_selective_backward(spec)


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
