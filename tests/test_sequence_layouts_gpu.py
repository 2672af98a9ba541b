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


def test_more_sequences_than_a_launch_has_blocks_for_their_joins():
    """4200 sequences x 2^20 states in blocks of 256 are more than 2^24 blocks; one sequence is long enough to be cut, the others have a row."""
    S, D, N = 4200, 16384, 64
    long = 2000
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    lengths = [1] * S
    lengths[4111] = long
    starts = torch.tensor([0, *lengths], device="cuda").cumsum(0).to(torch.int32)
    T = int(starts[-1])
    x, dt, b, c = rand(T, D), rand(T, D), rand(T, 1, N), rand(T, 1, N)
    a = -torch.rand(D, N, generator=g, device="cuda") - 0.1
    out = ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True, starts=starts)
    lo = int(starts[4111])
    rows = slice(lo, lo + long)
    # the same sequence alone is cut elsewhere: the same states up to fp32's roundings, results up to one of theirs
    alone = ssam.ssam_scan_selective(x[rows], dt[rows], a, b[rows], c[rows], softplus=True)
    assert ssam.ssam_scan_selective_workspace_bytes(x, a, starts=starts) > 0
    assert (out[rows].float() - alone.float()).abs().max() <= 2 ** -7 * alone.float().abs().max()
    # single rows: y = d u (b . c), products and sums of fp32
    d = torch.nn.functional.softplus(dt[:lo].double())
    want = d * x[:lo].double() * (b[:lo, 0].double() * c[:lo, 0].double()).sum(-1, keepdim=True)
    mag = d * x[:lo].double().abs() * (b[:lo, 0].double() * c[:lo, 0].double()).abs().sum(-1, keepdim=True)
    assert ((out[:lo].double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.001 + 100 * 2.0 ** -24 * mag).all()


def test_marks_that_no_card_holds():
    """2^26 entries of a megabyte: torch's own error, before anything runs."""
    x = torch.zeros(1, 4096, device="cuda").expand(1 << 30, 4096)
    with pytest.raises(torch.OutOfMemoryError):
        ssam.ssam_scan_selective_marks(x, torch.zeros(4096, 64, device="cuda"))
    out = ssam.ssam_conv1d(x[:8], torch.ones(4096, 2, device="cuda"))      # and the next call is none the worse
    assert not out.any()
