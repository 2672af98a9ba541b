"""How far the sequence operators' tensors may reach, on the host: extents whose bytes or offsets do not fit 64 bits are refused, those
below are compared as they are."""
import pytest

import paper_1907_06154_amd.sequence as seq
from test_sequence_abi import ALIAS, DIM, NULL, Conv, ConvBack, ConvStep, Rows, Scan, ScanBack, ScanStep, Seq, at, call, size

FAR = 1 << 40                    # the longest stride
ROWS = 1 << 30


@pytest.fixture(scope="module")
def L():
    return seq._load()


def conv(**change):
    s = Conv(dtype=3, param_dtype=3, channels=64, taps=4, seq=Seq(1, ROWS, None, None), x=Rows(at(0), 0, 64), out=Rows(at(1), 0, 64), weight=at(-2))
    for k, v in change.items():
        setattr(s, k, v)
    return s


def test_rows_of_a_filter(L):
    f = lambda **c: call(L, "ssam_conv1d", conv(**c))  # noqa: E731
    # 2^18 rows 2^40 apart are below 2^59 elements, 2^20 and more are not; the weight lies on the result, which is found out behind that
    few, many = Seq(1, 1 << 18, None, None), Seq(1, 1 << 20, None, None)
    for name in ("x", "out"):
        far = {name: Rows(at(0), 0, FAR), "weight": at(1)}
        if name == "out":
            far["weight"], far["x"] = at(0), Rows(at(1), 0, 64)
        assert f(seq=few, **far) == ALIAS and f(seq=many, **far) == DIM and f(**far) == DIM, name
        assert f(seq=Seq(1, 1 << 18, at(40), at(41)), **far) == ALIAS and f(seq=Seq(1, ROWS, at(40), at(41)), **far) == DIM, name
        assert f(**{**far, name: Rows(at(0), 0, FAR + 1)}) == DIM, name
    # sequences as well, and both together: each below 2^59 elements
    assert f(seq=Seq(1 << 18, 2, None, None), x=Rows(at(0), FAR, 64), out=Rows(at(1), 128, 64), weight=at(1)) == ALIAS
    assert f(seq=Seq(1 << 20, 2, None, None), x=Rows(at(0), FAR, 64), out=Rows(at(1), 128, 64), weight=at(1)) == DIM
    both = Seq((1 << 18) + 1, (1 << 18) + 1, None, None)
    assert f(seq=both, x=Rows(at(0), FAR, FAR), weight=at(1), out=Rows(at(1), 64 << 19, 64)) == DIM
    # a far end that wraps around 2^64 bytes is no "no overlap": 2^23 rows of 2^40 elements of 2 bytes
    assert f(seq=Seq(1, (1 << 23) + 1, None, None), x=Rows(at(0), 0, FAR), out=Rows(at(0) + 64, 0, FAR)) == DIM


def test_rows_of_the_gradients(L):
    def make(**change):
        s = ConvBack(dtype=3, param_dtype=3, channels=64, taps=4, seq=Seq(1, 1 << 20, None, None), x=Rows(at(0), 0, 64), grad_out=Rows(at(8), 0, 64),
                     grad_in=Rows(at(16), 0, 64), weight=at(-2))
        for k, v in change.items():
            setattr(s, k, v)
        return s
    for name in ("x", "grad_out", "grad_in"):
        assert call(L, "ssam_conv1d_backward", make(**{name: Rows(at(0), 0, FAR)})) == DIM, name

    def back(**change):
        rows = {n: Rows(at(8 * i), 0, 64) for i, n in enumerate(("x", "dt", "b", "c", "grad_out", "grad_in"))}
        s = ScanBack(dtype=0, channels=64, states=16, groups=2, seq=Seq(1, 1 << 20, None, None), b_group=16, c_group=16, a=at(-1), marks=at(-4), **rows)
        for k, v in change.items():
            setattr(s, k, v)
        return s
    for name in ("grad_b", "grad_c"):
        assert call(L, "ssam_scan_selective_backward", back(**{name: Rows(at(100), 0, FAR), "work": None})) == DIM, name


def test_slots(L):
    rows = dict(x=Rows(at(1), 0, 64), out=Rows(at(2), 0, 64))
    f = lambda **c: call(L, "ssam_conv1d_step", ConvStep(**{**dict(dtype=2, param_dtype=2, channels=64, taps=4, rows=5, weight=at(3), state=at(5),  # noqa: E731
                                                                    slot_of=at(0)), **rows, **c}))
    assert f(slots=1 << 18, slot_stride=FAR, out=Rows(at(5), 0, 64)) == ALIAS and f(slots=1 << 20, slot_stride=FAR, out=Rows(at(5), 0, 64)) == DIM
    assert f(slots=ROWS, slot_stride=FAR) == DIM and f(slots=9, slot_stride=192, rows=1 << 20, x=Rows(at(1), 0, FAR)) == DIM
    more = dict(dt=Rows(at(4), 0, 64), b=Rows(at(6), 0, 64), c=Rows(at(7), 0, 64), a=at(-1), groups=2, b_group=16, c_group=16)
    g = lambda **c: call(L, "ssam_scan_selective_step", ScanStep(**{**dict(dtype=2, channels=64, states=16, rows=5, state=at(5), slot_of=at(0)),  # noqa: E731
                                                                            **rows, **more, **c}))
    assert g(slots=1 << 18, slot_stride=FAR, out=Rows(at(5), 0, 64)) == ALIAS and g(slots=1 << 20, slot_stride=FAR, out=Rows(at(5), 0, 64)) == DIM
    assert g(slots=9, slot_stride=1024, rows=1 << 20, dt=Rows(at(4), 0, FAR)) == DIM
    # groups of b: 2^18 of them 2^40 apart are within reach, 2^20 are not
    for n, want in ((18, ALIAS), (20, DIM)):
        c = dict(channels=1 << n, states=4, groups=1 << n, slots=0, slot_stride=1 << n << 2, rows=1, out=Rows(at(30), 0, 1 << n), a=at(30))
        assert g(b_group=FAR, c_group=4, **c) == want and g(b_group=4, c_group=FAR, **c) == want, n


def test_scans(L):
    rows = {n: Rows(at(8 * i), 0, 64) for i, n in enumerate(("x", "dt", "out", "b", "c"))}
    base = dict(dtype=3, channels=64, states=16, groups=2, b_group=16, c_group=16, a=at(-1), marks=None)
    f = lambda **c: call(L, "ssam_scan_selective", Scan(**{**base, **rows, **c}))  # noqa: E731
    for name in ("x", "dt", "out", "b", "c"):           # the batch stride: rows are held closer together
        assert f(seq=Seq(1 << 20, 16, None, None), **{name: Rows(at(0), FAR, 64)}) == DIM, name
    # marks of more bytes than 64 bits hold, and plans of more blocks than a launch has
    big = Seq(1 << 10, ROWS, None, None)
    wide = dict(channels=1 << 24, states=64, groups=1, **{n: Rows(at(8 * i), 0, 1 << 24) for i, n in enumerate(("x", "dt", "out"))})
    assert f(seq=big, marks=at(90), **wide) == DIM and f(seq=big, **wide) == DIM
    assert size(L, "ssam_scan_selective_workspace_bytes", Scan(**{**base, **wide, "seq": big})) == 0
    each = dict(wide, groups=1 << 24)                   # as many tiles as channels
    assert size(L, "ssam_scan_selective_workspace_bytes", Scan(**{**base, **each, "seq": big})) == 0
    assert size(L, "ssam_scan_selective_backward_workspace_bytes", ScanBack(dtype=3, channels=1 << 24, states=64, groups=1, seq=big, grad_a=at(91),
                                                                            grad_b=Rows(at(92), 0, 64))) == 0
    assert size(L, "ssam_conv1d_backward_workspace_bytes", ConvBack(dtype=3, param_dtype=3, channels=1 << 24, taps=8, seq=big, grad_bias=at(91))) == 0
    # the largest that fit a launch are planned as they are
    long = Scan(**{**base, "seq": Seq(1, ROWS, None, None)})
    assert size(L, "ssam_scan_selective_workspace_bytes", long) > 0 and f(seq=Seq(1, ROWS, None, None)) == NULL


def test_columns_of_time_major_buffers(L):
    """Halves of one buffer [rows][sequences][2 x channels] are no overlap: refused for what is checked last, not for aliasing."""
    for lead, batch, row in ((Seq(4, 1 << 28, None, None), 2048, 4 * 2048), (Seq(4, 1 << 28, None, None), 2048 << 28, 2048),
                             (Seq(1 << 30, 1, None, None), 2048, 7), (Seq(1, 1 << 30, None, None), 5, 2048)):
        f = lambda x, out: call(L, "ssam_conv1d", conv(channels=1024, taps=1, seq=lead, x=Rows(at(0) + x, batch, row),  # noqa: E731
                                                       out=Rows(at(0) + out, batch, row)))
        assert f(0, 2048) == DIM and f(2048, 0) == DIM and f(0, 2046) == ALIAS and f(2046, 0) == ALIAS and f(2048, 2) == ALIAS, (batch, row)
    # an input that all sequences share, and one that all rows share, beside a result in the other half
    wide = dict(channels=1024, taps=1, seq=Seq(4, 1 << 28, None, None))
    assert call(L, "ssam_conv1d", conv(x=Rows(at(0), 0, 4 * 2048), out=Rows(at(0) + 2048, 2048, 4 * 2048), **wide)) == ALIAS     # (other strides)
    assert call(L, "ssam_conv1d", conv(x=Rows(at(0), 0, 2048), out=Rows(at(0) + 2048, 2048 << 28, 2048), **wide)) == DIM
    assert call(L, "ssam_conv1d", conv(x=Rows(at(0), 2048, 0), out=Rows(at(0) + 2048, 2048, 4 * 2048), **wide)) == DIM
    assert call(L, "ssam_conv1d", conv(x=Rows(at(0), 2048, 0), out=Rows(at(0) + 2046, 2048, 4 * 2048), **wide)) == ALIAS
