"""Infinities and NaN at the sequence operators' edges: what lies behind a sequence, above it, between its pieces and behind its states
adds nothing, not even zero times an infinity."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402

INF = float("inf")
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g).to(dtype).cuda()


# pieces of 8 rows: sequences that end inside one, with it, and one row behind it (which the piece before looks at)
@pytest.mark.parametrize("value", [INF, float("nan")])
@pytest.mark.parametrize("rows,W", [(5, 4), (8, 2), (9, 4), (17, 8), (33, 3), (1, 5), (64, 4)])
def test_the_last_input_reaches_the_last_tap_alone(rows, W, value):
    for dtype in TYPES:
        print(dtype, flush=True)
        g = torch.Generator().manual_seed(rows)
        D, at = 70, 11
        x, dy, w = (randn(g, *s, dtype=dtype) for s in ((rows, D), (rows, D), (D, W)))
        h = randn(g, 1, W - 1, D, dtype=dtype)
        clean = ssam.ssam_conv1d_backward(dy, x, w, d_state=h)
        x[-1, at] = value
        got = ssam.ssam_conv1d_backward(dy, x, w, d_state=h)
        assert not torch.isfinite(got.weight[at, W - 1])
        got.weight[at, W - 1] = clean.weight[at, W - 1]
        assert torch.equal(got.weight, clean.weight) and torch.equal(got.x, clean.x)


def test_the_carried_rows_of_an_empty_sequence_reach_no_tap():
    g = torch.Generator().manual_seed(1)
    D, W = 70, 4
    x, dy, w, h = randn(g, 3, 9, D), randn(g, 3, 9, D), randn(g, D, W), randn(g, 3, W - 1, D)
    lengths = torch.tensor([9, 0, 4], dtype=torch.int32, device="cuda")
    clean = ssam.ssam_conv1d_backward(dy, x, w, d_state=h, lengths=lengths)
    h[1] = INF
    got = ssam.ssam_conv1d_backward(dy, x, w, d_state=h, lengths=lengths)
    assert torch.equal(got.weight, clean.weight) and torch.equal(got.x, clean.x)


@pytest.mark.parametrize("rows,W", [(5, 4), (8, 2), (9, 4), (17, 8), (2, 5), (0, 3), (64, 4)])
def test_a_tap_reaches_the_rows_under_it_alone(rows, W):
    """An infinite tap j: the gradient of row t has it only where row t + W - 1 - j is one of the sequence."""
    g = torch.Generator().manual_seed(rows)
    D, at = 70, 11
    x, dy, w = randn(g, rows, D), randn(g, rows, D), randn(g, D, W)
    dlast = randn(g, 1, W - 1, D)
    clean = ssam.ssam_conv1d_backward(dy, x, w, d_grad_final=dlast, state_grad=True)
    for j in range(W):
        there = w[at, j].item()
        w[at, j] = INF
        got = ssam.ssam_conv1d_backward(dy, x, w, d_grad_final=dlast, state_grad=True)
        w[at, j] = there
        grads = torch.cat([got.state[0], got.x])                     # rows -(W - 1) .. rows - 1
        want = torch.cat([clean.state[0], clean.x])
        t = torch.arange(-(W - 1), rows, device="cuda") + W - 1 - j
        has = (t >= 0) & (t < rows)
        assert not torch.isfinite(grads[has, at]).any()
        grads[has, at] = want[has, at]
        assert torch.equal(grads, want), j


@pytest.mark.parametrize("rows", [5, 16, 33, 250])
@pytest.mark.parametrize("N", [4, 8, 16, 32, 64])
def test_the_last_state_reaches_no_rate(rows, N):
    """The gradient at a decay rate holds the states before each row: the one behind the last row is not among them."""
    g = torch.Generator().manual_seed(rows)
    D, at = 70, 11
    x, dt, dy, z = (randn(g, rows, D) for _ in range(4))
    b, c = randn(g, rows, 1, N), randn(g, rows, 1, N)
    a = -(torch.rand(D, N, generator=g) + 0.1).cuda()
    dlast = randn(g, 1, D, N)

    def back():
        marks = ssam.ssam_scan_selective_marks(x, a)
        ssam.ssam_scan_selective(x, dt, a, b, c, gate=z, softplus=True, d_marks=marks)
        return ssam.ssam_scan_selective_backward(dy, x, dt, a, b, c, marks, gate=z, softplus=True, d_grad_final=dlast, state_grad=True)

    clean = back()
    x[-1, at] = INF
    got = back()
    assert torch.isfinite(clean.a).all() and torch.equal(got.a, clean.a)
    assert torch.equal(got.state, clean.state) and torch.equal(got.dt[:-1], clean.dt[:-1]) and torch.equal(got.x, clean.x)
    assert torch.equal(got.c[:-1], clean.c[:-1]) and not torch.isfinite(got.c[-1]).any()


STATES = [1, 2, 3, 4, 5, 7, 8, 9, 13, 16, 17, 20, 32, 33, 50, 64]      # those that fill the lanes' registers, and those that do not


class Positive:
    """A scan whose terms are all positive, so that infinities add up to infinities."""

    def __init__(self, rows, N, dtype, D=70):
        g = torch.Generator().manual_seed(N)
        pos = lambda *s: (torch.rand(s, generator=g) + 0.25).to(dtype).cuda()  # noqa: E731
        self.x, self.dt, self.dy, self.b, self.c = pos(rows, D), pos(rows, D) / 8, pos(rows, D), pos(rows, 1, N), pos(rows, 1, N)
        self.a = -(torch.rand(D, N, generator=g) * 0.5 + 0.1).cuda()

    def forward(self, **more):
        return ssam.ssam_scan_selective(self.x, self.dt, self.a, self.b, self.c, **more)

    def marked(self):
        marks = ssam.ssam_scan_selective_marks(self.x, self.a)
        self.forward(d_marks=marks)
        return marks

    def back(self, marks):
        return ssam.ssam_scan_selective_backward(self.dy, self.x, self.dt, self.a, self.b, self.c, marks, state_grad=True)


@pytest.mark.parametrize("N", STATES)
def test_an_infinite_input_is_an_infinite_output(N):
    for dtype, rows in zip(TYPES, (30, 20, 200)):
        for name in ("x", "dt"):
            print(dtype, name, flush=True)
            k = Positive(rows, N, dtype)
            clean, (t, at) = k.forward(), (7, 11)
            getattr(k, name)[t, at] = INF
            last = torch.empty(1, *k.a.shape, device="cuda")
            got = k.forward(d_final=last)
            reached = slice(t, rows) if rows < 150 else slice(t, 30)       # (a long sequence is cut; its states pass the join)
            assert (got[reached, at] == INF).all(), got[reached, at]
            if rows < 150:
                assert (last[0, at] == INF).all()
            got[t:, at] = clean[t:, at]
            assert torch.equal(got, clean)


@pytest.mark.parametrize("N", STATES)
def test_an_infinite_input_of_a_single_row(N):
    for dtype in TYPES:
        k = Positive(6, N, dtype)
        pool = torch.rand(6, *k.a.shape, device="cuda")
        k.x[2, 11] = INF
        got = ssam.ssam_scan_selective_step(k.x, k.dt, k.a, k.b, k.c, pool)
        assert got[2, 11] == INF and (pool[2, 11] == INF).all()
        got[2, 11], pool[2, 11] = 0, 0
        assert torch.isfinite(got).all() and torch.isfinite(pool).all()


@pytest.mark.parametrize("N", STATES)
def test_the_gates_gradient_without_a_skip(N):
    for dtype in TYPES:
        rows, t, at = 40, 21, 11
        k = Positive(rows, N, dtype)
        z = torch.ones_like(k.x)
        k.x[t, at] = INF
        marks = ssam.ssam_scan_selective_marks(k.x, k.a)
        out = k.forward(gate=z, d_marks=marks)
        got = ssam.ssam_scan_selective_backward(k.dy, k.x, k.dt, k.a, k.b, k.c, marks, gate=z)
        for v in (out, got.gate):
            assert (v[t:, at] == INF).all()
            v[t:, at] = 0
            assert torch.isfinite(v).all()


@pytest.mark.parametrize("N", STATES)
def test_an_infinite_gradient_and_an_infinite_state_on_the_way_back(N):
    for dtype in TYPES:
        print(dtype, flush=True)
        rows, t, at = 40, 21, 11
        k = Positive(rows, N, dtype)
        marks = k.marked()
        clean = k.back(marks)
        there = k.dy[t, at].item()
        k.dy[t, at] = INF
        got = k.back(marks)
        assert (got.x[:t + 1, at] == INF).all() and (got.state[0, at] == INF).all()
        got.x[:t + 1, at], got.state[0, at] = clean.x[:t + 1, at], clean.state[0, at]
        assert torch.equal(got.x, clean.x) and torch.equal(got.state, clean.state)
        k.dy[t, at] = there
        k.x[t, at] = INF                   # an infinite state from row t on: the rows behind it lose their time steps' gradients
        got = k.back(k.marked())
        assert (got.dt[t + 1:, at] == -INF).all(), got.dt[t + 1:, at]
        got.dt[t:, at] = clean.dt[t:, at]
        assert torch.equal(got.dt, clean.dt) and torch.equal(got.x, clean.x)
        assert (got.c[t:] == INF).all() and torch.equal(got.c[:t], clean.c[:t])


@pytest.mark.parametrize("rate", [INF, 3e38, -INF, -3e38])
def test_an_infinite_rate_passes_the_end_of_its_sequence(rate):
    """A state behind the last row is that of the last row, whatever its rate."""
    for rows in (5, 16, 33):
        k = Positive(rows, 16, torch.float32)
        h, last = torch.ones(1, *k.a.shape, device="cuda"), torch.empty(1, *k.a.shape, device="cuda")
        k.forward(d_state=h, d_final=last)
        clean = last.clone()
        k.a[11, 3] = rate
        k.forward(d_state=h, d_final=last)
        want = INF if rate > 0 else (k.dt[-1, 11] * k.x[-1, 11] * k.b[-1, 0, 3]).item()
        assert last[0, 11, 3].item() == want
        last[0, 11, 3] = clean[0, 11, 3]
        assert torch.equal(last, clean)


@pytest.mark.parametrize("N", [4, 8, 13, 16, 32, 64])
def test_an_infinite_state_passes_pieces(N):
    """Each row's decay is above zero, a piece's is not: an infinite state, or gradient, times it stays infinite all the same."""
    rows, at = 300, 11
    k = Positive(rows, N, torch.float32)
    k.a = -30 * torch.ones_like(k.a)
    k.dt = k.dt.clamp(min=0.12)
    assert ssam.ssam_scan_selective_workspace_bytes(k.x, k.a) > 0         # it is cut
    assert (k.dt.max() * 30 < 80) and (k.dt[:32].sum(0) * 30 > 110).all()
    there = k.x[7, at].item()
    k.x[7, at] = INF
    last = torch.empty(1, *k.a.shape, device="cuda")
    out = k.forward(d_final=last)
    assert (out[7:, at] == INF).all() and (last[0, at] == INF).all()
    out[7:, at], last[0, at] = 0, 0
    assert torch.isfinite(out).all() and torch.isfinite(last).all()
    k.x[7, at] = there
    k.dy[290, at] = INF
    got = k.back(k.marked())
    assert (got.x[:291, at] == INF).all() and (got.state[0, at] == INF).all()
    got.x[:291, at], got.state[0, at] = 0, 0
    assert torch.isfinite(got.x).all() and torch.isfinite(got.state).all()


@pytest.mark.parametrize("D,N", [(70, 16), (6, 16), (70, 4), (130, 8), (33, 32), (1, 64), (64, 16), (128, 5)])
def test_an_infinity_of_b_or_c_reaches_its_own_sums(D, N):
    """The gradients of b and c are sums over channels: those that a tile has room for but the call does not have are not among them."""
    for dtype, rows in zip(TYPES, (40, 20, 150)):
        print(dtype, flush=True)
        k = Positive(rows, N, dtype, D)
        t, n = 17, N - 1
        clean = k.back(k.marked())
        there = k.b[t, 0, n].item()
        k.b[t, 0, n] = INF                  # an infinite state of every channel from row t on
        got = k.back(k.marked())
        assert (got.c[t:, 0, n] == INF).all()
        got.c[t:, 0, n] = clean.c[t:, 0, n]
        assert torch.equal(got.c, clean.c) and torch.equal(got.b, clean.b)
        k.b[t, 0, n] = there
        k.c[t, 0, n] = INF                  # an infinite gradient of every channel's state up to row t
        got = k.back(k.marked())
        assert (got.b[:t + 1, 0, n] == INF).all()
        got.b[:t + 1, 0, n] = clean.b[:t + 1, 0, n]
        assert torch.equal(got.b, clean.b) and torch.equal(got.c, clean.c)
