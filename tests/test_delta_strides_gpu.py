"""The scan with a matrix per head where q, k, v and the results' gradient each lie in a buffer of their own width, in rows and in heads: the same
bits as with all of them dense.  What lies between the rows is NaN, and so is what lies behind the last one."""
import pytest

from test_delta_gpu import spans_of
from test_sequence_gpu import TYPES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402

# extra channels of a row: of q, k, v, dout
APART = {"q far": (900, 0, 0, 0), "k far": (0, 901, 0, 0), "all": (7, 350, 64, 33), "v far": (0, 0, 500, 0), "q and v": (64, 3, 0, 77)}
ROWS = {"64": (64,), "128": (128,), "200": (200,), "2 x 64": (2, 64), "3 x 70": (3, 70)}


def beside(x, more):
    """x with `more` channels behind each row, NaN all of them, and a row's worth behind the last row."""
    flat = x.flatten(-2)
    lead, width = flat.shape[:-1], flat.shape[-1]
    rows = flat.reshape(-1, width)
    buf = torch.full((rows.shape[0] + 1, width + more), float("nan"), dtype=x.dtype, device=x.device)
    buf[:-1, :width] = rows
    return buf[:-1, :width].unflatten(0, lead).unflatten(-1, x.shape[-2:])


def inputs(lead, dt, Hk, H, K, V, seed):
    g = torch.Generator().manual_seed(seed)
    t = TYPES[dt]
    make = lambda *s: torch.randn(*lead, *s, generator=g)  # noqa: E731
    q, k = (torch.nn.functional.normalize(make(Hk, K), dim=-1).to(t).cuda() for _ in range(2))
    v, dout = (make(H, V).to(t).cuda() for _ in range(2))
    return q, k, v, (-torch.rand(*lead, H, generator=g) * 0.5).cuda(), torch.sigmoid(make(H)).cuda(), dout


def everything(q, k, v, g, beta, dout, state, dlast, unit, dev):
    marks = ssam.ssam_scan_delta_marks(k, v, **dev)
    final = torch.zeros_like(state)
    out = ssam.ssam_scan_delta(q, k, v, g, beta, unit=unit, d_state=state, d_final=final, d_marks=marks, **dev)
    grads = ssam.ssam_scan_delta_backward(dout, q, k, v, g, beta, marks, unit=unit, d_grad_final=dlast, state_grad=True, **dev)
    return {"out": out, "final": final, **grads._asdict()}


@pytest.mark.parametrize("apart", APART)
@pytest.mark.parametrize("rows", [*ROWS, "packed_long", "padded"])
@pytest.mark.parametrize("K", [1, 5, 8, 16, 20, 32, 33, 64, 100, 128, 200])
def test_the_rows_of_each_lie_where_it_says(K, rows, apart):
    lead, dev, spans = (ROWS[rows], {}, None) if rows in ROWS else spans_of(rows)
    Hk, H, V, S = 2, 4, 24, len(spans) if spans else lead[0] if len(lead) == 2 else 1
    g = torch.Generator().manual_seed(K)
    state, dlast = (torch.randn(S, H, K, V, generator=g).cuda() for _ in range(2))
    for dt in TYPES:
        q, k, v, gate, beta, dout = inputs(lead, dt, Hk, H, K, V, K)
        dense = everything(q, k, v, gate, beta, dout, state, dlast, True, dev)
        apart_ = [beside(x, more) for x, more in zip((q, k, v, dout), APART[apart])]
        assert all(torch.equal(a, b) for a, b in zip(apart_, (q, k, v, dout)))
        got = everything(*apart_[:3], gate, beta, apart_[3], state, dlast, True, dev)
        for n, x in dense.items():
            assert torch.isfinite(x).all() and torch.equal(got[n], x), (dt, n, int((got[n] != x).sum()))


@pytest.mark.parametrize("K", [8, 32, 64, 128])
def test_heads_before_rows(K):
    """Heads that lie further apart than rows, and as far for q as rows do for k."""
    lead, Hk, H, V = (130,), 3, 3, 40
    state, dlast = torch.zeros(1, H, K, V, device="cuda"), torch.ones(1, H, K, V, device="cuda")
    for dt in TYPES:
        q, k, v, gate, beta, dout = inputs(lead, dt, Hk, H, K, V, K)
        dense = everything(q, k, v, gate, beta, dout, state, dlast, True, {})
        turned = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
        for a, b in ((turned, lambda x: x), (lambda x: x, turned), (turned, turned)):
            got = everything(a(q), b(k), b(v), gate, beta, a(dout), state, dlast, True, {})
            for n, x in dense.items():
                assert torch.equal(got[n], x), (dt, n)


@pytest.mark.parametrize("apart", APART)
@pytest.mark.parametrize("K", [1, 20, 32, 128, 200])
def test_single_rows_lie_where_it_says(K, apart):
    for dt in TYPES:
        q, k, v, gate, beta, _ = inputs((70,), dt, 2, 4, K, 24, K)
        state = torch.randn(70, 4, K, 24, generator=torch.Generator().manual_seed(K)).cuda()
        other = state.clone()
        want = ssam.ssam_scan_delta_step(q, k, v, gate, beta, state, unit=True)
        q, k, v = (beside(x, more) for x, more in zip((q, k, v), APART[apart]))
        got = ssam.ssam_scan_delta_step(q, k, v, gate, beta, other, unit=True)
        assert torch.isfinite(want).all() and torch.equal(got, want) and torch.equal(other, state), dt
