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
