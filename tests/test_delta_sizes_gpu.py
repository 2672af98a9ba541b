"""The scan with a matrix per head where values of very different sizes share 64 rows: a value of 32 bits is held with an error of 2^-22 of itself or
2^-35 of the largest that it is scaled with, whichever is more, and what that comes to in a result, worked out from the block's own matrices."""
import numpy as np
import pytest

import delta_reference as ref
import sequence_reference as seqref
from test_sequence_gpu import TYPES, f64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402

HELD = 2.0 ** -35
SIZES = [2.0 ** -8, 1e-5, 1e-7, 1e-9, 1e-12]


def two(n, at, K, V, size, small_first, seed):
    """n rows in fp32, from row `at` on, which forgets all before it, of another size: values and the result's gradient."""
    g = torch.Generator().manual_seed(seed)
    unit = lambda: torch.nn.functional.normalize(torch.randn(n, 1, K, generator=g), dim=-1)  # noqa: E731
    q, k, v, dout = unit(), unit(), torch.randn(n, 1, V, generator=g), torch.randn(n, 1, V, generator=g)
    lower = slice(0, at) if small_first else slice(at, n)
    v[lower] *= size
    dout[lower] *= size
    gate = -0.1 * torch.rand(n, 1, generator=g)
    gate[at] = -float("inf")
    beta = torch.sigmoid(torch.randn(n, 1, generator=g))
    return [x.cuda() for x in (q, k, v, gate, beta, dout)], lower


def matrices(q, k, gate, beta, scale):
    """(I + A diag(beta))^-1, (I + diag(beta) A)^-1 and scale (Q K^T o D) of one block and head."""
    n = len(q)
    G = np.cumsum(np.maximum(gate, -1000.0))
    lower = np.tril(np.ones((n, n), bool))
    D = np.where(lower, np.exp(np.where(lower, G[:, None] - G[None], 0.0)), 0.0)
    A = np.tril((k @ k.T) * D, -1)
    return np.linalg.inv(np.eye(n) + A * beta), np.linalg.inv(np.eye(n) + beta[:, None] * A), scale * (q @ k.T) * D


def within(what, got, want, bound, lower):
    """`bound` off beside what rounding may leave of a half's own size."""
    got = f64(got).reshape(want.shape)
    upper = np.ones(len(want), bool)
    upper[lower] = False
    for half in (lower, upper):
        off = np.abs(got - want)[half]
        own = 8 * ref.delta_noise(len(want)) * np.abs(want[half]).max(0)
        assert (off <= bound[half] + own).all(), (what, half, (off / (bound[half] + own)).max())


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("small_first", [False, True])
@pytest.mark.parametrize("K,V", [(64, 40), (20, 16), (128, 128), (200, 24)])
def test_rows_of_two_sizes(size, small_first, K, V):
    """The correction's solution T X, U = beta T X, out = P U; the gradient beta T'^T P^T dO with T' = (I + diag(beta) A)^-1, since beta T = T' beta.  Before each product its columns are held
    with that error of the largest of the 64 rows; the matrices are zero between the two halves, so that only a half's own rows add their errors."""
    n = 64
    (q, k, v, gate, beta, dout), lower = two(n, 40, K, V, size, small_first, K)
    marks = ssam.ssam_scan_delta_marks(k, v)
    out = ssam.ssam_scan_delta(q, k, v, gate, beta, d_marks=marks)
    dv = ssam.ssam_scan_delta_backward(dout, q, k, v, gate, beta, marks).v
    Q, Kk, X, dO = (f64(x)[:, 0] for x in (q, k, v, dout))
    b = f64(beta)[:, 0]
    T, Tb, P = matrices(Q, Kk, f64(gate)[:, 0], b, K ** -0.5)
    most = lambda a: np.abs(a).max(0)  # noqa: E731
    R = T @ X
    U = b[:, None] * R
    held = lambda M, x: HELD * np.abs(M).sum(1)[:, None] * most(x)  # noqa: E731    of M times x's columns
    within("out", out, P @ U, np.abs(P) @ (b[:, None] * held(T, X)) + held(P, U), lower)
    dU = P.T @ dO
    dY = Tb.T @ dU
    within("dv", dv, b[:, None] * dY, b[:, None] * (np.abs(Tb.T) @ held(P.T, dO) + held(Tb.T, dU)), lower)


@pytest.mark.parametrize("size", SIZES)
def test_rows_of_their_own_64_keep_their_digits(size):
    """The same rows apart: 64 rows of one size, then 64 of the other."""
    for small_first in (False, True):
        (q, k, v, gate, beta, dout), lower = two(128, 64, 64, 40, size, small_first, 3)
        out = ssam.ssam_scan_delta(q, k, v, gate, beta)
        want, _, _ = ref.delta(*(f64(x) for x in (q, k, v)), np.maximum(f64(gate), -1000.0), f64(beta), 64 ** -0.5, np.zeros((1, 64, 40)))
        within("out", out, want[:, 0], np.zeros((128, 40)), lower)


@pytest.mark.parametrize("power", [12, 20, 26, 30, 33, 40])
@pytest.mark.parametrize("dt", TYPES)
def test_elements_of_two_sizes_in_a_query(dt, power):
    """Nothing is written: out = scale S^T q, and where q's largest element is, the state is zero.  Elements of q beside that one: bf16 exactly to 2^-27 of it
    and 2^-34 of it off below; fp32 as above; fp16 exactly."""
    n, K, V = 70, 64, 32
    g = torch.Generator().manual_seed(power)
    q = torch.randn(n, 1, K, generator=g).clamp(-1, 1) * 2.0 ** -power
    q[:, :, 5] = 1.0
    q = q.to(TYPES[dt]).cuda()
    k, v = torch.zeros_like(q), torch.zeros(n, 1, V, dtype=TYPES[dt], device="cuda")
    state = torch.randn(1, 1, K, V, generator=g).cuda()
    state[:, :, 5] = 0
    # (the result's own rounding out of the way: fp16 reaches down to 2^-24, so everything is brought up)
    out = ssam.ssam_scan_delta(q, k, v, None, torch.zeros(n, 1, device="cuda"), scale=2.0 ** power, d_state=state)
    S, Q = f64(state)[0, 0], f64(q)[:, 0]
    want = 2.0 ** power * Q @ S
    element = {"float32": np.maximum(2.0 ** -22 * np.abs(Q), HELD), "bfloat16": np.where(np.abs(Q) < 2.0 ** -27, 2.0 ** -34, 0.0), "float16": np.zeros_like(Q)}[dt]
    element[:, 5] = 0
    # the state's elements in pairs, products and sums of at most 64 in fp32, the result's type
    size = np.abs(Q) @ np.abs(S) * 2.0 ** power      # (none of q's largest element: there the state is zero)
    Q[:, 5] = 0
    tol = 2.0 ** power * element @ np.abs(S) + size * (2.0 ** -21 + 70 * seqref.U) + 2.0 ** (power - 35) * np.abs(Q).sum(1)[:, None] * np.abs(S).max(0)
    tol = tol + seqref.HALF_STEP[dt] * (np.abs(want) + tol) + seqref.TINY[dt]
    off = np.abs(f64(out)[:, 0] - want)
    assert (off <= tol).all(), (off / tol).max()
