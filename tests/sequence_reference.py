"""The sequence operators' definitions in 64 bits, one sequence at a time, and how far fp32 arithmetic may be from them.

u = 2^-24 below is fp32's rounding.  Every bound is a multiple of u times the same sum with every term's magnitude in its
place (`mag`), plus half a step of the result's type.
"""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 1e-37, "float16": 2.0 ** -25, "bfloat16": 1e-37}     # half the least subnormal (fp16), results below fp32's normals


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def softplus(x):
    return np.logaddexp(x, 0.0)


def spans(rows, starts=None, lengths=None, sequences=None):
    """[(sequence, first flat row, rows)] of a call's sequences."""
    if starts is not None:
        return [(i, int(b), int(e) - int(b)) for i, (b, e) in enumerate(zip(starts, starts[1:]))]
    if sequences is None:
        return [(0, 0, rows)]
    return [(i, i * rows, rows if lengths is None else int(lengths[i])) for i in range(sequences)]


# ---- filter ------------------------------------------------------------------------------------------------------------

def conv1d(x, w, bias, silu, state):
    """x [n, D], w [D, W], state [W - 1, D] -> y, final state, and |error| <= of y before it is rounded to its type.

    p: W products and W additions, each within u of its size: (W + 1) u mag.  silu(p): its slope is below 1.1; exp, 1 + e, the
    reciprocal and the product are 1 u, u, 2 u and u off, and the rounded exponent adds 2 |p| u: (8 + 2 |p|) u |y|."""
    n, (D, W) = x.shape[0], w.shape
    rows = np.concatenate([state, x])
    p, mag = np.zeros((n, D)) + bias, np.zeros((n, D)) + np.abs(bias)
    for j in range(W):
        p += w[:, j] * rows[j:j + n]
        mag += np.abs(w[:, j] * rows[j:j + n])
    bound = (W + 1) * U * mag
    y = p
    if silu:
        y = p * sigmoid(p)
        bound = 1.1 * bound + (8 + 2 * np.abs(p)) * U * np.abs(y)
    return y, rows[n:], bound


def conv1d_back(dy, x, w, bias, silu, state, dfinal):
    """Gradients of x, w, bias, state and their magnitudes."""
    n, (D, W) = x.shape[0], w.shape
    rows = np.concatenate([state, x])
    q, qm = dy.copy(), np.abs(dy)
    if silu:
        p, mag = np.zeros((n, D)) + bias, np.zeros((n, D)) + np.abs(bias)
        for j in range(W):
            p += w[:, j] * rows[j:j + n]
            mag += np.abs(w[:, j] * rows[j:j + n])
        s = sigmoid(p)
        q = dy * s * (1 + p * (1 - s))
        # the slope's own slope is below 0.5: an error of p counts half as much; 1 and |p| (1 - s) are its terms
        qm = np.abs(dy) * (1.1 + mag + np.abs(p))
    drows, dm = np.zeros_like(rows), np.zeros_like(rows)
    dw, wm = np.zeros((D, W)), np.zeros((D, W))
    for j in range(W):
        dw[:, j] = (q * rows[j:j + n]).sum(0)
        wm[:, j] = (qm * np.abs(rows[j:j + n])).sum(0)
        drows[j:j + n] += q * w[:, j]
        dm[j:j + n] += qm * np.abs(w[:, j])
    if dfinal is not None:
        drows[n:] += dfinal
        dm[n:] += np.abs(dfinal)
    return (drows[W - 1:], dw, q.sum(0), drows[:W - 1]), (dm[W - 1:], wm, qm.sum(0), dm[:W - 1])


# ---- scan --------------------------------------------------------------------------------------------------------------

def scan_states(u, d, a, b, h0):
    """u, d [n, D], a [D, N], b [n, D, N] -> h [n + 1, D, N] with h[0] = h0."""
    h = np.empty((u.shape[0] + 1, *a.shape))
    h[0] = h0
    for t in range(u.shape[0]):
        h[t + 1] = np.exp(d[t][:, None] * a) * h[t] + (d[t] * u[t])[:, None] * b[t]
    return h


def _factors(z):
    if z is None:
        return 1.0, 0.0
    s = sigmoid(z)
    return z * s, s * (1 + z * (1 - s))


def scan(u, d, a, b, c, skip, z, h0):
    """Outputs and last state."""
    h = scan_states(u, d, a, b, h0)
    y = (h[1:] * c).sum(-1) + skip * u
    return y * _factors(z)[0], h[-1]


def scan_back(dout, u, d, a, b, c, skip, z, h0, dlast, size=False):
    """Gradients of u, d, a, b, c (per channel), skip, z, h0.  size: with every term's magnitude instead."""
    s1, s2 = _factors(z)
    rates = a
    if size:
        dout, u, b, c, skip, h0, dlast, rates = (np.abs(v) for v in (dout, u, b, c, skip, h0, dlast, a))
        s1, s2 = np.abs(s1), (0.0 if z is None else 1.1 + np.abs(z) * sigmoid(z) * (1 - sigmoid(z)))
    n = u.shape[0]
    h = scan_states(u, d, a, b, h0)
    y = (h[1:] * c).sum(-1) + skip * u
    dz = dout * y * s2
    dy = dout * s1
    g = np.empty((n, *a.shape))
    carry = dlast
    for t in reversed(range(n)):
        g[t] = c[t] * dy[t][:, None] + carry
        carry = np.exp(d[t][:, None] * a) * g[t]
    x = np.exp(d[..., None] * a) * h[:-1]
    q = g * x
    gb = (g * b).sum(-1)
    return {"x": skip * dy + d * gb, "d": (rates * q).sum(-1) + u * gb, "a": (d[..., None] * q).sum(0), "b": g * (d * u)[..., None],
            "c": h[1:] * dy[..., None], "skip": (dy * u).sum(0), "gate": dz, "state": carry}


def scan_kappa(n):
    """Relative error of one term of a scan of n rows.  A decay is exp2(d a2): the hardware's exp2 is 2 u off; a2 is rounded twice, d is
    within 8 u (below) and their product once, so the decay is off by another 11 |d a| u, and a chain of decays by 11 u times what it
    decayed by, X: e^-X X <= 30 e^-30 past X = 30, below u of the chain's first term.  A sequence of more than 128 rows may be cut into
    pieces of 64 rows at most (at these sizes), whose time steps are added up: 64 additions, 64 u X more.  Every row adds the rounding of
    a product and a sum and exp2's own: n (2 + 1.4) u; the gate, the products before and behind: 24 u.
    A softplus, log1p(e) with e = exp2(-log2(e) |x|) where x < 0: log2(e) and its product with x are 1.3 u off, so e is off by 1.3 |x| u
    and exp2's 2 u, the logarithm adds 4: (6 + 1.3 |x|) u.  That is 8 u to x = -1.5; below, d (1.3 |x| - 2) is at most 0.1, so that a row
    moves a decay by 0.1 |a| u more, |a| <= 3.1: n (2 + 1.4 + 0.3) u in all, n 4 u."""
    return (4 * n + 30 * 11 + (30 * 64 if n > 64 else 0) + 24) * U


def allowed(want, mag, kappa, dtype):
    return HALF_STEP[dtype] * np.abs(want) * (1 + kappa) + kappa * mag + TINY[dtype]
