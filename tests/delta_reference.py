"""The gated delta rule and the root-mean-square norm in 64 bits, one sequence at a time, row after row, and how far the kernels may be from
them.  u = 2^-24 is fp32's rounding."""
import numpy as np

from sequence_reference import HALF_STEP, TINY, U, sigmoid

UNIT_EPS = 1e-6


def unit(x):
    return x / np.sqrt((x * x).sum(-1, keepdims=True) + UNIT_EPS)


def through_unit(x, d):
    """Gradient of x for d, that of unit(x)."""
    size = np.sqrt((x * x).sum(-1, keepdims=True) + UNIT_EPS)
    return (d - x / size * (x / size * d).sum(-1, keepdims=True)) / size


def delta(q, k, v, g, beta, scale, h0):
    """q, k [n, H, K], v [n, H, V], g, beta [n, H], h0 [H, K, V] -> out, last state, and what the way back needs of every row."""
    h, out, kept = h0.copy(), np.zeros_like(v), []
    for t in range(q.shape[0]):
        s = np.exp(g[t])[:, None, None] * h
        miss = v[t] - (s * k[t][:, :, None]).sum(1)
        h = s + k[t][:, :, None] * (beta[t][:, None] * miss)[:, None]
        out[t] = scale * (h * q[t][:, :, None]).sum(1)
        kept.append((s, miss, h))
    return out, h, kept


def delta_back(dout, q, k, v, g, beta, scale, kept, dlast):
    """Gradients of q, k, v, g, beta, h0, and the sizes of what g's, beta's, k's and v's are made of: products of the lengths of what is multiplied."""
    d = dlast.copy()
    r = {n: np.zeros_like(a) for n, a in (("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta), ("size", g), ("bsize", g), ("ksize", k), ("vsize", v))}
    length = lambda a, axis: np.sqrt((a * a).sum(axis))  # noqa: E731
    for t in reversed(range(q.shape[0])):
        s, miss, h = kept[t]
        r["q"][t] = scale * (h * dout[t][:, None]).sum(-1)
        d = d + scale * q[t][:, :, None] * dout[t][:, None]
        du = (d * k[t][:, :, None]).sum(1)
        r["beta"][t] = (du * miss).sum(-1)
        dmiss = beta[t][:, None] * du
        r["k"][t] = (d * (beta[t][:, None] * miss)[:, None]).sum(-1) - (s * dmiss[:, None]).sum(-1)
        r["v"][t] = dmiss
        r["vsize"][t] = beta[t][:, None] * length(d, 1) * length(k[t], -1)[:, None]
        r["bsize"][t] = length(length(d, 1) * length(k[t], -1)[:, None], -1) * length(miss, -1)
        r["ksize"][t] = length(d, -1) * length(beta[t][:, None] * miss, -1)[:, None] + length(s, -1) * length(dmiss, -1)[:, None]
        d = d - k[t][:, :, None] * dmiss[:, None]
        r["g"][t] = (d * s).sum((-1, -2))
        r["size"][t] = np.sqrt((d * d).sum((-1, -2)) * (s * s).sum((-1, -2)))
        d = np.exp(g[t])[:, None, None] * d
    r["state"] = d
    return r


def delta_noise(rows):
    """Relative size, as a root mean square, of what rounding may leave on outputs of a sequence of so many rows whose keys have unit length.

    A row's correction I - beta k k^T has norm at most 1 for beta in [0, 1], and so has a decay: errors of a state are never larger a row
    later, they add up.  What enters in a block of 64 rows: some twelve values in line (the state, X, R, U, its decayed form, O, the two
    matrices; on the way back as many) are held as pairs of fp16, truncated at 2^-21 of their size, or are sums of up to 256 products in
    fp32, whose roundings, independent, leave sqrt(256) u = 2^-20.  In squares, sqrt(12) 2^-20 = 2^-18.2 a block; a state's blocks add in
    squares too."""
    return 2.0 ** -18 * np.sqrt(1.0 + np.ceil(rows / 64.0))


def norm(x, w, gate, groups, eps):
    """[n, D] -> out and the relative error that its fp32 arithmetic may have.

    A lane adds at most 64 squares, then at most ten partial sums: 75 u of the mean, half of that of the root; the root, the reciprocal
    and three products 6 u: below 48 u.  The gate: exp, 1 + e, a reciprocal, two products, and 2 |z| u of the exponent's rounding."""
    n, D = x.shape
    y = x.reshape(n, groups, -1)
    y = (y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * w).reshape(n, D)
    kappa = np.full_like(y, 48 * U)
    if gate is not None:
        y = y * gate * sigmoid(gate)
        kappa = kappa + (10 + 2 * np.abs(gate)) * U
    return y, kappa


def norm_back(dout, x, w, gate, dsum, groups, eps):
    """Gradients of x, w, gate, the sizes of their terms, and the relative error of one term as above: 150 u (the means twice, products)
    and the gate's."""
    n, D = x.shape
    parts = lambda a: a.reshape(n, groups, -1)  # noqa: E731
    X = parts(x)
    r = 1.0 / np.sqrt((X * X).mean(-1, keepdims=True) + eps)
    d, dgate, gsize, extra = parts(dout), None, None, 0.0
    if gate is not None:
        z, s = parts(gate), sigmoid(parts(gate))
        y = X * r * w
        dgate = (d * y * s * (1 + z * (1 - s))).reshape(n, D)
        gsize = (np.abs(d * y) * (1.1 + np.abs(z))).reshape(n, D)
        d = d * z * s
        extra = (12 + 3 * np.abs(gate).max()) * U
    a = d * w * r
    dx = a - X * r * r * (a * X).mean(-1, keepdims=True)
    xsize = np.abs(a) + np.abs(X) * r * r * np.abs(a * X).mean(-1, keepdims=True)
    dw, wsize = (d * X * r).sum((0, 1)), np.abs(d * X * r).sum((0, 1))
    dx, xsize = dx.reshape(n, D), xsize.reshape(n, D)
    if dsum is not None:
        dx, xsize = dx + dsum, xsize + np.abs(dsum)
    return dx, dw, dgate, xsize, wsize, gsize, 150 * U + extra


def rounded(want, size, kappa, dtype):
    """Tolerance of a value that is `kappa` of `size` off before it is rounded to its type."""
    return HALF_STEP[dtype] * np.abs(want) * (1 + 8 * U) + kappa * size * (1 + HALF_STEP[dtype]) + TINY[dtype]
