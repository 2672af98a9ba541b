"""Causal filter and selective scan along time, their gradients and single-row forms, against their definitions in 64 bits."""
import numpy as np
import pytest

import sequence_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
NAME = {v: k for k, v in TYPES.items()}
SENTINEL = 7.0


def f64(t):
    return t.detach().double().cpu().numpy()


def randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def check(what, got, want, tol):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), f"{what}: not finite"
    bad = np.abs(got - want) > tol
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / tol, 0)), got.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} values off, worst at {i}: {got[i]!r} for {want[i]!r}, allowed {tol[i]:.3e}")


def wide(g, lead, channels, dtype, form):
    """Rows of `channels`: contiguous, or the middle columns of a wider buffer with an odd stride."""
    if form == "dense":
        return randn(g, *lead, channels, dtype=dtype)
    return randn(g, *lead, channels + 5, dtype=dtype)[..., 3:3 + channels]


# (leading extents, starts, lengths): one sequence; a batch; a padded batch with an empty row; packed ones, some of them empty, with
# rows before the first and behind the last that belong to none
LAYOUTS = {
    "one": ((37,), None, None), "single_row": ((1,), None, None), "batch": ((3, 21), None, None), "padded": ((4, 19), None, [19, 0, 1, 7]),
    "packed": ((90,), [2, 2, 19, 20, 20, 51, 88], None), "long": ((300,), None, None), "packed_long": ((333,), [0, 1, 200, 200, 330], None),
    # more pieces than the join takes at a time
    "pieces": ((2300,), None, None), "batch_pieces": ((2, 1200), None, None), "padded_pieces": ((3, 1300), None, [1300, 129, 0]),
    "packed_pieces": ((2200,), [3, 1500, 1500, 1530, 2190], None),
    # more packed sequences than a wave has lanes, and than two rounds of 64 tell apart; every third or fourth empty
    "crowd": ((700,), [5 + s * 4 + s % 3 * 2 for s in range(131)], None), "swarm": ((5300,), [s - s % 4 // 3 for s in range(5201)], None),
}


def layout(name):
    lead, starts, lengths = LAYOUTS[name]
    dev = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    spans = ref.spans(lead[-1], starts, lengths, lead[0] if len(lead) == 2 else None)
    return lead, dict(starts=dev(starts), lengths=dev(lengths)), spans


def flat(t, lead):
    return f64(t).reshape(int(np.prod(lead)), *t.shape[len(lead):])


# ---- filter ------------------------------------------------------------------------------------------------------------
CONV = [(lay, dt, W, D, silu, bias, state, form)
        for lay, dt, W, D, silu, bias, state, form in [
            ("one", "float32", 4, 64, True, True, True, "dense"), ("one", "bfloat16", 4, 513, True, True, True, "wide"),
            ("single_row", "float16", 4, 7, False, True, True, "dense"), ("single_row", "float32", 1, 1, True, False, False, "dense"),
            ("batch", "bfloat16", 3, 1030, False, True, False, "wide"), ("batch", "float16", 8, 65, True, False, True, "dense"),
            ("padded", "float32", 5, 33, True, True, True, "wide"), ("padded", "bfloat16", 4, 512, True, True, True, "dense"),
            ("packed", "float32", 4, 257, True, True, True, "dense"), ("packed", "float16", 6, 8, False, True, True, "wide"),
            ("packed", "bfloat16", 2, 100, True, True, False, "wide"), ("long", "bfloat16", 7, 40, True, True, True, "dense"),
            ("packed_long", "float32", 4, 20, False, False, True, "dense"),
            ("crowd", "bfloat16", 4, 130, True, True, True, "wide"), ("swarm", "float32", 3, 9, True, True, True, "dense")]]


def conv_case(lay, dt, W, D, bias, state, form, params=None):
    g = torch.Generator().manual_seed(hash((W, D)) % 1000)
    lead, seq, spans = layout(lay)
    dtype = TYPES[dt]
    x = wide(g, lead, D, dtype, form)
    w = randn(g, D, W, dtype=params or dtype)
    b = randn(g, D, dtype=params or dtype) if bias else None
    h = randn(g, len(spans), W - 1, D, dtype=dtype) if state else None
    return g, lead, seq, spans, x, w, b, h


def conv_state(h, i, W, D):
    return np.zeros((W - 1, D)) if h is None else f64(h)[i]


@pytest.mark.parametrize("lay,dt,W,D,silu,bias,state,form", CONV)
def test_conv1d(lay, dt, W, D, silu, bias, state, form):
    print(lay, dt, W, D, flush=True)
    params = torch.float32 if D % 2 else None
    g, lead, seq, spans, x, w, b, h = conv_case(lay, dt, W, D, bias, state, form, params)
    out = torch.full((*lead, D), SENTINEL, dtype=x.dtype, device="cuda")
    final = torch.full((len(spans), W - 1, D), SENTINEL, dtype=x.dtype, device="cuda")
    res = ssam.ssam_conv1d(x, w, bias=b, silu=silu, d_state=h, d_final=final, d_out=out, **seq)
    assert res is out
    want = np.full((int(np.prod(lead)), D), SENTINEL)
    tol = np.zeros_like(want)
    xs = flat(x, lead)
    for i, lo, n in spans:
        y, last, bound = ref.conv1d(xs[lo:lo + n], f64(w), 0.0 if b is None else f64(b), silu, conv_state(h, i, W, D))
        want[lo:lo + n] = y
        tol[lo:lo + n] = ref.HALF_STEP[dt] * (np.abs(y) + bound) + bound + ref.TINY[dt]
        assert np.array_equal(f64(final)[i], last), f"state after sequence {i}"
    check("out", out.reshape(want.shape), want, tol)      # rows of no sequence: exactly as they were
    # a new result holds zeros there, and the state may be handed on in place
    fresh = ssam.ssam_conv1d(x, w, bias=b, silu=silu, d_state=h, **seq).reshape(want.shape)
    outside = tol[:, 0] == 0
    assert torch.equal(fresh[torch.from_numpy(~outside).cuda()], out.reshape(want.shape)[torch.from_numpy(~outside).cuda()])
    assert not fresh[torch.from_numpy(outside).cuda()].any()
    if h is not None:
        both = h.clone()
        ssam.ssam_conv1d(x, w, bias=b, silu=silu, d_state=both, d_final=both, d_out=out, **seq)
        assert torch.equal(both, final)


@pytest.mark.parametrize("lay,dt,W,D,silu,bias,state,form", CONV)
def test_conv1d_backward(lay, dt, W, D, silu, bias, state, form):
    print(lay, dt, W, D, flush=True)
    params = torch.float32 if D % 2 else None
    g, lead, seq, spans, x, w, b, h = conv_case(lay, dt, W, D, bias, state, form, params)
    dy = wide(g, lead, D, x.dtype, form)
    dfinal = randn(g, len(spans), W - 1, D, dtype=x.dtype) if state else None
    got = ssam.ssam_conv1d_backward(dy, x, w, bias=b, silu=silu, d_state=h, d_grad_final=dfinal, state_grad=True, **seq)
    rows = int(np.prod(lead))
    dx, dxm = np.zeros((rows, D)), np.zeros((rows, D))
    sums = [np.zeros((D, W)), np.zeros((D, W)), np.zeros(D), np.zeros(D)]
    ds, dsm = np.zeros((len(spans), W - 1, D)), np.zeros((len(spans), W - 1, D))
    for i, lo, n in spans:
        val, mag = ref.conv1d_back(flat(dy, lead)[lo:lo + n], flat(x, lead)[lo:lo + n], f64(w), 0.0 if b is None else f64(b), silu,
                                   conv_state(h, i, W, D), None if dfinal is None else f64(dfinal)[i])
        dx[lo:lo + n], dxm[lo:lo + n], ds[i], dsm[i] = val[0], mag[0], val[3], mag[3]
        sums[0] += val[1]
        sums[1] += mag[1]
        sums[2] += val[2]
        sums[3] += mag[2]
    # q: the filter again and a sigmoid, (W + 12) u of its terms; W products and sums; sums of rows: one addition a row
    kappa = (2 * W + 14) * ref.U
    total = kappa + rows * ref.U
    pdt = NAME[w.dtype]
    outside = np.ones(rows, bool)
    for _, lo, n in spans:
        outside[lo:lo + n] = False
    tol = ref.allowed(dx, dxm, kappa, dt)
    tol[outside] = 0
    check("x", got.x.reshape(rows, D), dx, tol)
    check("weight", got.weight, sums[0], ref.allowed(sums[0], sums[1], total, pdt))
    if b is not None:
        check("bias", got.bias, sums[2], ref.allowed(sums[2], sums[3], total, pdt))
    check("state", got.state, ds, ref.allowed(ds, dsm, kappa, dt))
    again = ssam.ssam_conv1d_backward(dy, x, w, bias=b, silu=silu, d_state=h, d_grad_final=dfinal, state_grad=True, **seq)
    assert all(torch.equal(p, q) for p, q in zip(got, again) if p is not None), "the same call twice"


@pytest.mark.parametrize("dt,W,D,silu", [("bfloat16", 4, 520, True), ("float32", 3, 5, False), ("float16", 8, 77, True), ("bfloat16", 1, 64, True),
                                         ("bfloat16", 4, 525, True), ("float16", 2, 515, False), ("float32", 4, 259, True)])
def test_conv1d_step(dt, W, D, silu):
    g = torch.Generator().manual_seed(5)
    dtype = TYPES[dt]
    R, pool = 7, 9
    w, b = randn(g, D, W, dtype=dtype), randn(g, D, dtype=dtype)
    x = randn(g, R, D + 3, dtype=dtype)[:, 1:1 + D]
    state = randn(g, pool, 2, W - 1, D, dtype=dtype)[:, 1]               # one of two layers' slots
    before = state.clone()
    # slot 3 three times, one passed over, one behind the pool
    slots = [3, 0, -1, 3, 8, 3, 9]
    out = torch.full((R, D), SENTINEL, dtype=dtype, device="cuda")
    ssam.ssam_conv1d_step(x, w, state, bias=b, silu=silu, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), d_out=out)
    want, tol, after = np.full((R, D), SENTINEL), np.zeros((R, D)), f64(before)
    for r, s in enumerate(slots):
        if 0 <= s < pool:
            y, after[s], bound = ref.conv1d(f64(x)[r:r + 1], f64(w), f64(b), silu, after[s])
            want[r], tol[r] = y[0], (ref.HALF_STEP[dt] * (np.abs(y) + bound) + bound + ref.TINY[dt])[0]
    check("out", out, want, tol)
    assert np.array_equal(f64(state), after)
    # without slots row r has slot r
    plain = ssam.ssam_conv1d_step(x, w, before.clone(), bias=b, silu=silu)
    y0 = np.concatenate([ref.conv1d(f64(x)[r:r + 1], f64(w), f64(b), silu, f64(before)[r])[0] for r in range(R)])
    assert np.abs(f64(plain) - y0).max() <= 4 * ref.HALF_STEP[dt] * (1 + np.abs(y0).max()) * (W + 8)


# ---- scan --------------------------------------------------------------------------------------------------------------
SCAN = [  # layout, type, channels, states, groups, softplus, gate, skip, state, form
    ("one", "float32", 64, 16, 1, True, True, True, True, "dense"), ("one", "bfloat16", 67, 16, 1, True, True, True, True, "wide"),
    ("single_row", "float32", 1, 1, 1, False, False, False, False, "dense"), ("single_row", "bfloat16", 130, 16, 1, True, True, True, True, "dense"),
    ("batch", "float16", 96, 8, 2, True, True, True, True, "wide"), ("batch", "float32", 300, 3, 1, True, False, True, False, "dense"),
    ("padded", "float32", 24, 13, 4, True, True, True, True, "wide"), ("padded", "bfloat16", 128, 16, 1, True, False, True, True, "dense"),
    ("packed", "float32", 66, 5, 6, False, True, False, True, "dense"), ("packed", "bfloat16", 200, 16, 1, True, True, True, True, "wide"),
    ("packed", "float16", 35, 33, 1, True, True, True, False, "dense"), ("one", "float32", 18, 64, 2, True, True, True, True, "dense"),
    ("one", "bfloat16", 70, 20, 1, True, True, True, True, "wide"), ("one", "float16", 260, 4, 1, True, True, True, True, "wide"),
    ("long", "float32", 64, 16, 1, True, True, True, True, "dense"), ("long", "bfloat16", 20, 32, 1, True, True, True, True, "wide"),
    ("packed_long", "float32", 70, 8, 1, True, True, True, True, "dense"), ("packed_long", "bfloat16", 12, 50, 2, True, False, True, True, "wide"),
    ("pieces", "float32", 20, 4, 1, True, True, True, True, "dense"), ("batch_pieces", "float16", 136, 8, 2, True, False, True, True, "wide"),
    ("padded_pieces", "bfloat16", 70, 16, 1, True, True, False, True, "dense"), ("packed_pieces", "float32", 66, 20, 2, True, True, True, True, "wide"),
    ("crowd", "bfloat16", 65, 16, 1, True, True, True, True, "wide"), ("swarm", "float32", 6, 3, 1, True, False, True, True, "dense"),
    ("packed_pieces", "bfloat16", 9, 33, 3, False, True, True, False, "dense")]


class ScanCase:
    def __init__(self, lay, dt, D, N, G, softplus, gate, skip, state, form):
        g = self.g = torch.Generator().manual_seed(100 * N + D)
        self.lead, self.seq, self.spans = layout(lay)
        dtype = self.dtype = TYPES[dt]
        self.dt, self.D, self.N, self.G, self.softplus, self.form = dt, D, N, G, softplus, form
        self.x, self.raw = wide(g, self.lead, D, dtype, form), wide(g, self.lead, D, dtype, form)
        self.bias = randn(g, D) - 2 if softplus else None
        if not softplus:
            self.raw = self.raw.abs() * 0.1
        self.a = -(torch.rand(D, N, generator=g) * 3 + 0.05).cuda()
        both = wide(g, self.lead, 2 * G * N, dtype, form)
        self.b, self.c = both[..., :G * N].unflatten(-1, (G, N)), both[..., G * N:].unflatten(-1, (G, N))
        self.skip = randn(g, D) if skip else None
        self.z = wide(g, self.lead, D, dtype, form) if gate else None
        self.h0 = randn(g, len(self.spans), D, N) if state else None
        self.args = dict(skip=self.skip, gate=self.z, dt_bias=self.bias, softplus=softplus, **self.seq)
        self.rows = int(np.prod(self.lead))
        self.longest = max(n for _, _, n in self.spans)
        self.inside = np.zeros(self.rows, bool)
        for _, lo, n in self.spans:
            self.inside[lo:lo + n] = True

    def inputs(self, i, lo, n):
        f = lambda t: flat(t, self.lead)[lo:lo + n]  # noqa: E731
        raw = f(self.raw) + (0.0 if self.bias is None else f64(self.bias))
        d = ref.softplus(raw) if self.softplus else raw
        each = self.D // self.G
        b, c = np.repeat(f(self.b), each, 1), np.repeat(f(self.c), each, 1)
        skip = np.zeros(self.D) if self.skip is None else f64(self.skip)
        h0 = np.zeros((self.D, self.N)) if self.h0 is None else f64(self.h0)[i]
        return f(self.x), d, f64(self.a), b, c, skip, None if self.z is None else f(self.z), h0, raw

    def forward(self):
        """Outputs, last states and what both may be off by."""
        out, tol = np.full((self.rows, self.D), SENTINEL), np.zeros((self.rows, self.D))
        last, ltol = np.zeros((len(self.spans), self.D, self.N)), np.zeros((len(self.spans), self.D, self.N))
        kappa = ref.scan_kappa(self.longest)
        for i, lo, n in self.spans:
            u, d, a, b, c, skip, z, h0, _ = self.inputs(i, lo, n)
            out[lo:lo + n], last[i] = ref.scan(u, d, a, b, c, skip, z, h0)
            # magnitudes: every factor's; the gate's error is relative (8 u) and |z| u of its exponent, within |z| + 1 of the value
            mag, lmag = ref.scan(np.abs(u), d, a, np.abs(b), np.abs(c), np.abs(skip), None, np.abs(h0))
            if z is not None:
                mag *= np.abs(z * ref.sigmoid(z)) * (1 + np.abs(z) / 8)
            tol[lo:lo + n] = ref.allowed(out[lo:lo + n], mag, kappa, self.dt)
            ltol[i] = ref.allowed(last[i], lmag, kappa, "float32")
        return out, tol, last, ltol

    def call(self, **more):
        return ssam.ssam_scan_selective(self.x, self.raw, self.a, self.b, self.c, d_state=self.h0, **self.args, **more)


@pytest.mark.parametrize("spec", SCAN, ids=lambda s: "-".join(map(str, s)))
def test_scan_selective(spec):
    print(spec, flush=True)
    k = ScanCase(*spec)
    want, tol, last, ltol = k.forward()
    out = torch.full((*k.lead, k.D), SENTINEL, dtype=k.dtype, device="cuda")
    final = torch.full((len(k.spans), k.D, k.N), SENTINEL, device="cuda")
    assert k.call(d_out=out, d_final=final) is out
    check("out", out.reshape(k.rows, k.D), want, tol)
    check("final", final, last, ltol)
    marks = ssam.ssam_scan_selective_marks(k.x, k.a, **k.seq)
    marked = k.call(d_marks=marks)
    inside = torch.from_numpy(k.inside).cuda()
    assert torch.equal(marked.reshape(k.rows, k.D)[inside], out.reshape(k.rows, k.D)[inside])
    assert not marked.reshape(k.rows, k.D)[~inside].any()
    if k.h0 is not None:
        both = k.h0.clone()
        ssam.ssam_scan_selective(k.x, k.raw, k.a, k.b, k.c, d_state=both, d_final=both, d_out=out, **k.args)
        assert torch.equal(both, final), "the state in place"


@pytest.mark.parametrize("spec", SCAN, ids=lambda s: "-".join(map(str, s)))
def test_scan_selective_backward(spec):
    print(spec, flush=True)
    k = ScanCase(*spec)
    D, N, G = k.D, k.N, k.G
    dout = wide(k.g, k.lead, D, k.dtype, k.form)
    dlast = randn(k.g, len(k.spans), D, N) if k.h0 is not None else None
    marks = ssam.ssam_scan_selective_marks(k.x, k.a, **k.seq)
    k.call(d_marks=marks)
    back = lambda: ssam.ssam_scan_selective_backward(dout, k.x, k.raw, k.a, k.b, k.c, marks, d_grad_final=dlast, state_grad=True, **k.args)  # noqa: E731
    got = back()
    val, mag = ({n: np.zeros((k.rows, *s)) for n, s in (("x", (D,)), ("d", (D,)), ("b", (G, N)), ("c", (G, N)), ("gate", (D,)))} for _ in range(2))
    for v in (val, mag):
        v.update(a=np.zeros((D, N)), skip=np.zeros(D), dt_bias=np.zeros(D), state=np.zeros((len(k.spans), D, N)))
    for i, lo, n in k.spans:
        u, d, a, b, c, skip, z, h0, raw = k.inputs(i, lo, n)
        end = np.zeros((D, N)) if dlast is None else f64(dlast)[i]
        for v, size in ((val, False), (mag, True)):
            r = ref.scan_back(flat(dout, k.lead)[lo:lo + n], u, d, a, b, c, skip, z, h0, end, size)
            if k.softplus:
                r["d"] = r["d"] * ref.sigmoid(raw)
            for name in ("x", "d", "gate"):
                v[name][lo:lo + n] = r[name]
            for name in ("b", "c"):
                v[name][lo:lo + n] = r[name].reshape(n, G, D // G, N).sum(2)
            v["a"] += r["a"]
            v["skip"] += r["skip"]
            v["dt_bias"] += r["d"].sum(0)
            v["state"][i] = r["state"]
    # forward states and gradients pass the same chains: twice a term's error, and the gate's exponents (|z| < 6) 16 u more
    kappa = 2 * ref.scan_kappa(k.longest) + 16 * ref.U
    sums = kappa + k.rows * ref.U                      # one addition a row
    across = kappa + (16 + D // 64 + 1) * ref.U        # a tree inside a block, then a block after the other
    for name, t, e, dt in (("x", got.x, kappa, k.dt), ("d", got.dt, kappa, k.dt), ("gate", got.gate, kappa, k.dt), ("b", got.b, across, k.dt),
                           ("c", got.c, across, k.dt)):
        if t is None:
            continue
        tol = ref.allowed(val[name], mag[name], e, dt)
        tol[~k.inside] = 0
        check(name, t.reshape(val[name].shape), val[name], tol)
    for name, t, e in (("a", got.a, sums), ("skip", got.skip, sums), ("dt_bias", got.dt_bias, sums), ("state", got.state, kappa)):
        if t is not None:
            check(name, t, val[name], ref.allowed(val[name], mag[name], e, "float32"))
    assert all(torch.equal(p, q) for p, q in zip(got, back()) if p is not None), "the same call twice"


@pytest.mark.parametrize("dt,D,N,G,gate", [("bfloat16", 130, 16, 1, True), ("float32", 6, 1, 3, False), ("float16", 70, 33, 1, True),
                                           ("float32", 64, 4, 1, True), ("bfloat16", 99, 8, 3, True), ("float32", 66, 20, 2, False),
                                           ("bfloat16", 64, 64, 1, True)])
def test_scan_selective_step(dt, D, N, G, gate):
    g = torch.Generator().manual_seed(N)
    dtype = TYPES[dt]
    R, pool = 6, 5
    x, raw = randn(g, R, D + 1, dtype=dtype)[:, 1:], randn(g, R, D, dtype=dtype)
    z = randn(g, R, D, dtype=dtype) if gate else None
    both = randn(g, R, 2 * G * N + 1, dtype=dtype)
    b, c = both[:, 1:1 + G * N].unflatten(-1, (G, N)), both[:, 1 + G * N:].unflatten(-1, (G, N))
    a, skip, bias = -(torch.rand(D, N, generator=g) * 3).cuda(), randn(g, D), randn(g, D) - 2
    state = randn(g, pool, 2, D, N)[:, 1]
    before = state.clone()
    slots = [2, 2, -7, 0, 2, 5]
    out = torch.full((R, D), SENTINEL, dtype=dtype, device="cuda")
    ssam.ssam_scan_selective_step(x, raw, a, b, c, state, skip=skip, gate=z, dt_bias=bias, softplus=True,
                                  slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), d_out=out)
    want, tol, after = np.full((R, D), SENTINEL), np.zeros((R, D)), f64(before)
    size = np.abs(after)
    d = ref.softplus(f64(raw) + f64(bias))
    wide_b, wide_c = np.repeat(f64(b), D // G, 1), np.repeat(f64(c), D // G, 1)
    kappa = ref.scan_kappa(3)
    for r, s in enumerate(slots):
        if 0 <= s < pool:
            zr = None if z is None else f64(z)[r:r + 1]
            y, after[s] = ref.scan(f64(x)[r:r + 1], d[r:r + 1], f64(a), wide_b[r:r + 1], wide_c[r:r + 1], f64(skip), zr, after[s])
            m, size[s] = ref.scan(np.abs(f64(x)[r:r + 1]), d[r:r + 1], f64(a), np.abs(wide_b[r:r + 1]), np.abs(wide_c[r:r + 1]), np.abs(f64(skip)),
                                  None, size[s])
            if zr is not None:
                m = m * np.abs(zr * ref.sigmoid(zr)) * (1 + np.abs(zr) / 8)
            want[r], tol[r] = y[0], ref.allowed(y, m, kappa, dt)[0]
    check("out", out, want, tol)
    check("state", state, after, ref.allowed(after, size, kappa, "float32"))
    untouched = [s for s in range(pool) if s not in slots]
    assert torch.equal(state[untouched], before[untouched])


# ---- as they are used together -----------------------------------------------------------------------------------------
class Layer:
    """A small state space layer's parameters."""

    def __init__(self, D, N, W, dtype, seed=1):
        g = torch.Generator().manual_seed(seed)
        self.w, self.wb = randn(g, D, W, dtype=dtype, scale=0.5), randn(g, D, dtype=dtype, scale=0.1)
        self.proj = randn(g, D, D + 2 * N, dtype=dtype, scale=D ** -0.5)
        self.a = -torch.arange(1, N + 1, dtype=torch.float32).repeat(D, 1).cuda()
        self.skip, self.bias = randn(g, D), randn(g, D) - 3
        self.D, self.N = D, N

    def split(self, v):
        p = v @ self.proj
        b, c = p[..., self.D:self.D + self.N], p[..., self.D + self.N:]
        return p[..., :self.D], b.unsqueeze(-2), c.unsqueeze(-2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_prompt_then_tokens_is_the_whole_sequence(dtype):
    """Filter and scan over a prompt, then token by token from the states it left, against one call over everything."""
    D, N, W, rows, cut = 96, 16, 4, 101, 90
    net = Layer(D, N, W, dtype)
    g = torch.Generator().manual_seed(2)
    xz = randn(g, rows, 2 * D, dtype=dtype)

    def prompt(xz, conv_state, state):
        v = ssam.ssam_conv1d(xz[:, :D], net.w, bias=net.wb, silu=True, d_final=conv_state)
        dt, b, c = net.split(v)
        return ssam.ssam_scan_selective(v, dt, net.a, b, c, skip=net.skip, gate=xz[:, D:], dt_bias=net.bias, softplus=True, d_final=state)

    whole_conv, whole_state = torch.empty(1, W - 1, D, dtype=dtype, device="cuda"), torch.empty(1, D, N, device="cuda")
    whole = prompt(xz, whole_conv, whole_state)
    conv_pool, pool = torch.zeros(3, W - 1, D, dtype=dtype, device="cuda"), torch.zeros(3, D, N, device="cuda")
    first = prompt(xz[:cut], conv_pool[1:2], pool[1:2])
    at = torch.tensor([1], dtype=torch.int32, device="cuda")
    outs = [first]
    for t in range(cut, rows):
        row = xz[t:t + 1]
        v = ssam.ssam_conv1d_step(row[:, :D], net.w, conv_pool, bias=net.wb, silu=True, slots=at)
        dt, b, c = net.split(v)
        outs.append(ssam.ssam_scan_selective_step(v, dt, net.a, b, c, pool, skip=net.skip, gate=row[:, D:], dt_bias=net.bias, softplus=True, slots=at))
    got = torch.cat(outs)
    assert torch.equal(conv_pool[1:2], whole_conv) and not conv_pool[0].any() and not pool[2].any()
    # the projection's own rounding may differ between one row and many: a step or two of the type on every input
    step = 2 * ref.HALF_STEP[NAME[dtype]]
    scale = whole.float().abs().max()
    assert (got.float() - whole.float()).abs().max() <= (16 * step + 1e-5) * scale
    assert (pool[1:2] - whole_state).abs().max() <= (16 * step + 1e-5) * whole_state.abs().max()
    # and the prompt in two calls, the state handed on
    conv_state, state = torch.zeros(1, W - 1, D, dtype=dtype, device="cuda"), torch.zeros(1, D, N, device="cuda")
    parts = []
    for lo, hi in ((0, 1), (1, 40), (40, rows)):
        v = ssam.ssam_conv1d(xz[lo:hi, :D], net.w, bias=net.wb, silu=True, d_state=conv_state, d_final=conv_state)
        dt, b, c = net.split(v)
        parts.append(ssam.ssam_scan_selective(v, dt, net.a, b, c, skip=net.skip, gate=xz[lo:hi, D:], dt_bias=net.bias, softplus=True, d_state=state,
                                              d_final=state))
    assert torch.equal(conv_state, whole_conv)
    assert (torch.cat(parts).float() - whole.float()).abs().max() <= (16 * step + 1e-5) * scale


def test_gradient_against_differences():
    """The loss sum(out * r) along a random direction of all inputs: (f(+e) - f(-e)) / 2e in fp32.  f is a sum of 5000 values of size 1,
    off by 1e-4 at most; with e = 2^-6 that is 3e-3 of the difference's 1, and the third derivative adds e^2."""
    g = torch.Generator().manual_seed(3)
    T, D, N, W = 40, 128, 16, 4
    p = {"x": randn(g, T, D), "w": randn(g, D, W, scale=0.5), "wb": randn(g, D, scale=0.1), "dt": randn(g, T, D, scale=0.3),
         "a": -(torch.rand(D, N, generator=g) + 0.5).cuda(), "b": randn(g, T, 1, N, scale=0.5), "c": randn(g, T, 1, N, scale=0.5), "skip": randn(g, D),
         "z": randn(g, T, D), "bias": randn(g, D) - 1}
    r = randn(g, T, D)

    def forward(p, marks=None):
        v = ssam.ssam_conv1d(p["x"], p["w"], bias=p["wb"], silu=True)
        return v, ssam.ssam_scan_selective(v, p["dt"], p["a"], p["b"], p["c"], skip=p["skip"], gate=p["z"], dt_bias=p["bias"], softplus=True, d_marks=marks)

    marks = ssam.ssam_scan_selective_marks(p["x"], p["a"])
    v, _ = forward(p, marks)
    s = ssam.ssam_scan_selective_backward(r, v, p["dt"], p["a"], p["b"], p["c"], marks, skip=p["skip"], gate=p["z"], dt_bias=p["bias"], softplus=True)
    k = ssam.ssam_conv1d_backward(s.x, p["x"], p["w"], bias=p["wb"], silu=True)
    grads = {"x": k.x, "w": k.weight, "wb": k.bias, "dt": s.dt, "a": s.a, "b": s.b, "c": s.c, "skip": s.skip, "z": s.gate, "bias": s.dt_bias}
    e = 2.0 ** -6
    for name in p:
        way = randn(g, *p[name].shape)
        way = way / way.norm()
        there, back = dict(p), dict(p)
        there[name], back[name] = p[name] + e * way, p[name] - e * way
        slope = ((forward(there)[1].double() - forward(back)[1].double()) * r.double()).sum().item() / (2 * e)
        want = (grads[name].double() * way.double()).sum().item()
        assert abs(slope - want) <= 1e-2 * (1 + grads[name].double().norm().item()), (name, slope, want)


def test_captured_and_replayed():
    """A training step and a token's step in graphs, replayed several times with eager work between."""
    D, N, W, T = 128, 16, 4, 200
    net = Layer(D, N, W, torch.bfloat16)
    g = torch.Generator().manual_seed(4)
    x, z, dt, dy = (randn(g, T, D, dtype=torch.bfloat16) for _ in range(4))
    b, c = (randn(g, T, 1, N, dtype=torch.bfloat16) for _ in range(2))
    marks = ssam.ssam_scan_selective_marks(x, net.a)
    row = dict(skip=net.skip, gate=z, dt_bias=net.bias, softplus=True)

    def train():
        v = ssam.ssam_conv1d(x, net.w, bias=net.wb, silu=True)
        y = ssam.ssam_scan_selective(v, dt, net.a, b, c, d_marks=marks, **row)
        s = ssam.ssam_scan_selective_backward(dy, v, dt, net.a, b, c, marks, **row)
        k = ssam.ssam_conv1d_backward(s.x, x, net.w, bias=net.wb, silu=True)
        return [y, *(t for t in (*s, *k) if t is not None)]

    pool, conv_pool = torch.zeros(4, D, N, device="cuda"), torch.zeros(4, W - 1, D, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([2, 0], dtype=torch.int32, device="cuda")

    def token():
        v = ssam.ssam_conv1d_step(x[:2], net.w, conv_pool, bias=net.wb, silu=True, slots=slots)
        return ssam.ssam_scan_selective_step(v, dt[:2], net.a, b[:2], c[:2], pool, skip=net.skip, gate=z[:2], dt_bias=net.bias, softplus=True, slots=slots)

    eager = [t.clone() for t in train()]
    tokens = [token().clone() for _ in range(3)]
    states = [pool.clone(), conv_pool.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        train()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        trained = train()
    with torch.cuda.graph(graphs[1]):
        said = token()
    pool.zero_()
    conv_pool.zero_()
    for i in range(3):
        for t in trained:
            t.zero_()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(trained, eager)), i
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(said, tokens[i]), i
        (x.float() @ x.float().t()).sum().item()
    assert torch.equal(pool, states[0]) and torch.equal(conv_pool, states[1])


def test_on_another_stream():
    D, N, T = 64, 16, 500
    g = torch.Generator().manual_seed(6)
    x, dt = randn(g, T, D), randn(g, T, D)
    b, c = randn(g, T, 1, N), randn(g, T, 1, N)
    a = -(torch.rand(D, N, generator=g) + 0.1).cuda()
    here = ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    outs = [ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True, stream=other) for _ in range(4)]
    junk = [torch.full((1 << 16,), float("nan"), device="cuda") for _ in range(8)]      # takes what the calls gave back
    torch.cuda.synchronize()
    del junk
    assert all(torch.equal(o, here) for o in outs)


def test_what_a_call_allocates_belongs_to_its_stream():
    """Results start as zeros where rows may belong to no sequence: filled on the call's stream, not behind the current one's work."""
    D, N, T = 64, 16, 500
    g = torch.Generator().manual_seed(8)
    x, dt, dy = (randn(g, T, D) for _ in range(3))
    b, c = randn(g, T, 1, N), randn(g, T, 1, N)
    a, w = -(torch.rand(D, N, generator=g) + 0.1).cuda(), randn(g, D, 4)
    starts = torch.tensor([0, 200, 490], dtype=torch.int32, device="cuda")
    marks = ssam.ssam_scan_selective_marks(x, a, starts=starts)
    pool, slots = torch.zeros(3, 3, D, device="cuda"), torch.tensor([0, 2], dtype=torch.int32, device="cuda")

    def calls(stream):
        y = ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True, d_marks=marks, starts=starts, stream=stream)
        s = ssam.ssam_scan_selective_backward(dy, x, dt, a, b, c, marks, softplus=True, starts=starts, stream=stream)
        return [y, s.x, s.b, s.a, ssam.ssam_conv1d(x, w, starts=starts, stream=stream),
                *ssam.ssam_conv1d_backward(dy, x, w, starts=starts, stream=stream)[:2],
                ssam.ssam_conv1d_step(x[:2], w, pool.clone() if stream is None else pools, slots=slots, stream=stream)]

    want = calls(None)
    pools = pool.clone()
    heavy = torch.ones(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(4):
        heavy = heavy @ heavy * 1e-4                     # milliseconds of the current stream's
    got = calls(other)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_two_streams_at_once():
    """Calls in flight together have workspaces of their own."""
    D, N, T = 256, 16, 3000
    g = torch.Generator().manual_seed(10)
    sets = [[randn(g, T, D), randn(g, T, D), -(torch.rand(D, N, generator=g) + 0.1).cuda(), randn(g, T, 1, N), randn(g, T, 1, N), randn(g, T, D),
             randn(g, D, 4)] for _ in range(2)]

    def calls(x, dt, a, b, c, dy, w, stream):
        marks = ssam.ssam_scan_selective_marks(x, a)
        y = ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True, d_marks=marks, stream=stream)
        s = ssam.ssam_scan_selective_backward(dy, x, dt, a, b, c, marks, softplus=True, stream=stream)
        k = ssam.ssam_conv1d_backward(dy, x, w, silu=True, stream=stream)
        return [marks, y, *(t for t in (*s, *k) if t is not None)]

    want = [calls(*s, None) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [calls(*s, stream) for _ in range(4) for s, stream in zip(sets, streams)]
    torch.cuda.synchronize()
    for i, result in enumerate(got):
        assert all(torch.equal(p, q) for p, q in zip(result, want[i % 2])), i


def test_infinities_stay_in_their_sequence_and_channel():
    """A NaN or an infinity in one channel of one sequence, or in rows of no sequence, reaches nothing else."""
    D, N = 64, 16
    g = torch.Generator().manual_seed(7)
    x, dt, z = (randn(g, 120, D) for _ in range(3))
    b, c = randn(g, 120, 1, N), randn(g, 120, 1, N)
    a = -(torch.rand(D, N, generator=g) + 0.1).cuda()
    a[5, 3] = float("-inf")
    w = randn(g, D, 4)
    starts = torch.tensor([0, 50, 50, 117], dtype=torch.int32, device="cuda")
    clean = ssam.ssam_scan_selective(x, dt, a, b, c, gate=z, softplus=True, starts=starts)
    clean_conv = ssam.ssam_conv1d(x, w, silu=True, starts=starts)
    assert torch.isfinite(clean).all()
    for t in (x, dt, z, b, c):
        t[117:] = float("nan")
    x[20, 9] = float("inf")
    final = torch.empty(3, D, N, device="cuda")
    got, got_conv = ssam.ssam_scan_selective(x, dt, a, b, c, gate=z, softplus=True, starts=starts, d_final=final), ssam.ssam_conv1d(x, w, silu=True, starts=starts)
    for u, v in ((got, clean), (got_conv, clean_conv)):
        same = torch.ones_like(u, dtype=torch.bool)
        same[20:50, 9] = False
        assert torch.equal(u[same], v[same])
        assert not torch.isfinite(u[20, 9])
    assert torch.isfinite(final[1:]).all() and torch.isfinite(final[0, :9]).all() and torch.isfinite(final[0, 10:]).all()


@pytest.mark.parametrize("rows", [5, 33])
def test_an_infinite_state_passes_the_end_of_its_sequence(rows):
    """Tiles end behind the last row: what lies there adds nothing, not even zero times an infinity."""
    D, N = 64, 16
    g = torch.Generator().manual_seed(9)
    x, dt, dy = randn(g, rows, D).abs() + 0.1, randn(g, rows, D), randn(g, rows, D).abs() + 0.1
    b, c = randn(g, rows, 1, N), randn(g, rows, 1, N)
    a = -(torch.rand(D, N, generator=g) + 0.1).cuda()
    b[-1, 0, 3] = float("inf")
    final, marks = torch.empty(1, D, N, device="cuda"), ssam.ssam_scan_selective_marks(x, a)
    ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True, d_final=final, d_marks=marks)
    assert (final[0, :, 3] == float("inf")).all() and torch.isfinite(final[0, :, :3]).all() and torch.isfinite(final[0, :, 4:]).all()
    b[-1, 0, 3], c[-1, 0, 3] = 0.5, float("inf")
    got = ssam.ssam_scan_selective_backward(dy, x, dt, a, b, c, marks, softplus=True, state_grad=True)
    assert (got.b[-1, 0, 3] == float("inf")).all() and (got.state[0, :, 3] == float("inf")).all()
    assert torch.isfinite(got.state[0, :, :3]).all() and torch.isfinite(got.b[:, 0, :3]).all() and torch.isfinite(got.c).all()


def test_refusals_of_the_binding():
    """Shapes, types, layouts: refused before anything runs."""
    D, N = 8, 4
    x, w = torch.zeros(6, D, device="cuda"), torch.zeros(D, 4, device="cuda")
    a, b = torch.zeros(D, N, device="cuda"), torch.zeros(6, 1, N, device="cuda")
    starts = torch.tensor([0, 6], dtype=torch.int32, device="cuda")

    def refused(match, f, *args, error=ValueError, **kw):
        with pytest.raises(error, match=match):
            f(*args, **kw)
    conv, step = ssam.ssam_conv1d, ssam.ssam_conv1d_step
    refused("weight", conv, x, w[:7])
    refused("weight", conv, x, w.half())
    refused("bias", conv, x, w, bias=torch.zeros(D))
    refused("bias", conv, x, w, bias=torch.zeros(7, device="cuda"))
    refused("d_in", conv, x[0], w)
    refused("contiguous channels", conv, x.t().contiguous().t(), w)
    refused("unsupported dtype", conv, x.double(), w.double(), error=TypeError)
    refused("d_out", conv, x, w, d_out=x[:5].clone())
    refused("d_state", conv, x, w, d_state=torch.zeros(2, 3, D, device="cuda"))
    refused("starts", conv, x, w, starts=starts.long())
    refused("starts", conv, x.view(2, 3, D), w, starts=starts)
    refused("starts", conv, x, w, starts=starts, lengths=starts)
    refused("lengths", conv, x, w, lengths=starts)
    refused("lengths", conv, x.view(2, 3, D), w, lengths=starts[:1])
    refused(None, conv, x, torch.zeros(D, 9, device="cuda"), error=ssam.SsamError)
    refused(None, conv, x, w, d_out=x, error=ssam.SsamError)
    refused("slot for each", step, x, w, torch.zeros(5, 3, D, device="cuda"))
    refused("d_state", step, x, w, torch.zeros(6, 2, D, device="cuda"))
    refused("contiguous slots", step, x, w, torch.zeros(6, 3, 2 * D, device="cuda")[..., ::2])
    refused("overlap", step, x, w, torch.zeros(3, D, device="cuda").expand(6, 3, D))
    refused("slots", step, x, w, torch.zeros(6, 3, D, device="cuda"), slots=starts)
    scan, back, mark = ssam.ssam_scan_selective, ssam.ssam_scan_selective_backward, ssam.ssam_scan_selective_marks
    refused("a must", scan, x, x, a.half(), b, b)
    refused("a must", scan, x, x, a.t(), b, b)
    refused("d_dt", scan, x, x.half(), a, b, b)
    refused("c and b", scan, x, x, a, b, torch.zeros(6, 2, N, device="cuda"))
    refused("c and b", scan, x, x, a, torch.zeros(6, 1, 3, device="cuda"), torch.zeros(6, 1, 3, device="cuda"))
    refused("b must", scan, x, x, a, b[:, 0], b)
    refused("skip", scan, x, x, a, b, b, skip=torch.zeros(D, device="cuda").half())
    refused("gate", scan, x, x, a, b, b, gate=x[:, :7])
    refused("d_marks", scan, x, x, a, b, b, d_marks=torch.zeros(1, N, D, device="cuda"))
    refused("d_marks", scan, x.repeat(8, 1), x.repeat(8, 1), a, b.repeat(8, 1, 1), b.repeat(8, 1, 1), d_marks=mark(x, a))
    refused("d_marks", back, x, x, x, a, b, b, a)
    refused("must be a tensor", back, None, x, x, a, b, b, mark(x, a), error=TypeError)
    refused(None, scan, x, x, a, torch.zeros(6, 3, N, device="cuda"), torch.zeros(6, 3, N, device="cuda"), error=ssam.SsamError)
    big = torch.zeros(400, D, device="cuda")
    bb = torch.zeros(400, 1, N, device="cuda")
    refused(None, scan, big, big, a, bb, bb, d_work=torch.zeros(8, device="cuda"), error=ssam.SsamError)


def test_own_workspace_and_results():
    D, N = 64, 16
    g = torch.Generator().manual_seed(9)
    x, dt = randn(g, 400, D), randn(g, 400, D)
    b, c = randn(g, 400, 1, N), randn(g, 400, 1, N)
    a = -(torch.rand(D, N, generator=g) + 0.1).cuda()
    need = ssam.ssam_scan_selective_workspace_bytes(x, a)
    assert need > 0
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")        # NaN everywhere
    out = torch.full((400, D), float("nan"), device="cuda")
    assert ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True, d_work=work, d_out=out) is out
    assert torch.equal(out, ssam.ssam_scan_selective(x, dt, a, b, c, softplus=True))


def test_offsets_past_32_bits():
    """Rows 2^31 elements and more behind the first: a tall buffer of which only the last rows are a sequence."""
    D, N, W = 1024, 4, 4
    T = (1 << 32) // D + 70            # 2^32 elements and 70 rows
    g = torch.Generator().manual_seed(8)
    x = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
    tail = randn(g, 64, D, dtype=torch.bfloat16)
    x[T - 64:] = tail
    starts = torch.tensor([T - 64, T], dtype=torch.int32, device="cuda")
    w = randn(g, D, W, dtype=torch.bfloat16)
    out = torch.empty_like(x)
    ssam.ssam_conv1d(x, w, silu=True, starts=starts, d_out=out)
    assert torch.equal(out[T - 64:], ssam.ssam_conv1d(tail, w, silu=True))
    a = -(torch.rand(D, N, generator=g) + 0.1).cuda()
    bc = torch.zeros(T, 2, N, dtype=torch.bfloat16, device="cuda")
    bc[T - 64:] = randn(g, 64, 2, N, dtype=torch.bfloat16)
    ssam.ssam_scan_selective(x, x, a, bc[:, :1], bc[:, 1:], softplus=True, starts=starts, d_out=out)
    short = ssam.ssam_scan_selective(tail, tail, a, bc[T - 64:, :1], bc[T - 64:, 1:], softplus=True)
    assert torch.equal(out[T - 64:], short)
