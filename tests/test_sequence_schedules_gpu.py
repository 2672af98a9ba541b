"""The sequence operators at sizes that run the schedules of real calls: pieces of more than one tile, whole sequences of many tiles, the
filter's longer pieces, and slots far apart; against their definitions in 64 bits, evaluated on the device."""
import numpy as np
import pytest

import sequence_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_1907_06154_amd as ssam  # noqa: E402

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
NAME = {v: k for k, v in TYPES.items()}
SENTINEL = 7.0


def check(what, got, want, tol):
    got = got.double().reshape(want.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = (got - want).abs() / tol.clamp(min=1e-300)
    bad = off > 1
    bad |= (tol == 0) & (got != want)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} values off, the worst {off.max().item():.3g} times what is allowed"


def allowed(want, mag, kappa, dt):
    return ref.HALF_STEP[dt] * want.abs() * (1 + kappa) + kappa * mag + ref.TINY[dt]


# ---- scan --------------------------------------------------------------------------------------------------------------

# name: leading extents, starts, lengths, channels, states, type, gate, rows of a piece forward and back (None: sequences stay whole)
SCANS = {
    "whole_9": ((130, 203), None, None, 256, 9, "bfloat16", True, None, None),
    "whole_8": ((260, 150), None, None, 256, 8, "float16", False, None, None),
    "whole_padded_20": ((300, 170), None, [170 - i * 7 % 171 for i in range(300)], 256, 20, "float32", True, None, None),
    "pieces_4": ((8, 333), None, None, 4160, 4, "float32", True, 64, 96),
    "whole_then_pieces_16": ((5, 333), None, None, 4160, 16, "bfloat16", True, None, 128),
    "pieces_16": ((1500,), None, None, 4160, 16, "float16", True, 96, 96),
    # more sequences than one launch of the gradients takes
    "many_16": ((11003, 3), None, [i * 5 % 4 for i in range(11003)], 130, 16, "bfloat16", True, None, None),
    "packed_4": ((6000,), [0, 17, 2900, 2900, 5000, 5990], None, 4160, 4, "bfloat16", True, 64, 128),
}


class Scan:
    def __init__(self, name):
        lead, starts, lengths, D, N, dt, gate, self.piece, self.back_piece = SCANS[name]
        g = torch.Generator(device="cuda").manual_seed(len(name) + N)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        dtype = TYPES[dt]
        self.lead, self.D, self.N, self.dt = lead, D, N, dt
        self.x, self.raw, self.dout = (rand(*lead, D).to(dtype) for _ in range(3))
        self.z = rand(*lead, D).to(dtype) if gate else None
        self.b, self.c = rand(*lead, 1, N).to(dtype), rand(*lead, 1, N).to(dtype)
        self.bias, self.skip = rand(D) - 3, rand(D)
        self.a = -(torch.rand(D, N, generator=g, device="cuda") * 3 + 0.05)
        self.spans = ref.spans(lead[-1], starts, lengths, lead[0] if len(lead) == 2 else None)
        S = len(self.spans)
        self.h0, self.dlast = rand(S, D, N), rand(S, D, N)
        dev = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.seq = dict(starts=dev(starts), lengths=dev(lengths))
        self.args = dict(skip=self.skip, gate=self.z, dt_bias=self.bias, softplus=True, **self.seq)

    def groups(self):
        """[(sequences, first flat row of each, rows)] of sequences that are evaluated side by side, a padded batch's short ones with them."""
        if len(self.lead) == 2:
            return [(list(range(self.lead[0])), [lo for _, lo, _ in self.spans], self.lead[1])]
        return [([i], [lo], n) for i, lo, n in self.spans if n]

    def definition(self, size):
        """Everything in 64 bits; size: with every term's magnitude instead."""
        mag = (lambda v: v.abs()) if size else (lambda v: v)
        D, N, rows = self.D, self.N, int(np.prod(self.lead))
        flat = lambda t: t.reshape(rows, *t.shape[len(self.lead):])  # noqa: E731
        a, skip = self.a.double(), mag(self.skip.double())
        v = {n: torch.zeros(rows, D, dtype=torch.float64, device="cuda") for n in ("out", "x", "d", "gate")}
        v.update({n: torch.zeros(rows, N, dtype=torch.float64, device="cuda") for n in ("b", "c")})
        v.update(a=torch.zeros_like(a), skip=torch.zeros_like(skip), dt_bias=torch.zeros_like(skip), final=mag(self.h0.double()).clone(),
                 state=mag(self.dlast.double()).clone())                  # (of an empty sequence they pass as they are)
        for seqs, first, n in self.groups():
            first = torch.tensor(first, device="cuda")
            length = torch.tensor([self.spans[i][2] for i in seqs], device="cuda")

            def row(t):
                at = (first + t).clamp(max=rows - 1)
                live = (t < length)[:, None]
                raw = flat(self.raw)[at].double() + self.bias.double()
                d = torch.logaddexp(raw, torch.zeros_like(raw)) * live           # behind a sequence's end nothing changes
                u, b, c = (mag(flat(t_)[at].double()) for t_ in (self.x, self.b, self.c))
                return at, live, raw, d, u, b, c, torch.exp(d[..., None] * a)

            h = mag(self.h0[seqs].double())
            hs = torch.empty(n + 1, *h.shape, dtype=torch.float64, device="cuda")
            hs[0] = h
            for t in range(n):
                at, live, raw, d, u, b, c, e = row(t)
                hs[t + 1] = e * hs[t] + (d * u)[..., None] * b
            v["final"][seqs] = hs[n]
            carry = mag(self.dlast[seqs].double())
            for t in reversed(range(n)):
                at, live, raw, d, u, b, c, e = row(t)
                go = mag(flat(self.dout)[at].double()) * live
                y = (hs[t + 1] * c).sum(-1) + skip * u
                s1, s2 = 1.0, 0.0
                if self.z is not None:
                    z = flat(self.z)[at].double()
                    s = torch.sigmoid(z)
                    s1, s2 = mag(z * s), (1.1 + z.abs() * s * (1 - s)) if size else s * (1 + z * (1 - s))
                    fwd = y * s1 * ((1 + z.abs() / 8) if size else 1)
                else:
                    fwd = y
                dy = go * s1
                g = c * dy[..., None] + carry
                q = g * e * hs[t] * live[..., None]
                gb = (g * b).sum(-1)
                dd = ((mag(a) * q).sum(-1) + u * gb) * torch.sigmoid(raw) * live
                keep, to = live[:, 0], at[live[:, 0]]
                for name, val in (("out", fwd), ("x", skip * dy + d * gb), ("d", dd), ("gate", go * y * s2),
                                  ("b", (g * (d * u)[..., None]).sum(1)), ("c", (hs[t + 1] * dy[..., None]).sum(1))):
                    v[name][to] = val[keep]
                v["a"] += (d[..., None] * q).sum(0)
                v["skip"] += (dy * u).sum(0)
                v["dt_bias"] += dd.sum(0)
                carry = torch.where(live[..., None], e * g, carry)
            v["state"][seqs] = carry
        return v


def kappa(n, piece):
    """ref.scan_kappa for pieces of any length: n rows of 4 u, 11 u of a chain's exponent up to 30, the gate's and other factors' 24 u, and where
    sequences are cut the sums of a piece's time steps, `piece` additions."""
    return (4 * n + 30 * 11 + (30 * piece if piece and n > piece else 0) + 24) * ref.U


@pytest.mark.parametrize("name", SCANS)
def test_scan(name):
    print(name, flush=True)
    k = Scan(name)
    rows, S, D, N = int(np.prod(k.lead)), len(k.spans), k.D, k.N
    longest = max(n for _, _, n in k.spans)
    # the schedule that the case is for
    need = ssam.ssam_scan_selective_workspace_bytes(k.x, k.a, **k.seq)
    if k.piece is None:
        assert need == 0
    else:
        slots = k.lead[0] // k.piece + S if len(k.lead) == 1 and k.seq["starts"] is not None else -(-k.lead[-1] // k.piece) * S
        assert need == slots * (D * N + D) * 4
    val, mag = k.definition(False), k.definition(True)
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for _, lo, n in k.spans:
        inside[lo:lo + n] = True
    out = torch.full((*k.lead, D), SENTINEL, dtype=k.x.dtype, device="cuda")
    final, marks = torch.full_like(k.h0, SENTINEL), ssam.ssam_scan_selective_marks(k.x, k.a, **k.seq)
    ssam.ssam_scan_selective(k.x, k.raw, k.a, k.b, k.c, d_state=k.h0, d_final=final, d_marks=marks, d_out=out, **k.args)
    e = kappa(longest, k.piece)
    tol = allowed(val["out"], mag["out"], e, k.dt)
    val["out"][~inside], tol[~inside] = SENTINEL, 0
    check("out", out, val["out"], tol)
    check("final", final, val["final"], allowed(val["final"], mag["final"], e, "float32"))
    plain = ssam.ssam_scan_selective(k.x, k.raw, k.a, k.b, k.c, d_state=k.h0, **k.args).reshape(rows, D)
    assert torch.equal(plain[inside], out.reshape(rows, D)[inside]) and not plain[~inside].any()
    got = ssam.ssam_scan_selective_backward(k.dout, k.x, k.raw, k.a, k.b, k.c, marks, d_grad_final=k.dlast, state_grad=True, **k.args)
    e = kappa(longest, k.piece) + kappa(longest, k.back_piece) + 16 * ref.U        # states and gradients, each their chains
    sums, across = e + rows * ref.U, e + (16 + D // 64 + 1) * ref.U
    for name, t, err in (("x", got.x, e), ("d", got.dt, e), ("gate", got.gate, e), ("b", got.b, across), ("c", got.c, across)):
        if t is not None:
            tol = allowed(val[name], mag[name], err, k.dt)
            tol[~inside] = 0
            check(name, t, val[name], tol)
    for name, t, err in (("a", got.a, sums), ("skip", got.skip, sums), ("dt_bias", got.dt_bias, sums), ("state", got.state, e)):
        check(name, t, val[name], allowed(val[name], mag[name], err, "float32"))


# ---- filter ------------------------------------------------------------------------------------------------------------

# leading extents, starts, channels, taps, type, rows of a piece forward and back: the most rows for which slots x strips reach 4096
FILTERS = {
    "batch": ((3, 11003), None, 1000, 4, "float32", 16, 32), "two": ((2, 9001), None, 1000, 3, "float32", 16, 16),
    "long": ((70001,), None, 1030, 8, "bfloat16", 32, 64),
    "packed": ((70001,), [0, 33, 34, 34, 20000, 60001, 69990], 777, 7, "float16", 32, 64),
}


def filter_piece(lead, starts, channels, each, longest):
    """Rows of a piece by the library's rule."""
    strips, rows = -(-channels // (64 * each)), longest
    slots = lambda: lead[0] // rows + len(starts) - 1 if starts else -(-lead[-1] // rows) * (lead[0] if len(lead) == 2 else 1)  # noqa: E731
    while rows > 8 and slots() * strips < 4096:
        rows //= 2
    return rows, slots()


@pytest.mark.parametrize("name", FILTERS)
def test_filter(name):
    print(name, flush=True)
    lead, starts, D, W, dt, piece, back_piece = FILTERS[name]
    dtype = TYPES[dt]
    assert filter_piece(lead, starts, D, 128 // torch.finfo(dtype).bits, 16 if W <= 4 else 32)[0] == piece
    assert filter_piece(lead, starts, D, 4, 64)[0] == back_piece
    g = torch.Generator(device="cuda").manual_seed(W)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    spans = ref.spans(lead[-1], starts, None, lead[0] if len(lead) == 2 else None)
    S, rows = len(spans), int(np.prod(lead))
    x, dy, w, b, h, dlast = rand(*lead, D), rand(*lead, D), rand(D, W), rand(D), rand(S, W - 1, D), rand(S, W - 1, D)
    seq = dict(starts=None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda"))
    out, final = torch.full((*lead, D), SENTINEL, dtype=dtype, device="cuda"), torch.empty_like(h)
    ssam.ssam_conv1d(x, w, bias=b, silu=True, d_state=h, d_final=final, d_out=out, **seq)
    got = ssam.ssam_conv1d_backward(dy, x, w, bias=b, silu=True, d_state=h, d_grad_final=dlast, state_grad=True, **seq)
    dw, dwm, db, dbm = (torch.zeros(s, dtype=torch.float64, device="cuda") for s in ((D, W), (D, W), D, D))
    kap = (2 * W + 14) * ref.U
    flat = lambda t: t.reshape(rows, D)  # noqa: E731
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    w64, b64 = w.double(), b.double()
    for i, lo, n in spans:                       # as ref.conv1d and ref.conv1d_back, and with their bounds
        inside[lo:lo + n] = True
        line = torch.cat([h[i].double(), flat(x)[lo:lo + n].double()])
        p, pm = b64.expand(n, D).clone(), b64.abs().expand(n, D).clone()
        for j in range(W):
            p += w64[:, j] * line[j:j + n]
            pm += (w64[:, j] * line[j:j + n]).abs()
        s = torch.sigmoid(p)
        y = p * s
        bound = 1.1 * (W + 1) * ref.U * pm + (8 + 2 * p.abs()) * ref.U * y.abs()
        if n:
            check("out", flat(out)[lo:lo + n], y, ref.HALF_STEP[dt] * (y.abs() + bound) + bound + ref.TINY[dt])
        assert torch.equal(final[i].double(), line[n:])
        go = flat(dy)[lo:lo + n].double()
        q, qm = go * s * (1 + p * (1 - s)), go.abs() * (1.1 + pm + p.abs())
        dr, dm = torch.zeros_like(line), torch.zeros_like(line)
        for j in range(W):
            dw[:, j] += (q * line[j:j + n]).sum(0)
            dwm[:, j] += (qm * line[j:j + n].abs()).sum(0)
            dr[j:j + n] += q * w64[:, j]
            dm[j:j + n] += qm * w64[:, j].abs()
        dr[n:] += dlast[i].double()
        dm[n:] += dlast[i].double().abs()
        db += q.sum(0)
        dbm += qm.sum(0)
        if n:
            check("x", flat(got.x)[lo:lo + n], dr[W - 1:], allowed(dr[W - 1:], dm[W - 1:], kap, dt))
        check("state", got.state[i], dr[:W - 1], allowed(dr[:W - 1], dm[:W - 1], kap, dt))
    assert (flat(out)[~inside] == SENTINEL).all() and not flat(got.x)[~inside].any()
    total = kap + rows * ref.U
    check("weight", got.weight, dw, allowed(dw, dwm, total, dt))
    check("bias", got.bias, db, allowed(db, dbm, total, dt))


# ---- slots -------------------------------------------------------------------------------------------------------------

def far_slots(rows, pool):
    """Rows' slots: each its own, but for pairs 1, 63, 64, 65, 511, 512 and 513 rows apart, one slot named by every 70th row, and some outside."""
    slots = np.random.default_rng(3).permutation(pool)[:rows]
    taken = set(range(0, rows, 70))
    slots[sorted(taken)] = slots[0]
    for k, apart in enumerate((1, 63, 64, 65, 511, 512, 513)):
        r = next(r for r in range(3 + 5 * k, rows) if r not in taken and r + apart not in taken)
        slots[r + apart] = slots[r]
        taken |= {r, r + apart}
    for r, bad in ((9, -1), (100, pool), (rows - 1, -2 ** 31), (rows - 2, 2 ** 31 - 1)):
        while r in taken:
            r -= 1
        slots[r] = bad
        taken.add(r)
    return slots.astype(np.int64)


@pytest.mark.parametrize("dt,W,D", [("float32", 4, 40), ("bfloat16", 3, 530), ("float16", 8, 3)])
def test_filter_step_with_slots_far_apart(dt, W, D):
    rows, pool = 640, 700
    g = torch.Generator().manual_seed(W)
    rand = lambda *s: torch.randn(s, generator=g).to(TYPES[dt]).cuda()  # noqa: E731
    x, w, b, state = rand(rows, D), rand(D, W), rand(D), rand(pool, W - 1, D)
    before, slots = state.double().cpu().numpy(), far_slots(rows, pool)
    out = torch.full((rows, D), SENTINEL, dtype=x.dtype, device="cuda")
    ssam.ssam_conv1d_step(x, w, state, bias=b, silu=True, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), d_out=out)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    want, tol = np.full((rows, D), SENTINEL), np.zeros((rows, D))
    for r, s in enumerate(slots):
        if 0 <= s < pool:
            y, before[s], bound = ref.conv1d(f(x)[r:r + 1], f(w), f(b), True, before[s])
            want[r], tol[r] = y[0], (ref.HALF_STEP[dt] * (np.abs(y) + bound) + bound + ref.TINY[dt])[0]
    check("out", out, torch.tensor(want).cuda(), torch.tensor(tol).cuda())
    assert np.array_equal(f(state), before)


@pytest.mark.parametrize("dt,D,N", [("float32", 20, 16), ("bfloat16", 70, 5), ("float16", 7, 33)])
def test_scan_step_with_slots_far_apart(dt, D, N):
    rows, pool = 640, 700
    g = torch.Generator().manual_seed(N)
    rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x, raw, z = (rand(rows, D).to(TYPES[dt]).cuda() for _ in range(3))
    b, c = (rand(rows, 1, N).to(TYPES[dt]).cuda() for _ in range(2))
    a, skip, bias = -(torch.rand(D, N, generator=g) * 3).cuda(), rand(D).cuda(), (rand(D) - 2).cuda()
    state = rand(pool, D, N).cuda()
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    after, slots = f(state), far_slots(rows, pool)
    size = np.abs(after)
    out = torch.full((rows, D), SENTINEL, dtype=x.dtype, device="cuda")
    ssam.ssam_scan_selective_step(x, raw, a, b, c, state, skip=skip, gate=z, dt_bias=bias, softplus=True,
                                  slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), d_out=out)
    want, tol = np.full((rows, D), SENTINEL), np.zeros((rows, D))
    u, d, zz = f(x), ref.softplus(f(raw) + f(bias)), f(z)
    bb, cc = np.repeat(f(b), D, 1), np.repeat(f(c), D, 1)
    e = ref.scan_kappa(10)                           # the slot of every 70th row gets ten rows
    for r, s in enumerate(slots):
        if 0 <= s < pool:
            y, after[s] = ref.scan(u[r:r + 1], d[r:r + 1], f(a), bb[r:r + 1], cc[r:r + 1], f(skip), zz[r:r + 1], after[s])
            m, size[s] = ref.scan(np.abs(u[r:r + 1]), d[r:r + 1], f(a), np.abs(bb[r:r + 1]), np.abs(cc[r:r + 1]), np.abs(f(skip)), None, size[s])
            m = m * np.abs(zz[r] * ref.sigmoid(zz[r])) * (1 + np.abs(zz[r]) / 8)
            want[r], tol[r] = y[0], ref.allowed(y, m, e, dt)[0]
    check("out", out, torch.tensor(want).cuda(), torch.tensor(tol).cuda())
    check("state", state, torch.tensor(after).cuda(), torch.tensor(ref.allowed(after, size, e, "float32")).cuda())


@pytest.mark.parametrize("rows", [1, 7, 600])
@pytest.mark.parametrize("dt", list(TYPES))
def test_steps_without_slots(rows, dt):
    """Row r has slot r: bit for bit what naming them gives."""
    D, N, W = 67, 9, 4
    g = torch.Generator().manual_seed(rows)
    rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x, raw = (rand(rows, D).to(TYPES[dt]).cuda() for _ in range(2))
    b, c = (rand(rows, 1, N).to(TYPES[dt]).cuda() for _ in range(2))
    a, w = -(torch.rand(D, N, generator=g) * 3).cuda(), rand(D, W).to(TYPES[dt]).cuda()
    named = torch.arange(rows, dtype=torch.int32, device="cuda")
    conv_pool, pool = rand(rows + 2, W - 1, D).to(TYPES[dt]).cuda(), rand(rows + 2, D, N).cuda()
    results = []
    for slots in (None, named):
        p, q = conv_pool.clone(), pool.clone()
        results.append([ssam.ssam_conv1d_step(x, w, p, silu=True, slots=slots), p, ssam.ssam_scan_selective_step(x, raw, a, b, c, q, softplus=True, slots=slots), q])
    assert all(torch.equal(u, v) for u, v in zip(*results))
    assert torch.equal(results[0][1][rows:], conv_pool[rows:]) and torch.equal(results[0][3][rows:], pool[rows:])


def test_time_steps():
    """A single state that forgets everything shows the time step: softplus within the (6 + 1.3 |x|) u that the references' bounds count for it
    (and half a step of the result), from time steps of 2e-9 on."""
    x = torch.linspace(-20, 20, 160001, device="cuda")[:, None].contiguous()
    one = torch.ones_like(x)
    got = ssam.ssam_scan_selective(one, x, torch.full((1, 1), float("-inf"), device="cuda"), one[..., None], one[..., None], softplus=True)
    want = torch.logaddexp(x.double(), torch.zeros_like(x, dtype=torch.float64))
    check("softplus", got, want, (6 + 1.3 * x.double().abs() + 1) * ref.U * want)
