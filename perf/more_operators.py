"""Timed cases of the layer around the sequence operators' second kind of scan: the gated delta rule, whose state is a
matrix per head that every row corrects (along time, its gradients, single tokens), and the root-mean-square norm
that stands before and behind such a layer (with the residual's addition, per head with a gate, with an output in
8 bits, its gradients).

The plain forms below are elementary torch operations in 32 bits; where `own` is true the same inputs go through
the library's entry points.  Rows are tokens.  Widths and lengths are those of the library's sequence operators
(single tokens, 1537 .. 32768 rows, widths to 8192), ragged and odd ones among them.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 64                # rows that the plain form takes together
UNIT_EPS = 1e-6           # under the root where rows of q and k are brought to unit length
NORM_EPS = 1e-6

MAX_DELTA = 8 * 4096 * 32 * 128 * 128         # rows x heads x state of the largest listed prompt
MAX_DELTA_TRAIN = 4 * 2048 * 16 * 128 * 128
MAX_DELTA_STEP = 256 * 32 * 128 * 128
MAX_NORM = 32768 * 4096                       # rows x channels
MAX_NORM_TRAIN = 16384 * 4096
MAX_NORM_E4M3 = 8192 * 8192


def listed():
    return [
        # one conversation, one token: the latency of a call
        {"name": "delta_step_bf16_1x32x128", "op": "delta_step", "dtype": "bf16", "seqs": 1, "key_heads": 16, "heads": 32, "dk": 128, "dv": 128,
         "unit": True},
        # a full serving batch, states in a pool of slots
        {"name": "delta_step_bf16_256x32x128", "op": "delta_step", "dtype": "bf16", "seqs": 256, "key_heads": 16, "heads": 32, "dk": 128,
         "dv": 128, "unit": True},
        # one prompt of ordinary length that goes on from a cached prefix
        {"name": "delta_bf16_1x4096x32x128", "op": "delta", "dtype": "bf16", "seqs": 1, "rows": 4096, "ragged": False, "key_heads": 16,
         "heads": 32, "dk": 128, "dv": 128, "unit": True, "carried": True},
        # many prompts packed one behind the other, heads of odd sizes
        {"name": "delta_f16_8191x6x96x80_ragged", "op": "delta", "dtype": "f16", "seqs": 37, "rows": 8191, "ragged": True, "key_heads": 3,
         "heads": 6, "dk": 96, "dv": 80, "unit": True, "carried": True},
        # a prompt batch that fills the card
        {"name": "delta_bf16_8x4096x32x128", "op": "delta", "dtype": "bf16", "seqs": 8, "rows": 32768, "ragged": False, "key_heads": 16,
         "heads": 32, "dk": 128, "dv": 128, "unit": True, "carried": False},
        # a training step's micro batch
        {"name": "delta_train_bf16_4x2048x16x128", "op": "delta_train", "dtype": "bf16", "seqs": 4, "rows": 8192, "ragged": False,
         "key_heads": 16, "heads": 16, "dk": 128, "dv": 128, "unit": True, "carried": False},
        # packed documents, small model in 32 bits, heads of odd sizes that share their keys
        {"name": "delta_train_f32_1537x3x41x50_ragged", "op": "delta_train", "dtype": "f32", "seqs": 5, "rows": 1537, "ragged": True,
         "key_heads": 1, "heads": 3, "dk": 41, "dv": 50, "unit": False, "carried": False},
        # one conversation, one token: the norm before a layer
        {"name": "norm_bf16_1x4096", "op": "norm", "dtype": "bf16", "rows": 1, "groups": 1, "width": 4096, "residual": True, "gate": False},
        # a prompt batch that fills the card
        {"name": "norm_bf16_32768x4096", "op": "norm", "dtype": "bf16", "rows": 32768, "groups": 1, "width": 4096, "residual": True,
         "gate": False},
        # the norm behind a layer with matrix states: each head by itself, gated, odd sizes
        {"name": "norm_f16_4003x12x100_gated", "op": "norm", "dtype": "f16", "rows": 4003, "groups": 12, "width": 100, "residual": False,
         "gate": True},
        # a training step's micro batch
        {"name": "norm_train_bf16_16384x4096", "op": "norm_train", "dtype": "bf16", "rows": 16384, "groups": 1, "width": 4096,
         "residual": True, "gate": False},
        # before a product in 8 bits, a scale for each 128 channels
        {"name": "norm_e4m3_bf16_8192x8192", "op": "norm_e4m3", "dtype": "bf16", "rows": 8192, "groups": 1, "width": 8192, "residual": True,
         "gate": False, "block": 128},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_delta(rng, op):
    case = {"op": op, "dtype": rng.choices(["bf16", "f16", "f32"], weights=[2, 1, 1])[0]}
    if op == "delta_step":
        case["seqs"] = _log(rng, 1, 512)
    else:
        case["ragged"] = rng.random() < 0.5
        if case["ragged"]:
            case["seqs"], case["rows"] = _log(rng, 1, 64), _log(rng, 64, 32768)
        else:
            case["seqs"] = _log(rng, 1, 16)
            case["rows"] = case["seqs"] * _log(rng, 16, 16384)
        case["carried"] = op == "delta" and rng.random() < 0.5
    case["key_heads"] = _log(rng, 1, 32)
    case["heads"] = case["key_heads"] * rng.choice([1, 1, 2, 3, 4])
    case["dk"] = rng.choice([128, 128, 64, _log(rng, 16, 160), 256])
    case["dv"] = rng.choice([128, 128, 64, _log(rng, 16, 160), 2 * case["dk"]])
    case["unit"] = rng.random() < 0.75
    return case


def _draw_norm(rng, op):
    case = {"op": op, "dtype": rng.choices(["bf16", "f16", "f32"], weights=[2, 1, 1])[0], "rows": _log(rng, 1, 65536)}
    if rng.random() < 0.3:
        case.update(groups=_log(rng, 2, 64), width=rng.choice([64, 128, 128, 256, _log(rng, 16, 512)]), gate=True, residual=False)
    else:
        width = _log(rng, 64, 16384)
        case.update(groups=1, width=width if rng.random() < 0.4 else (width + 63) // 64 * 64, gate=False, residual=rng.random() < 0.75)
    if op == "norm_e4m3":
        case["block"] = rng.choice([b for b in (case["width"], 128, 64) if case["width"] % b == 0])
    return case


def _fits(case):
    op = case["op"]
    if op.startswith("delta"):
        states = case.get("rows", case["seqs"]) * case["heads"] * case["dk"] * case["dv"]
        return states <= {"delta": MAX_DELTA, "delta_train": MAX_DELTA_TRAIN, "delta_step": MAX_DELTA_STEP}[op]
    values = case["rows"] * case["groups"] * case["width"]
    return values <= {"norm": MAX_NORM, "norm_train": MAX_NORM_TRAIN, "norm_e4m3": MAX_NORM_E4M3}[op]


def draw(rng):
    while True:
        op = rng.choices(["delta", "delta_train", "delta_step", "norm", "norm_train", "norm_e4m3"], weights=[25, 20, 12, 18, 15, 10])[0]
        case = _draw_delta(rng, op) if op.startswith("delta") else _draw_norm(rng, op)
        if _fits(case):
            return case


def work(case):
    e, op = SIZE[case["dtype"]], case["op"]
    if op.startswith("delta"):
        S, H, state = case["seqs"], case["heads"], case["dk"] * case["dv"]
        T, keys, values = case.get("rows", S), case["key_heads"] * case["dk"], H * case["dv"]
        nbytes = T * (e * (2 * keys + 2 * values) + 8 * H)
        flops = 7 * T * H * state
        if op == "delta_step" or case["carried"]:
            nbytes += 2 * 4 * S * H * state
        if op == "delta_train":
            nbytes += T * (e * (2 * keys + 2 * values) + 8 * H)
            flops += 15 * T * H * state
        return {"bytes": nbytes, "flops": flops}
    T, D, W = case["rows"], case["groups"] * case["width"], case["width"]
    nbytes, flops = T * D * e * 2 + W * e, 4 * T * D
    if case["residual"]:
        nbytes += 2 * T * D * e
    if case["gate"]:
        nbytes, flops = nbytes + T * D * e, flops + 5 * T * D
    if op == "norm_e4m3":
        nbytes += T * D * (1 - e) + 4 * T * (D // case["block"])
        flops += 3 * T * D
    if op == "norm_train":        # the gradient comes in, the sum's too, and those of the input, the weight and the gate leave
        nbytes += T * D * e * (2 + case["residual"] + case["gate"]) + W * e
        flops += (10 + 8 * case["gate"]) * T * D
    return {"bytes": nbytes, "flops": flops}


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype)


def _lengths(case, seed):
    """First rows of packed sequences and the row behind the last: random lengths, some of them zero; up to three rows
    behind the last sequence belong to none (a buffer rounded up).  Batches: every sequence has as many rows."""
    S, T = case["seqs"], case["rows"]
    if not case["ragged"]:
        return list(range(0, T + 1, T // S))
    g = torch.Generator().manual_seed(seed + 77)
    end = T - int(torch.randint(0, 4, (1,), generator=g))
    return [0] + torch.randint(0, end + 1, (S - 1,), generator=g).sort().values.tolist() + [end]


def _blocks(edges, rows):
    """How the plain form deals sequences out in blocks of rows: the longest first, so that those that have a c-th block come
    first; first block of each, how many have a c-th, the rows of every block and which of them there are."""
    begin, end = torch.tensor(edges[:-1]), torch.tensor(edges[1:])
    order = torch.argsort(end - begin, descending=True, stable=True)
    begin, end = begin[order], end[order]
    many = (end - begin + BLOCK - 1) // BLOCK
    base = torch.cumsum(many, 0) - many
    seq = torch.repeat_interleave(torch.arange(order.numel()), many)
    at = (begin[seq] + (torch.arange(seq.numel()) - base[seq]) * BLOCK)[:, None] + torch.arange(BLOCK)
    live = at < end[seq][:, None]
    active = [int((many > c).sum()) for c in range(int(many.max()) if many.numel() else 0)]
    return {"order": order.cuda(), "base": base.cuda(), "active": active, "rows": at.clamp(max=max(rows - 1, 0)).cuda(), "live": live.cuda()}


def prepare(case, seed):
    """What a layer holds: activations as the products before it leave them (q, k and v, an input and its gate are column
    ranges of one buffer), weights, states, the rows' layout and the buffers for the results."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, op = DTYPE[case["dtype"]], case["op"]
    s = {"op": op}
    if op.startswith("norm"):
        T, D = case["rows"], case["groups"] * case["width"]
        s.update(groups=case["groups"], block=case.get("block"))
        both = _randn(g, T, (2 if case["gate"] else 1) * D, dtype=dt)
        s["x"], s["gate"] = both[:, :D], both[:, D:] if case["gate"] else None
        s["w"] = 1 + _randn(g, case["width"], scale=0.1)
        s["w"] = s["w"].to(dt)
        s["residual"] = _randn(g, T, D, dtype=dt, scale=3.0) if case["residual"] else None
        s["sum"] = torch.empty(T, D, dtype=dt, device="cuda") if case["residual"] else None
        s["out"] = torch.empty(T, D, dtype=torch.float8_e4m3fn if op == "norm_e4m3" else dt, device="cuda")
        if op == "norm_train":
            s["grad"] = _randn(g, T, D, dtype=dt)
            s["grad_sum"] = _randn(g, T, D, dtype=dt) if case["residual"] else None
        return s
    S, Hk, H, dk, dv = case["seqs"], case["key_heads"], case["heads"], case["dk"], case["dv"]
    step = op == "delta_step"
    T = S if step else case["rows"]
    lead = (T,) if step or case["ragged"] else (S, T // S)
    # behind a filter with a SiLU: mostly small values, the larger ones positive, so that rows' keys are alike
    v = torch.randn(*lead, 2 * Hk * dk + H * dv, generator=g, device="cuda")
    v = v * torch.sigmoid(v)
    s.update(unit=case["unit"], scale=dk ** -0.5)
    if not case["unit"]:     # keys that come at unit length
        keys = v[..., :2 * Hk * dk].view(*lead, 2 * Hk, dk)
        keys /= keys.square().sum(-1, keepdim=True).add(UNIT_EPS).sqrt()
    v = v.to(dt)
    s["q"] = v[..., :Hk * dk].unflatten(-1, (Hk, dk))
    s["k"] = v[..., Hk * dk:2 * Hk * dk].unflatten(-1, (Hk, dk))
    s["v"] = v[..., 2 * Hk * dk:].unflatten(-1, (H, dv))
    s["beta"] = torch.sigmoid(_randn(g, *lead, H))
    # rates 1 .. 16 and time steps between 0.001 and 0.1 before the input has its say, as such layers start out
    first = torch.rand(H, generator=g, device="cuda").mul_(math.log(100.0)).sub_(math.log(1000.0)).exp_()
    rates = 1 + 15 * torch.rand(H, generator=g, device="cuda")
    s["g"] = -rates * torch.nn.functional.softplus(_randn(g, *lead, H) + torch.log(torch.expm1(first)))
    s["out"] = torch.zeros(*lead, H, dv, dtype=dt, device="cuda")
    if step:
        pool = S + S // 4 + 1
        s["slots"] = torch.randperm(pool, generator=g, device="cuda")[:S].to(torch.int32)
        s["state"] = _randn(g, pool, H, dk, dv, scale=0.3)
        return s
    s["edges"] = _lengths(case, seed)
    s["starts"] = torch.tensor(s["edges"], dtype=torch.int32, device="cuda") if case["ragged"] else None
    s["blocks"] = _blocks(s["edges"], T)
    if case["carried"]:
        s["state"], s["final"] = _randn(g, S, H, dk, dv, scale=0.3), torch.zeros(S, H, dk, dv, device="cuda")
    if op == "delta_train":
        s["grad"] = _randn(g, *lead, H, dv, dtype=dt)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _unit(x):
    return x / torch.sqrt(x.square().sum(-1, keepdim=True) + UNIT_EPS)


def _in_blocks(s, name):
    """[blocks, heads, BLOCK, ..] in 32 bits, zeros in rows that are not there."""
    x, b = s[name].float(), s["blocks"]
    x = x.reshape(-1, *x.shape[s["v"].dim() - 2:])[b["rows"]]
    live = b["live"].view(*b["live"].shape, *[1] * (x.dim() - 2))
    return torch.where(live, x, 0.0).transpose(1, 2)


def _keys(s, name):
    """q's or k's blocks as the rule takes them, a copy for every head that shares them."""
    x = _in_blocks(s, name)
    return (_unit(x) if s["unit"] else x).repeat_interleave(s["v"].shape[-2] // x.shape[1], 1)


def _delta_blocks(s):
    """What every block's rows have to do with one another, apart from the state: keys, decays and the inverse of the
    triangular system that their corrections solve."""
    q, k, v = _keys(s, "q"), _keys(s, "k"), _in_blocks(s, "v")
    beta, G = _in_blocks(s, "beta"), torch.cumsum(_in_blocks(s, "g"), -1)
    lower = torch.ones(BLOCK, BLOCK, dtype=torch.bool, device="cuda").tril()
    D = torch.exp(torch.where(lower, G[..., :, None] - G[..., None, :], -math.inf))
    A = torch.where(lower.tril(-1), k @ k.transpose(-1, -2).contiguous() * D, 0.0)
    inverse = torch.eye(BLOCK, device="cuda").expand(*A.shape).contiguous()
    M = -beta[..., None] * A
    for i in range(1, BLOCK):
        inverse[..., i, :i] = (M[..., i, None, :i] @ inverse[..., :i, :i])[..., 0, :]
    P = s["scale"] * (q @ k.transpose(-1, -2).contiguous()) * D
    return q, k, v, beta, G, D, A, inverse, P


def _delta(s):
    q, k, v, beta, G, D, A, inverse, P = _delta_blocks(s)
    b = s["blocks"]
    up, total = torch.exp(G)[..., None], torch.exp(G[..., -1])[..., None, None]     # decay from the block's start to a row, over the block
    rest = torch.exp(G[..., -1:] - G)[..., None]                                    # from a row to the block's end
    H, dk, dv = v.shape[1], k.shape[-1], v.shape[-1]
    state = s["state"][b["order"]] if "state" in s else torch.zeros(b["order"].numel(), H, dk, dv, device="cuda")
    starts = torch.zeros(v.shape[0], H, dk, dv, device="cuda") if s["op"] == "delta_train" else None
    out, x_all, u_all = torch.zeros_like(v), torch.zeros_like(v), torch.zeros_like(v)
    kt = (k * rest).transpose(-1, -2).contiguous()
    for c, m in enumerate(b["active"]):
        at = b["base"][:m] + c
        h = state[:m]
        x = v[at] - up[at] * (k[at] @ h)
        u = inverse[at] @ (beta[at][..., None] * x)
        out[at] = s["scale"] * (up[at] * (q[at] @ h)) + P[at] @ u
        if starts is not None:
            starts[at], x_all[at], u_all[at] = h, x, u
        state[:m] = total[at] * h + kt[at] @ u
    rows = _rows(s, out, s["out"])
    if s["op"] == "delta":
        if "state" not in s:
            return rows
        s["final"][b["order"]] = state
        return rows, s["final"]
    return {"out": rows, **_delta_gradients(s, q, k, beta, G, D, A, inverse, P, starts, x_all, u_all)}


def _rows(s, x, like):
    """Blocks [blocks, heads, BLOCK, ..] back in `like`, rows of no sequence left as they are."""
    b = s["blocks"]
    x = x.transpose(1, 2)[b["live"]].to(like.dtype)
    like.view(-1, *x.shape[1:])[b["rows"][b["live"]]] = x
    return like


def _delta_gradients(s, q, k, beta, G, D, A, inverse, P, starts, x, u):
    b, scale = s["blocks"], s["scale"]
    do = _in_blocks(s, "grad")
    H, dk, dv = u.shape[1], k.shape[-1], u.shape[-1]
    up, total, rest = torch.exp(G)[..., None], torch.exp(G[..., -1])[..., None, None], torch.exp(G[..., -1:] - G)[..., None]
    t = lambda a: a.transpose(-1, -2).contiguous()  # noqa: E731
    Pt, inverse_t, qt, kt = t(P), t(inverse), t(q * up * scale), t(k * up)
    dy, behind = torch.zeros_like(u), torch.zeros_like(starts)
    dstate = torch.zeros(b["order"].numel(), H, dk, dv, device="cuda")
    for c in reversed(range(len(b["active"]))):
        m = b["active"][c]
        at = b["base"][:m] + c
        dh = dstate[:m]
        behind[at] = dh
        du = Pt[at] @ do[at] + rest[at] * (k[at] @ dh)
        dy[at] = inverse_t[at] @ du
        dstate[:m] = total[at] * dh + qt[at] @ do[at] - kt[at] @ (beta[at][..., None] * dy[at])
    dx = beta[..., None] * dy
    r = x - A @ u                                     # what a row's correction is beta times of
    dP, dA = scale * (do @ t(u)) * D, torch.where(A != 0, -(dx @ t(u)) * D, 0.0)
    ht, dht = t(starts), t(behind)
    dq = scale * (up * (do @ ht)) + dP @ k
    reads = dA @ k - up * (dx @ ht)
    last = rest * (u @ dht)
    writes = t(dP) @ q + t(dA) @ k + last
    # a row's decay multiplies what it reads and divides what it writes
    dG = (q * dq).sum(-1) + (k * reads).sum(-1) - (k * writes).sum(-1)
    dG[..., -1] += total[..., 0, 0] * (starts * behind).sum((-1, -2)) + (k * last).sum((-1, -2))
    dg = dG.flip(-1).cumsum(-1).flip(-1)
    shared = lambda a: a.unflatten(1, (s["k"].shape[-2], -1)).sum(2)  # noqa: E731
    dq, dk = shared(dq), shared(reads + writes)
    if s["unit"]:
        def through(d, name):
            raw = _in_blocks(s, name)
            size = torch.sqrt(raw.square().sum(-1, keepdim=True) + UNIT_EPS)
            return (d - raw / size * (raw / size * d).sum(-1, keepdim=True)) / size
        dq, dk = through(dq, "q"), through(dk, "k")
    new = lambda a: torch.zeros(a.shape, dtype=a.dtype, device="cuda")  # noqa: E731
    return {"q": _rows(s, dq, new(s["q"])), "k": _rows(s, dk, new(s["k"])), "v": _rows(s, dx, new(s["v"])), "g": _rows(s, dg, new(s["g"])),
            "beta": _rows(s, (dy * r).sum(-1), new(s["beta"]))}


def _delta_step(s):
    at = s["slots"].long()
    q, k, v = (s[n].float() for n in ("q", "k", "v"))
    if s["unit"]:
        q, k = _unit(q), _unit(k)
    many = v.shape[1] // k.shape[1]
    q, k = q.repeat_interleave(many, 1), k.repeat_interleave(many, 1)
    h = torch.exp(s["g"])[..., None, None] * s["state"][at]
    u = s["beta"][..., None] * (v - (k[..., None] * h).sum(-2))
    h = h + k[..., None] * u[..., None, :]
    out = s["out"].copy_(s["scale"] * (q[..., None] * h).sum(-2))
    s["state"][at] = h
    return out, s["state"]


def _silu(x):
    return x * torch.sigmoid(x)


def _norm(s):
    G, x = s["groups"], s["x"]
    if s["residual"] is not None:
        x = s["sum"].copy_(x.float() + s["residual"].float())
    x = x.float().unflatten(-1, (G, -1))
    w = s["w"].float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + NORM_EPS)
    y = x * r * w
    gate = s["gate"].float().unflatten(-1, (G, -1)) if s["gate"] is not None else None
    z = (y * _silu(gate) if gate is not None else y).flatten(-2)
    if s["op"] == "norm_e4m3":
        z = z.unflatten(-1, (-1, s["block"]))
        most = z.abs().amax(-1, keepdim=True)
        scales = torch.where(most > 0, most / 448.0, 1.0)
        out = s["out"].copy_((z / scales).flatten(-2))
        return (out, scales[..., 0]) + ((s["sum"],) if s["sum"] is not None else ())
    out = s["out"].copy_(z)
    if s["op"] == "norm":
        return (out, s["sum"]) if s["sum"] is not None else out
    dz, dgate, to = s["grad"].float().unflatten(-1, (G, -1)), None, s["x"].dtype
    dy = dz
    if gate is not None:
        sig = torch.sigmoid(gate)
        dy, dgate = dz * gate * sig, (dz * y * sig * (1 + gate * (1 - sig))).flatten(-2).to(to)
    dw = (dy * x * r).sum((0, 1)).to(s["w"].dtype)
    a = dy * w * r
    dx = (a - x * (r * r) * (a * x).mean(-1, keepdim=True)).flatten(-2)
    if s["grad_sum"] is not None:
        dx = dx + s["grad_sum"].float()
    return {"out": out, "sum": s["sum"], "x": dx.to(to), "weight": dw, "gate": dgate}


# ---- the library's -----------------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_1907_06154_amd as ssam
    op = s["op"]
    if op.startswith("norm"):
        layer = dict(d_residual=s["residual"], d_sum=s["sum"], gate=s["gate"], groups=s["groups"], eps=NORM_EPS)
        if op == "norm_e4m3":
            got = ssam.ssam_rms_norm_e4m3(s["x"], s["w"], block=s["block"], d_out=s["out"], **layer)
            return (got.values, got.scales) + ((s["sum"],) if s["sum"] is not None else ())
        out = ssam.ssam_rms_norm(s["x"], s["w"], d_out=s["out"], **layer)
        if op == "norm":
            return (out, s["sum"]) if s["sum"] is not None else out
        grads = ssam.ssam_rms_norm_backward(s["grad"], s["x"] if s["sum"] is None else s["sum"], s["w"], d_grad_sum=s["grad_sum"], gate=s["gate"],
                                            groups=s["groups"], eps=NORM_EPS)
        return {"out": out, "sum": s["sum"], "x": grads.x, "weight": grads.weight, "gate": grads.gate}
    layer = (s["q"], s["k"], s["v"], s["g"], s["beta"])
    how = dict(scale=s["scale"], unit=s["unit"])
    if op == "delta_step":
        return ssam.ssam_scan_delta_step(*layer, s["state"], slots=s["slots"], d_out=s["out"], **how), s["state"]
    how["starts"] = s["starts"]
    if op == "delta":
        state, final = s.get("state"), s.get("final")
        out = ssam.ssam_scan_delta(*layer, d_state=state, d_final=final, d_out=s["out"], **how)
        return out if final is None else (out, final)
    marks = ssam.ssam_scan_delta_marks(s["k"], s["v"], starts=s["starts"])
    out = ssam.ssam_scan_delta(*layer, d_marks=marks, d_out=s["out"], **how)
    grads = ssam.ssam_scan_delta_backward(s["grad"], *layer, marks, **how)
    return {"out": out, "q": grads.q, "k": grads.k, "v": grads.v, "g": grads.g, "beta": grads.beta}


def run(state):
    if own:
        return _run_own(state)
    if state["op"].startswith("norm"):
        return _norm(state)
    return _delta_step(state) if state["op"] == "delta_step" else _delta(state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _exact_delta(case, s):
    """Row after row, all sequences and heads side by side, the longest sequences first; the way back makes the states of `block`
    rows at a time again."""
    H, dk, dv, S = case["heads"], case["dk"], case["dv"], case["seqs"]
    spans = sorted(zip(s["edges"], s["edges"][1:], range(S)), key=lambda e: e[0] - e[1])
    counts, begin = [e - b for b, e, _ in spans], torch.tensor([b for b, _, _ in spans], device="cuda")
    order = torch.tensor([i for _, _, i in spans], device="cuda")
    longest, rows, train = counts[0], case["rows"], s["op"] == "delta_train"
    if train and longest > 16384:
        return None
    flat = {n: s[n].reshape(rows, *s[n].shape[s["v"].dim() - 2:]) for n in ("q", "k", "v", "g", "beta", "grad") if n in s}
    many = H // case["key_heads"]
    new = lambda n: torch.zeros(flat[n].shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = new("v")

    def row(t):
        live = sum(n > t for n in counts)
        at = begin[:live] + t
        r = {n: f[at].double() for n, f in flat.items()}
        for n in ("q", "k"):
            r["size " + n] = torch.sqrt(torch.linalg.vecdot(r[n], r[n])[..., None] + UNIT_EPS)
            if case["unit"]:
                r[n] = r[n] / r["size " + n]
            r[n] = r[n].repeat_interleave(many, 1)
        return r, live, at

    def forward(r, h):
        h = h * torch.exp(r["g"])[..., None, None]
        miss = r["v"] - torch.einsum("shkv,shk->shv", h, r["k"])
        return h, miss, h + torch.einsum("shk,shv->shkv", r["k"], r["beta"][..., None] * miss)

    state = s["state"][order].double() if "state" in s else torch.zeros(S, H, dk, dv, dtype=torch.float64, device="cuda")
    block, kept = 64, []
    for t in range(longest):
        if train and t % block == 0:
            kept.append(state.clone())
        r, live, at = row(t)
        h = forward(r, state[:live])[2]
        state[:live] = h
        out[at] = s["scale"] * torch.einsum("shkv,shk->shv", h, r["q"])
    out = out.view(s["out"].shape)
    if not train:
        return (out, state[torch.argsort(order)]) if "state" in s else out
    grads = {n: new(n) for n in ("q", "k", "v", "g", "beta")}
    dstate = torch.zeros(S, H, dk, dv, dtype=torch.float64, device="cuda")
    for t0 in reversed(range(0, longest, block)):
        state, seen = kept.pop(), []
        for t in range(t0, min(longest, t0 + block)):
            r, live, at = row(t)
            decayed, miss, h = forward(r, state[:live])
            state[:live] = h
            seen.append((r, live, at, decayed, miss, h))
        for r, live, at, decayed, miss, h in reversed(seen):
            d = dstate[:live] + s["scale"] * torch.einsum("shk,shv->shkv", r["q"], r["grad"])
            dq = s["scale"] * torch.einsum("shkv,shv->shk", h, r["grad"])
            du = torch.einsum("shkv,shk->shv", d, r["k"])
            dmiss = r["beta"][..., None] * du
            dkeys = torch.einsum("shkv,shv->shk", d, r["beta"][..., None] * miss) - torch.einsum("shkv,shv->shk", decayed, dmiss)
            d = d - torch.einsum("shk,shv->shkv", r["k"], dmiss)
            grads["g"][at] = (d * decayed).sum((-1, -2))
            grads["beta"][at] = (du * miss).sum(-1)
            grads["v"][at] = dmiss
            for n, v in (("q", dq), ("k", dkeys)):
                v = v.unflatten(1, (-1, many)).sum(2)
                if case["unit"]:
                    e = flat[n][at].double() / r["size " + n]
                    v = (v - e * (e * v).sum(-1, keepdim=True)) / r["size " + n]
                grads[n][at] = v
            dstate[:live] = d * torch.exp(r["g"])[..., None, None]
    return {"out": out, **{n: v.view(s[n].shape) for n, v in grads.items()}}


def _exact_delta_step(case, s):
    at, many = s["slots"].long(), case["heads"] // case["key_heads"]
    q, k = (torch.repeat_interleave(s[n].double(), many, 1) for n in ("q", "k"))
    if case["unit"]:
        q, k = (e / torch.sqrt(torch.einsum("shk,shk->sh", e, e) + UNIT_EPS)[..., None] for e in (q, k))
    state = s["state"].double()
    h = torch.einsum("shkv,sh->shkv", state[at], torch.exp(s["g"].double()))
    u = torch.einsum("sh,shv->shv", s["beta"].double(), s["v"].double() - torch.einsum("shkv,shk->shv", h, k))
    h = h + torch.einsum("shk,shv->shkv", k, u)
    state[at] = h
    return s["scale"] * torch.einsum("shkv,shk->shv", h, q), state


def _exact_norm(case, s):
    """The norm is that of the sum as its type holds it, so that the sum is all that the way back needs."""
    T, G, W, op = case["rows"], case["groups"], case["width"], case["op"]
    x = s["x"].double()
    total = None
    if case["residual"]:
        total = (x + s["residual"].double()).to(s["x"].dtype)
        x = total.double()
    x, w = x.reshape(T, G, W), s["w"].double()
    size = torch.sqrt((x * x).sum(-1, keepdim=True) / W + NORM_EPS)
    y = x / size * w
    z = s["gate"].double().reshape(T, G, W) if case["gate"] else None
    e = y if z is None else y * z / (1 + torch.exp(-z))
    if op == "norm_e4m3":
        e = e.reshape(T, -1, case["block"])
        most = e.abs().amax(-1)
        scales = torch.where(most > 0, most / 448, torch.ones_like(most))
        values = (e / scales[..., None]).reshape(T, G * W).to(torch.float8_e4m3fn)
        return (values, scales) + ((total.double(),) if total is not None else ())
    out = e.reshape(T, G * W)
    if op == "norm":
        return (out, total.double()) if total is not None else out
    d = s["grad"].double().reshape(T, G, W)
    dgate = None
    if z is not None:
        sig = 1 / (1 + torch.exp(-z))
        dgate = (d * y * (sig + z * sig * (1 - sig))).reshape(T, G * W)
        d = d * z * sig
    dw = torch.einsum("tgw,tgw->w", d, x / size)
    d = d * w
    dx = d / size - x * torch.einsum("tgw,tgw->tg", d, x)[..., None] / (W * size ** 3)
    dx = dx.reshape(T, G * W)
    if case["residual"]:
        dx = dx + s["grad_sum"].double()
    return {"out": out, "sum": None if total is None else total.double(), "x": dx, "weight": dw, "gate": dgate}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(case, s)
    return _exact_delta_step(case, s) if case["op"] == "delta_step" else _exact_delta(case, s)
