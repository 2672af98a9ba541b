"""Timed cases of the sequence operators: the per-channel filter along time with carried state, the scan whose
terms decay by learned, input-dependent factors (a state space layer's), their gradients, and both for single
tokens with the states of many sequences in slots.

The plain forms below are elementary torch operations in 32 bits; where `own` is true the same inputs go through
the library's entry points.  Rows are tokens, channels lie side by side.  Widths and lengths are those of the
library's image and volume cases (512 .. 8192), ragged and odd ones, and single tokens.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}

MAX_CONV_VALUES = 32768 * 8192           # rows x channels of the largest listed filter
MAX_CONV_TRAIN_VALUES = 8 * 2048 * 4096
MAX_SCAN_STATES = 8 * 4096 * 4096 * 16   # rows x channels x states of the largest listed scan
MAX_TRAIN_STATES = 4 * 2048 * 2048 * 16
MAX_STEP_VALUES = 384 * 8192
MAX_STEP_STATES = 256 * 4096 * 16


def listed():
    return [
        # one conversation, one token: the latency of a call
        {"name": "conv1d_step_bf16_1x2048", "op": "conv1d_step", "dtype": "bf16", "seqs": 1, "channels": 2048, "taps": 4, "silu": True},
        # a full serving batch of a wide model, states in a pool of slots
        {"name": "conv1d_step_bf16_384x8192", "op": "conv1d_step", "dtype": "bf16", "seqs": 384, "channels": 8192, "taps": 4, "silu": True},
        # a few short prompts packed one behind the other, odd width
        {"name": "conv1d_f16_4003x1001_ragged", "op": "conv1d", "dtype": "f16", "seqs": 7, "rows": 4003, "ragged": True, "channels": 1001,
         "taps": 3, "silu": False, "carried": True},
        # a long document of a wide model
        {"name": "conv1d_bf16_32768x8192", "op": "conv1d", "dtype": "bf16", "seqs": 1, "rows": 32768, "ragged": False, "channels": 8192,
         "taps": 4, "silu": True, "carried": True},
        # a training step's micro batch
        {"name": "conv1d_train_bf16_8x2048x4096", "op": "conv1d_train", "dtype": "bf16", "seqs": 8, "rows": 16384, "ragged": False,
         "channels": 4096, "taps": 4, "silu": True, "carried": False},
        # one conversation, one token
        {"name": "scan_step_bf16_1x2048x16", "op": "scan_step", "dtype": "bf16", "seqs": 1, "channels": 2048, "states": 16, "groups": 1,
         "gate": True},
        # a full serving batch
        {"name": "scan_step_bf16_256x4096x16", "op": "scan_step", "dtype": "bf16", "seqs": 256, "channels": 4096, "states": 16, "groups": 1,
         "gate": True},
        # one prompt of ordinary length
        {"name": "scan_bf16_1x4096x4096x16", "op": "scan", "dtype": "bf16", "seqs": 1, "rows": 4096, "ragged": False, "channels": 4096,
         "states": 16, "groups": 1, "gate": True, "carried": True},
        # many prompts packed one behind the other, two groups of odd width
        {"name": "scan_f16_8191x2050x8_ragged", "op": "scan", "dtype": "f16", "seqs": 37, "rows": 8191, "ragged": True, "channels": 2050,
         "states": 8, "groups": 2, "gate": True, "carried": True},
        # a prompt batch that fills the card
        {"name": "scan_bf16_8x4096x4096x16", "op": "scan", "dtype": "bf16", "seqs": 8, "rows": 32768, "ragged": False, "channels": 4096,
         "states": 16, "groups": 1, "gate": True, "carried": False},
        # a training step's micro batch
        {"name": "scan_train_bf16_4x2048x2048x16", "op": "scan_train", "dtype": "bf16", "seqs": 4, "rows": 8192, "ragged": False,
         "channels": 2048, "states": 16, "groups": 1, "gate": True, "carried": False},
        # packed documents, small model in 32 bits, odd sizes, three groups
        {"name": "scan_train_f32_1537x513x32_ragged", "op": "scan_train", "dtype": "f32", "seqs": 5, "rows": 1537, "ragged": True,
         "channels": 513, "states": 32, "groups": 3, "gate": False, "carried": False},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Channels: half of them as they fall, half a multiple of 64."""
    v = _log(rng, lo, hi)
    return min(hi, max(64, (v + 32) // 64 * 64)) if rng.random() < 0.5 else v


def _draw(rng):
    op = rng.choices(["conv1d", "conv1d_train", "conv1d_step", "scan", "scan_train", "scan_step"], weights=[15, 15, 10, 25, 25, 10])[0]
    case = {"op": op, "dtype": rng.choices(["bf16", "f16", "f32"], weights=[2, 1, 1])[0]}
    if op.endswith("step"):
        case["seqs"] = _log(rng, 1, 512)
    else:
        case["ragged"] = rng.random() < 0.5
        if case["ragged"]:
            case["seqs"], case["rows"] = _log(rng, 1, 64), _log(rng, 64, 32768)
        else:
            case["seqs"] = _log(rng, 1, 16)
            case["rows"] = case["seqs"] * _log(rng, 16, 32768)
        case["carried"] = not op.endswith("train") and rng.random() < 0.5
    if op.startswith("conv1d"):
        case.update(channels=_width(rng, 128, 8192), taps=rng.choice([2, 3, 4, 4, 4, 5, 6, 8]), silu=rng.random() < 0.7)
    else:
        groups = rng.choice([1, 1, 1, 2, 4])
        case.update(channels=groups * _width(rng, 96, 8192 // groups), groups=groups, states=rng.choice([16, 16, 16, 4, 8, 13, 32, 64]),
                    gate=rng.random() < 0.7)
    return case


def _fits(case):
    op, values = case["op"], case["channels"] * case.get("rows", case["seqs"])
    if op == "conv1d":
        return values <= MAX_CONV_VALUES
    if op == "conv1d_train":
        return values <= MAX_CONV_TRAIN_VALUES
    if op == "conv1d_step":
        return values <= MAX_STEP_VALUES
    if op == "scan":
        return values * case["states"] <= MAX_SCAN_STATES
    if op == "scan_train":
        return values * case["states"] <= MAX_TRAIN_STATES
    return values * case["states"] <= MAX_STEP_STATES


def draw(rng):
    while True:
        case = _draw(rng)
        if _fits(case):
            return case


def work(case):
    e, D, S = SIZE[case["dtype"]], case["channels"], case["seqs"]
    T = case.get("rows", S)
    conv, step, train = case["op"].startswith("conv1d"), case["op"].endswith("step"), case["op"].endswith("train")
    if conv:
        W = case["taps"]
        nbytes = 2 * e * T * D + e * D * (W + 1)
        flops = T * D * (2 * W + (8 if case["silu"] else 0))
        if step or case["carried"]:
            nbytes += 2 * e * S * (W - 1) * D
        if train:
            nbytes += 2 * e * T * D + e * D * (W + 1)
            flops += T * D * (4 * W + (10 if case["silu"] else 0))
        return {"bytes": nbytes, "flops": flops}
    N, G, gate = case["states"], case["groups"], 1 if case["gate"] else 0
    nbytes = e * T * (D * (3 + gate) + 2 * G * N) + 4 * D * (N + 2)
    flops = T * D * (7 * N + 12 + 6 * gate)
    if step or case["carried"]:
        nbytes += 2 * 4 * S * D * N
    if train:
        nbytes += e * T * (D * (3 + gate) + 2 * G * N) + 4 * D * (N + 2)
        flops += T * D * (16 * N + 14 + 12 * gate)
    return {"bytes": nbytes, "flops": flops}


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype)


def _starts(case, seed):
    """First rows of packed sequences, and the row behind the last: random lengths, some of them zero; up to three
    rows behind the last sequence belong to none (a buffer rounded up)."""
    g = torch.Generator().manual_seed(seed + 77)
    end = case["rows"] - int(torch.randint(0, 4, (1,), generator=g))
    inner = torch.randint(0, end + 1, (case["seqs"] - 1,), generator=g).sort().values
    return torch.cat([torch.zeros(1, dtype=torch.int64), inner, torch.tensor([end])]).to(torch.int32).cuda()


def prepare(case, seed):
    """What a layer holds: activations as the products before it leave them (the filter's input and the gate are halves
    of one, the scan's B and C slices of another), weights, states, the rows' layout and the buffers for the results."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, D, S, op = DTYPE[case["dtype"]], case["channels"], case["seqs"], case["op"]
    step, train = op.endswith("step"), op.endswith("train")
    T = case.get("rows", S)
    lead = (T,) if step or case["ragged"] else (S, T // S)
    s = {"op": op, "starts": _starts(case, seed) if not step and case["ragged"] else None}
    xz = _randn(g, *lead, 2 * D, dtype=dt)
    s["x"], s["out"] = xz[..., :D], torch.zeros(*lead, D, dtype=dt, device="cuda")
    if train:
        s["grad"] = _randn(g, *lead, D, dtype=dt)
    if step:
        pool = S + S // 4 + 1
        s["slots"] = torch.randperm(pool, generator=g, device="cuda")[:S].to(torch.int32)
    if op.startswith("conv1d"):
        W = case["taps"]
        s["silu"] = case["silu"]
        s["w"], s["b"] = _randn(g, D, W, dtype=dt, scale=1 / math.sqrt(W)), _randn(g, D, dtype=dt, scale=0.1)
        if step:
            s["state"] = _randn(g, pool, W - 1, D, dtype=dt)
        elif case["carried"]:
            s["state"], s["final"] = _randn(g, S, W - 1, D, dtype=dt), torch.zeros(S, W - 1, D, dtype=dt, device="cuda")
        return s
    N, G = case["states"], case["groups"]
    rank = max(1, D // 32)
    proj = _randn(g, *lead, rank + 2 * G * N, dtype=dt)
    s["bb"] = proj[..., rank:rank + G * N].unflatten(-1, (G, N))
    s["cc"] = proj[..., rank + G * N:].unflatten(-1, (G, N))
    s["z"] = xz[..., D:] if case["gate"] else None
    s["dt"] = _randn(g, *lead, D, dtype=dt, scale=0.5)
    # time steps between 0.001 and 0.1 before the input has its say, decay rates 1 .. N, as such layers start out
    first = torch.rand(D, generator=g, device="cuda").mul_(math.log(100.0)).sub_(math.log(1000.0)).exp_()
    s["dt_bias"] = first + torch.log(-torch.expm1(-first))
    s["a"] = -(torch.arange(1, N + 1, device="cuda") * (1 + 0.1 * torch.rand(D, N, generator=g, device="cuda")))
    s["skip"] = 1 + _randn(g, D, scale=0.1)
    if step:
        s["state"] = _randn(g, pool, D, N, scale=0.5)
    elif case["carried"]:
        s["state"], s["final"] = _randn(g, S, D, N, scale=0.5), torch.zeros(S, D, N, device="cuda")
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _layout(s):
    """Of the rows laid flat: first rows, lengths, the sequence of each row, which rows start one, which belong to one."""
    lead = s["x"].shape[:-1]
    rows = math.prod(lead)
    if s["starts"] is not None:
        edges = s["starts"].long()
    else:
        edges = torch.arange(0, rows + 1, lead[-1], device="cuda")
    begin, count = edges[:-1], edges[1:] - edges[:-1]
    t = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(edges[1:].contiguous(), t, right=True).clamp(max=begin.numel() - 1)
    valid = t < edges[-1]
    return begin, count, seq, (t == begin[seq]) & valid, valid


def _conv_rows(s, x, begin, seq):
    """[rows, taps, channels]: the inputs under the taps of every row."""
    rows, D = x.shape
    W = s["w"].shape[1]
    src = torch.arange(rows, device="cuda")[:, None] + torch.arange(1 - W, 1, device="cuda")
    off = src - begin[seq][:, None]
    before = s["state"].float().reshape(-1, D) if "state" in s else torch.zeros(begin.numel() * (W - 1), D, device="cuda")
    return torch.cat([before, x])[torch.where(off >= 0, src + before.shape[0], seq[:, None] * (W - 1) + off + W - 1)]


def _silu(p, silu):
    return p * torch.sigmoid(p) if silu else p


def _conv1d(s):
    begin, count, seq, _, valid = _layout(s)
    D = s["x"].shape[-1]
    x, w, b = s["x"].float().reshape(-1, D), s["w"].float(), s["b"].float()
    W = w.shape[1]
    under = _conv_rows(s, x, begin, seq)
    p = (under * w.t()).sum(1) + b
    y = torch.where(valid[:, None], _silu(p, s["silu"]), 0.0).to(s["out"].dtype)
    out = s["out"].copy_(y.view(s["out"].shape))
    if s["op"] == "conv1d":
        if "state" not in s:
            return out
        src = (begin + count)[:, None] + torch.arange(1 - W, 0, device="cuda")
        off = src - begin[:, None]
        rows = torch.cat([s["state"].reshape(-1, D), s["x"].reshape(-1, D)])
        at = torch.arange(begin.numel(), device="cuda")[:, None] * (W - 1) + off + W - 1
        s["final"].copy_(rows[torch.where(off >= 0, src + s["state"].shape[0] * (W - 1), at)])
        return out, s["final"]
    dy = torch.where(valid[:, None], s["grad"].float().reshape(-1, D), 0.0)
    sig = torch.sigmoid(p)
    q = dy * (sig * (1 + p * (1 - sig))) if s["silu"] else dy
    t = torch.arange(x.shape[0], device="cuda")[:, None] + torch.arange(W, device="cuda")
    inside = (t < (begin + count)[seq][:, None]) & valid[:, None]
    later = q[t.clamp(max=x.shape[0] - 1)] * inside[:, :, None]
    dx = (later * w.t().flip(0)).sum(1)
    dw = (q[:, None, :] * torch.where(valid[:, None, None], under, 0.0)).sum(0).t()
    return out, dx.to(s["x"].dtype).view(s["x"].shape), dw.to(s["w"].dtype), q.sum(0).to(s["b"].dtype)


def _conv1d_step(s):
    at = s["slots"].long()
    rows = torch.cat([s["state"][at].float(), s["x"].float()[:, None]], 1)
    p = (rows * s["w"].float().t()).sum(1) + s["b"].float()
    out = s["out"].copy_(_silu(p, s["silu"]))
    s["state"][at] = rows[:, 1:].to(s["state"].dtype)
    return out, s["state"]


def _decayed_sums(a, x):
    """h_t = a_t h_{t-1} + x_t along the first axis, by doubling."""
    k = 1
    while k < x.shape[0]:
        x = torch.cat([x[:k], torch.addcmul(x[k:], a[k:], x[:-k])])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return x


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _scan(s):
    begin, count, seq, first, valid = _layout(s)
    rows, D = seq.numel(), s["x"].shape[-1]
    G, N = s["bb"].shape[-2:]
    wide = (rows, G, D // G)
    u, raw = s["x"].float().reshape(wide), s["dt"].float().reshape(wide) + s["dt_bias"].view(G, -1)
    bb, cc = s["bb"].float().reshape(rows, G, 1, N), s["cc"].float().reshape(rows, G, 1, N)
    A, skip = s["a"].view(G, -1, N), s["skip"].view(G, -1)
    d = _softplus(raw)
    a = torch.exp(d[..., None] * A)
    x = (d * u)[..., None] * bb
    if "state" in s:
        at, some = begin.clamp(max=rows - 1), (count > 0)[:, None, None, None]
        x = x.index_add(0, at, a[at] * s["state"].view(-1, G, D // G, N) * some)
    keep = (~first & valid)[:, None, None, None]
    h = _decayed_sums(torch.where(keep, a, 0.0), x)
    y = (h * cc).sum(-1) + skip * u
    z = s["z"].float().reshape(wide) if s["z"] is not None else None
    gated = y * _silu(z, True) if z is not None else y
    gated = torch.where(valid[:, None, None], gated, 0.0)
    out = s["out"].copy_(gated.reshape(s["out"].shape))
    if s["op"] == "scan":
        if "state" not in s:
            return out
        last = h[(begin + count - 1).clamp(min=0)].view(-1, D, N)
        s["final"].copy_(torch.where((count > 0)[:, None, None], last, s["state"]))
        return out, s["final"]
    dout = torch.where(valid[:, None, None], s["grad"].float().reshape(wide), 0.0)
    dz, dy = None, dout
    if z is not None:
        sig = torch.sigmoid(z)
        dy = dout * z * sig
        dz = (dout * y * sig * (1 + z * (1 - sig))).to(s["z"].dtype).reshape(s["z"].shape)
    behind = torch.cat([torch.where(keep, a, 0.0)[1:], torch.zeros_like(a[:1])])
    g = _decayed_sums(behind.flip(0), (cc * dy[..., None]).flip(0)).flip(0)
    q = g * (h - x)
    gb = (g * bb).sum(-1)
    du = skip * dy + d * gb
    ddt = torch.where(valid[:, None, None], ((A * q).sum(-1) + u * gb) * torch.sigmoid(raw), 0.0)
    live = valid[:, None, None]
    to = s["x"].dtype
    shape = s["x"].shape
    return {"out": out, "x": du.to(to).view(shape), "dt": ddt.to(to).view(shape), "z": dz,
            "b": (g * (d * u)[..., None]).sum(2).to(to).view(s["bb"].shape),
            "c": (h * dy[..., None]).sum(2).to(to).view(s["cc"].shape),
            "a": torch.where(live[..., None], q * d[..., None], 0.0).sum(0).view(D, N), "skip": (dy * u).sum(0).view(D),
            "dt_bias": ddt.sum(0).view(D)}


def _scan_step(s):
    at = s["slots"].long()
    S, D = s["x"].shape
    G, N = s["bb"].shape[-2:]
    u, raw = s["x"].float().view(S, G, -1), (s["dt"].float() + s["dt_bias"]).view(S, G, -1)
    d = _softplus(raw)
    h = s["state"][at].view(S, G, -1, N)
    h = torch.exp(d[..., None] * s["a"].view(G, -1, N)) * h + (d * u)[..., None] * s["bb"].float()[:, :, None]
    y = (h * s["cc"].float()[:, :, None]).sum(-1) + s["skip"].view(G, -1) * u
    if s["z"] is not None:
        y = y * _silu(s["z"].float().view(S, G, -1), True)
    out = s["out"].copy_(y.view(S, D))
    s["state"][at] = h.view(S, D, N)
    return out, s["state"]


# ---- the library's -----------------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_1907_06154_amd as ssam
    op = s["op"]
    if op == "conv1d_step":
        return ssam.ssam_conv1d_step(s["x"], s["w"], s["state"], bias=s["b"], silu=s["silu"], slots=s["slots"], d_out=s["out"]), s["state"]
    if op == "scan_step":
        out = ssam.ssam_scan_selective_step(s["x"], s["dt"], s["a"], s["bb"], s["cc"], s["state"], skip=s["skip"], gate=s["z"],
                                            dt_bias=s["dt_bias"], softplus=True, slots=s["slots"], d_out=s["out"])
        return out, s["state"]
    if op.startswith("conv1d"):
        state, final = s.get("state"), s.get("final")
        out = ssam.ssam_conv1d(s["x"], s["w"], bias=s["b"], silu=s["silu"], d_state=state, d_final=final, starts=s["starts"], d_out=s["out"])
        if op == "conv1d":
            return out if final is None else (out, final)
        grads = ssam.ssam_conv1d_backward(s["grad"], s["x"], s["w"], bias=s["b"], silu=s["silu"], starts=s["starts"])
        return out, grads.x, grads.weight, grads.bias
    layer = dict(skip=s["skip"], gate=s["z"], dt_bias=s["dt_bias"], softplus=True, starts=s["starts"])
    if op == "scan":
        state, final = s.get("state"), s.get("final")
        out = ssam.ssam_scan_selective(s["x"], s["dt"], s["a"], s["bb"], s["cc"], d_state=state, d_final=final, d_out=s["out"], **layer)
        return out if final is None else (out, final)
    marks = ssam.ssam_scan_selective_marks(s["x"], s["a"], starts=s["starts"])
    out = ssam.ssam_scan_selective(s["x"], s["dt"], s["a"], s["bb"], s["cc"], d_marks=marks, d_out=s["out"], **layer)
    grads = ssam.ssam_scan_selective_backward(s["grad"], s["x"], s["dt"], s["a"], s["bb"], s["cc"], marks, **layer)
    return {"out": out, "x": grads.x, "dt": grads.dt, "z": grads.gate, "b": grads.b, "c": grads.c, "a": grads.a, "skip": grads.skip,
            "dt_bias": grads.dt_bias}


def run(state):
    if own:
        return _run_own(state)
    op = state["op"]
    if op == "conv1d_step":
        return _conv1d_step(state)
    if op == "scan_step":
        return _scan_step(state)
    return _conv1d(state) if op.startswith("conv1d") else _scan(state)


# ---- the definitions in 64 bits, sequence by sequence ------------------------------------------------------------------

def _spans(s):
    lead = s["x"].shape[:-1]
    if s["starts"] is not None:
        edges = s["starts"].tolist()
    else:
        edges = list(range(0, math.prod(lead) + 1, lead[-1]))
    return [(b, e) for b, e in zip(edges, edges[1:])]


def _flat(t, keep):
    return t.double().reshape(-1, *t.shape[t.dim() - keep:])


def _exact_conv1d(case, s):
    D, W = case["channels"], case["taps"]
    w, b = s["w"].double(), s["b"].double()
    if case["op"] == "conv1d_step":
        at = s["slots"].long()
        p = b + w[:, -1] * s["x"].double()
        for j in range(W - 1):
            p = p + w[:, j] * s["state"][at, j].double()
        state = s["state"].double()
        state[at] = torch.cat([state[at, 1:], s["x"].double()[:, None]], 1)
        return p / (1 + torch.exp(-p)) if case["silu"] else p, state
    x = _flat(s["x"], 1)
    out, dx = torch.zeros_like(x), torch.zeros_like(x)
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    finals = []
    for i, (lo, hi) in enumerate(_spans(s)):
        before = s["state"][i].double() if "state" in s else torch.zeros(W - 1, D, dtype=torch.float64, device="cuda")
        rows = torch.cat([before, x[lo:hi]])
        n = hi - lo
        finals.append(rows[n:])
        p = b.repeat(n, 1)
        for j in range(W):
            p.addcmul_(rows[j:j + n], w[:, j])
        sig = 1 / (1 + torch.exp(-p))
        out[lo:hi] = p * sig if case["silu"] else p
        if case["op"] == "conv1d_train":
            q = _flat(s["grad"], 1)[lo:hi]
            if case["silu"]:
                q = q * (sig + p * sig * (1 - sig))
            db += q.sum(0)
            drows = torch.zeros_like(rows)
            for j in range(W):
                dw[:, j] += (q * rows[j:j + n]).sum(0)
                drows[j:j + n].addcmul_(q, w[:, j])
            dx[lo:hi] = drows[W - 1:]
    out = out.view(s["out"].shape)
    if case["op"] == "conv1d_train":
        return out, dx.view(s["x"].shape), dw, db
    return (out, torch.stack(finals)) if "state" in s else out


def _exact_scan(case, s):
    """Row after row.  Sequences run side by side, `block` rows of theirs at a time; the way back goes over the blocks in
    reverse and makes their states again from the block's first."""
    D, N, G, S = case["channels"], case["states"], case["groups"], case["seqs"]
    spans = _spans(s)
    begin = torch.tensor([lo for lo, _ in spans], device="cuda")
    count = torch.tensor([hi - lo for lo, hi in spans], device="cuda")
    longest = max(hi - lo for lo, hi in spans)
    rows = _flat(s["x"], 1).shape[0]
    A, skip = s["a"].double(), s["skip"].double()
    train = case["op"] == "scan_train"
    block = max(1, min(64, (1 << 27) // (S * D * N)))
    names = {"x": 1, "dt": 1, "bb": 2, "cc": 2, "z": 1, "grad": 1}
    flat = {k: s[k].reshape(rows, *s[k].shape[s[k].dim() - v:]) for k, v in names.items() if s.get(k) is not None}
    out = torch.zeros(rows, D, dtype=torch.float64, device="cuda")

    def load(t0):
        t = torch.arange(t0, min(longest, t0 + block), device="cuda")
        live = t[:, None] < count
        at = (begin + t[:, None]).clamp(max=rows - 1)
        v = {k: f[at].double() for k, f in flat.items()}
        v["bb"], v["cc"] = (v[k].repeat_interleave(D // G, 2) for k in ("bb", "cc"))
        v["raw"] = v["dt"] + s["dt_bias"].double()
        v["d"] = torch.logaddexp(v["raw"], torch.zeros_like(v["raw"])) * live[..., None]   # past a sequence's end nothing changes
        v["decay"], v["in"] = torch.exp(v["d"][..., None] * A), (v["d"] * v["x"])[..., None] * v["bb"]
        return v, live, at

    def forward(v, h):
        hs = torch.empty_like(v["in"])
        for k in range(hs.shape[0]):
            h = torch.addcmul(v["in"][k], v["decay"][k], h)
            hs[k] = h
        return hs

    h = s["state"].double() if "state" in s else torch.zeros(S, D, N, dtype=torch.float64, device="cuda")
    at_block = []
    for t0 in range(0, longest, block):
        v, live, at = load(t0)
        if train:
            at_block.append(h)
        hs = forward(v, h)
        h = hs[-1]
        y = (hs * v["cc"]).sum(-1) + skip * v["x"]
        if "z" in v:
            y = y * v["z"] / (1 + torch.exp(-v["z"]))
        out[at[live]] = y[live]
    out = out.view(s["out"].shape)
    if not train:
        return (out, h) if "state" in s else out
    grads = {k: torch.zeros(flat[k].shape, dtype=torch.float64, device="cuda") for k in ("x", "dt", "bb", "cc", "z") if k in flat}
    dA, dskip, dbias = torch.zeros_like(A), torch.zeros_like(skip), torch.zeros_like(skip)
    carry = torch.zeros(S, D, N, dtype=torch.float64, device="cuda")     # decay and gradient of the row behind, multiplied
    for i in reversed(range(len(at_block))):
        v, live, at = load(i * block)
        hs = forward(v, at_block[i])
        old = torch.cat([at_block[i][None], hs[:-1]])
        dout = v["grad"] * live[..., None]
        dy = dout
        if "z" in v:
            sig = 1 / (1 + torch.exp(-v["z"]))
            dy = dout * v["z"] * sig
            dz = dout * ((hs * v["cc"]).sum(-1) + skip * v["x"]) * (sig + v["z"] * sig * (1 - sig))
            grads["z"][at[live]] = dz[live]
        gs = v["cc"] * dy[..., None]
        for k in reversed(range(gs.shape[0])):
            gs[k] += carry
            carry = v["decay"][k] * gs[k]
        q = gs * v["decay"] * old
        gb = (gs * v["bb"]).sum(-1)
        ddt = ((q * A).sum(-1) + v["x"] * gb) / (1 + torch.exp(-v["raw"])) * live[..., None]
        grads["x"][at[live]] = (skip * dy + v["d"] * gb)[live]
        grads["dt"][at[live]] = ddt[live]
        grads["bb"][at[live]] = (gs * (v["d"] * v["x"])[..., None]).unflatten(2, (G, D // G)).sum(3)[live]
        grads["cc"][at[live]] = (hs * dy[..., None]).unflatten(2, (G, D // G)).sum(3)[live]
        dA += (q * v["d"][..., None]).sum((0, 1))
        dskip += (dy * v["x"]).sum((0, 1))
        dbias += ddt.sum((0, 1))
    return {"out": out, "x": grads["x"].view(s["x"].shape), "dt": grads["dt"].view(s["x"].shape),
            "z": grads["z"].view(s["z"].shape) if "z" in grads else None, "b": grads["bb"].view(s["bb"].shape),
            "c": grads["cc"].view(s["cc"].shape), "a": dA, "skip": dskip, "dt_bias": dbias}


def _exact_scan_step(case, s):
    G, D, at = case["groups"], case["channels"], s["slots"].long()
    x, raw = s["x"].double(), s["dt"].double() + s["dt_bias"].double()
    d = torch.logaddexp(raw, torch.zeros_like(raw))
    bb, cc = (s[k].double().repeat_interleave(D // G, 1) for k in ("bb", "cc"))
    state = s["state"].double()
    h = torch.exp(d[..., None] * s["a"].double()) * state[at] + (d * x)[..., None] * bb
    y = (h * cc).sum(-1) + s["skip"].double() * x
    if s["z"] is not None:
        y = y * s["z"].double() / (1 + torch.exp(-s["z"].double()))
    state[at] = h
    return y, state


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("conv1d"):
        return _exact_conv1d(case, s)
    return _exact_scan_step(case, s) if case["op"] == "scan_step" else _exact_scan(case, s)
