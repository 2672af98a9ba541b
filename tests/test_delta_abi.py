"""Host-only checks of the scan with a matrix per head and of the norm: every refusal of the C ABI, the sizes they plan, the structs that
the binding packs and the references' own gradients.  Every call here fails validation, or has nothing to do, before anything is launched."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import delta_reference as ref
import paper_1907_06154_amd as ssam
import paper_1907_06154_amd.sequence as seq
from test_sequence_abi import ALIAS, DIM, ENUM, NULL, OK, ROOT, SHAPE, Rows, Seq, at, call, ci, ll, many, size, struct, sz, vp

cf = ctypes.c_float
HEADS = "dtype heads key_heads key_dim value_dim unit"
Delta = struct("Delta", HEADS, many(cf, "scale"), many(Seq, "seq"), many(Rows, "q k v out g beta"), many(ll, "q_head k_head v_head out_head"),
               many(vp, "state final marks work"), many(sz, "work_bytes"))
DeltaBack = struct("DeltaBack", HEADS, many(cf, "scale"), many(Seq, "seq"), many(Rows, "q k v grad_out g beta"),
                   many(ll, "q_head k_head v_head grad_out_head"), many(vp, "marks grad_final"),
                   many(Rows, "grad_q grad_k grad_v grad_g grad_beta"), many(vp, "grad_state work"), many(sz, "work_bytes"))
DeltaStep = struct("DeltaStep", HEADS, many(cf, "scale"), many(ci, "rows slots"), many(vp, "slot_of"), many(Rows, "q k v out g beta"),
                   many(ll, "q_head k_head v_head out_head"), many(vp, "state"), many(ll, "slot_stride"))
Norm = struct("Norm", "dtype param_dtype channels groups block sequences rows", many(cf, "eps"), many(Rows, "x residual sum gate out"),
              many(vp, "weight scales"))
NormBack = struct("NormBack", "dtype param_dtype channels groups sequences rows", many(cf, "eps"),
                  many(Rows, "x gate grad_out grad_sum grad_in grad_gate"), many(vp, "weight grad_weight work"), many(sz, "work_bytes"))
KINDS = {"ssam_scan_delta_args": Delta, "ssam_scan_delta_backward_args": DeltaBack, "ssam_scan_delta_step_args": DeltaStep,
         "ssam_rms_norm_args": Norm, "ssam_rms_norm_backward_args": NormBack}


@pytest.fixture(scope="module")
def L():
    return seq._load()


def test_the_header_is_c_and_has_these_sizes(tmp_path):
    checks = "".join(f"_Static_assert(sizeof({n}) == {ctypes.sizeof(k)}, \"{n}\");\n" for n, k in KINDS.items())
    for n, k, pairs in (("ssam_scan_delta_args", Delta, "seq:seq q:q d_state:state q_head:q_head work_bytes:work_bytes"),
                        ("ssam_scan_delta_backward_args", DeltaBack, "d_marks:marks grad_q:grad_q d_grad_state:grad_state"),
                        ("ssam_scan_delta_step_args", DeltaStep, "d_slots:slot_of q:q slot_stride:slot_stride"),
                        ("ssam_rms_norm_args", Norm, "in:x gate:gate d_scales:scales"), ("ssam_rms_norm_backward_args", NormBack, "in:x d_work:work")):
        for pair in pairs.split():
            a, b = pair.split(":")
            checks += f"_Static_assert(offsetof({n}, {a}) == {getattr(k, b).offset}, \"{n} {a}\");\n"
    checks += '_Static_assert(SSAM_DELTA_ROWS == 64 && SSAM_MAX_KEY == 256, "");\n'
    (tmp_path / "c.c").write_text('#include "ssam_sequence.h"\n#include <stddef.h>\n' + checks)
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", "-o", str(tmp_path / "c.o"),
                    str(tmp_path / "c.c")], check=True)


def changed(s, change):
    for k, v in change.items():
        setattr(s, k, v)
    return s


def apart(s, rows, plain):
    """Addresses 2^46 bytes apart, for tensors that no card holds."""
    names = rows.split() + plain.split()
    place = {n: (i + 1) << 46 for i, n in enumerate(names)}
    return {n: Rows(place[n], getattr(s, n).batch, getattr(s, n).row) if n in rows.split() else place[n] for n in names}


# 2 sequences of 100 rows, 4 heads that share 2 keys of 32, values of 16; a row of q and k takes 64 elements, one of v and out as many.
COMMON = dict(dtype=3, heads=4, key_heads=2, key_dim=32, value_dim=16, unit=1, scale=0.1)
APART = dict(q_head=32, k_head=32, v_head=16)


def delta(**change):
    s = Delta(seq=Seq(2, 100, None, None), q=Rows(at(0), 6400, 64), k=Rows(at(1), 6400, 64), v=Rows(at(2), 6400, 64), out=Rows(at(3), 6400, 64),
              g=Rows(at(4), 400, 4), beta=Rows(at(5), 400, 4), out_head=16, state=at(6), final=at(7), marks=at(8), work=at(9), work_bytes=1 << 23,
              **COMMON, **APART)
    return changed(s, change)


def shapes(f):
    """What all three refuse."""
    assert f(dtype=1) == ENUM and f(dtype=9) == ENUM
    assert f(heads=0) == SHAPE and f(heads=3) == SHAPE and f(key_heads=0) == SHAPE and f(key_dim=0) == SHAPE and f(key_dim=257) == SHAPE
    assert f(value_dim=0) == SHAPE and f(value_dim=-1) == SHAPE
    assert f(value_dim=(1 << 22) + 1) == DIM and f(heads=1 << 25) == DIM
    for n in ("q_head", "k_head", "v_head"):
        assert f(**{n: -1}) == DIM and f(**{n: 1 << 62}) == DIM, n
    for n in ("q", "k", "v", "beta"):
        assert f(**{n: Rows(None, 0, 0)}) == NULL and f(**{n: Rows(at(0) + 1, 6400, 64)}) == DIM and f(**{n: Rows(at(0), 6400, -1)}) == DIM, n
    for n in ("q", "k", "v", "g", "beta"):      # rows further apart than a tile's offsets reach
        assert f(**{n: Rows(at(30), 1 << 40, (1 << 24) + 1)}) == DIM, n


def test_scan_delta_refusals(L):
    f = lambda **c: call(L, "ssam_scan_delta", delta(**c))  # noqa: E731
    assert L.ssam_scan_delta(None, None) == NULL
    shapes(f)
    assert f(out=Rows(None, 0, 0)) == NULL and f(work=None) == NULL
    assert f(seq=Seq(-1, 100, None, None)) == DIM and f(seq=Seq(2, -1, None, None)) == DIM
    assert f(seq=Seq(2, 100, at(20), None)) == NULL and f(seq=Seq(2, 100, at(20) + 1, at(20) + 5)) == DIM
    assert f(out=Rows(at(3), 6400, 63)) == DIM and f(out=Rows(at(3), 6336, 64)) == DIM      # rows that share elements
    assert f(out_head=15) == DIM and f(out_head=-16) == DIM                                  # heads that do
    assert f(state=at(6) + 2) == DIM and f(final=at(7) + 1) == DIM and f(marks=at(8) + 2) == DIM and f(work=at(9) + 8) == DIM
    need = size(L, "ssam_scan_delta_workspace_bytes", delta())
    assert need > 0 and f(work_bytes=need - 1) == DIM
    for n in ("q", "k", "v"):
        assert f(out=Rows(getattr(delta(), n).d + 128, 6400, 64)) == ALIAS, n
    plane = 2 * 4 * 32 * 16 * 4
    assert f(final=at(6) + 16) == ALIAS and f(state=at(7) + plane - 4) == ALIAS and f(final=at(8)) == ALIAS and f(final=at(9) + need - 4) == ALIAS
    assert f(marks=at(6)) == ALIAS and f(marks=at(4)) == ALIAS and f(work=at(5)) == ALIAS and f(work=at(3)) == ALIAS and f(out=Rows(at(6), 6400, 64)) == ALIAS
    # nothing to do
    assert f(seq=Seq(0, 100, None, None), q=Rows(None, 0, 0), work=None) == OK
    # no launch has so many blocks, no card so much memory
    for s in (Seq(1, 1 << 30, None, None), Seq(1 << 30, 1, None, None)):
        assert f(seq=s, state=None, final=None, marks=None, work_bytes=1 << 62, **apart(delta(), "q k v out g beta", "work")) == DIM


def test_scan_delta_plans(L):
    block = size(L, "ssam_scan_delta_workspace_bytes", delta(seq=Seq(1, 1, None, None), heads=1, key_heads=1))
    assert block > 0 and block % 16 == 0
    for s, slots in ((Seq(1, 64, None, None), 1), (Seq(1, 65, None, None), 2), (Seq(3, 0, None, None), 3), (Seq(7, 129, None, None), 21),
                     (Seq(5, 1000, at(20), at(21)), 20), (Seq(0, 10, None, None), 0)):
        d = delta(seq=s)
        assert size(L, "ssam_scan_delta_workspace_bytes", d) == slots * 4 * block, (s.sequences, s.rows)
        L.ssam_scan_delta_marks.restype = ll
        assert L.ssam_scan_delta_marks(ctypes.cast(ctypes.byref(d), ctypes.c_char_p)) == slots
    assert size(L, "ssam_scan_delta_workspace_bytes", delta(key_dim=300)) == 0
    huge = delta(seq=Seq(1 << 30, 1 << 10, None, None), heads=1 << 20, key_heads=1, value_dim=16)      # saturates, does not wrap
    assert size(L, "ssam_scan_delta_workspace_bytes", huge) >= 1 << 50


def delta_back(**change):
    s = DeltaBack(seq=Seq(2, 100, None, None), q=Rows(at(0), 6400, 64), k=Rows(at(1), 6400, 64), v=Rows(at(2), 6400, 64),
                  grad_out=Rows(at(3), 6400, 64), g=Rows(at(4), 400, 4), beta=Rows(at(5), 400, 4), grad_out_head=16, marks=at(6), grad_final=at(7),
                  grad_q=Rows(at(8), 6400, 64), grad_k=Rows(at(9), 6400, 64), grad_v=Rows(at(10), 6400, 64), grad_g=Rows(at(11), 400, 4),
                  grad_beta=Rows(at(12), 400, 4), grad_state=at(13), work=at(14), work_bytes=1 << 23, **COMMON, **APART)
    return changed(s, change)


def test_scan_delta_backward_refusals(L):
    f = lambda **c: call(L, "ssam_scan_delta_backward", delta_back(**c))  # noqa: E731
    assert L.ssam_scan_delta_backward(None, None) == NULL
    shapes(f)
    assert f(grad_out=Rows(None, 0, 0)) == NULL and f(marks=None) == NULL and f(work=None) == NULL
    assert f(grad_out_head=-1) == DIM and f(grad_out=Rows(at(30), 1 << 40, (1 << 24) + 1)) == DIM
    for n, width in (("grad_q", 64), ("grad_k", 64), ("grad_v", 64), ("grad_g", 4), ("grad_beta", 4)):
        d = getattr(delta_back(), n).d
        assert f(**{n: Rows(d + 1, 100 * width, width)}) == DIM and f(**{n: Rows(d, 100 * width, width - 1)}) == DIM, n
        assert f(**{n: Rows(at(0), 6400, 64)}) == ALIAS and f(**{n: Rows(at(14), 6400, 64)}) == ALIAS, n
    for n in ("marks", "grad_final", "grad_state"):
        assert f(**{n: at(20) + 2}) == DIM, n
    need = size(L, "ssam_scan_delta_backward_workspace_bytes", delta_back())
    assert need > 0 and f(work_bytes=need - 1) == DIM and f(work=at(14) + 4) == DIM
    assert f(grad_state=at(7)) == ALIAS and f(grad_state=at(6)) == ALIAS and f(work=at(6)) == ALIAS and f(grad_q=Rows(at(9) + 64, 6400, 64)) == ALIAS
    assert f(seq=Seq(0, 100, None, None), q=Rows(None, 0, 0), marks=None) == OK
    far = apart(delta_back(), "q k v grad_out g beta grad_q grad_k grad_v grad_g grad_beta", "marks work")
    assert f(seq=Seq(1, 1 << 30, None, None), work_bytes=1 << 62, **far) == DIM
    assert size(L, "ssam_scan_delta_backward_workspace_bytes", delta_back(seq=Seq(1 << 30, 1 << 10, None, None), heads=1 << 20, key_heads=1)) >= 1 << 50


def test_scan_delta_step_refusals(L):
    def make(**change):
        s = DeltaStep(rows=5, slots=7, slot_of=at(6), q=Rows(at(0), 0, 64), k=Rows(at(1), 0, 64), v=Rows(at(2), 0, 64), out=Rows(at(3), 0, 64),
                      g=Rows(at(4), 0, 4), beta=Rows(at(5), 0, 4), out_head=16, state=at(7), slot_stride=2048, **COMMON, **APART)
        return changed(s, change)
    f = lambda **c: call(L, "ssam_scan_delta_step", make(**c))  # noqa: E731
    assert L.ssam_scan_delta_step(None, None) == NULL
    shapes(f)
    assert f(out=Rows(None, 0, 0)) == NULL and f(state=None) == NULL and f(state=at(7) + 2) == DIM and f(slot_stride=2047) == DIM
    assert f(rows=-1) == DIM and f(slots=-1) == DIM and f(slot_of=at(6) + 1) == DIM and f(out=Rows(at(3), 0, 63)) == DIM and f(out_head=8) == DIM
    assert f(state=at(0)) == ALIAS and f(out=Rows(at(7) + 7 * 2048 * 4 - 4, 0, 64)) == ALIAS and f(out=Rows(at(2), 0, 64)) == ALIAS and f(state=at(6)) == ALIAS
    assert f(out=Rows(at(4), 0, 64)) == ALIAS
    assert f(rows=0) == OK and f(rows=0, state=None, q=Rows(None, 0, 0)) == OK


def norm(**change):
    s = Norm(dtype=3, param_dtype=0, channels=128, groups=2, block=32, sequences=2, rows=10, eps=1e-6, x=Rows(at(0), 1280, 128),
             residual=Rows(at(1), 1280, 128), sum=Rows(at(2), 1280, 128), gate=Rows(at(3), 1280, 128), out=Rows(at(4), 1280, 128), weight=at(5), scales=at(6))
    return changed(s, change)


@pytest.mark.parametrize("name", ["ssam_rms_norm", "ssam_rms_norm_e4m3"])
def test_rms_norm_refusals(L, name):
    f = lambda **c: call(L, name, norm(**c))  # noqa: E731
    assert getattr(L, name)(None, None) == NULL
    assert f(dtype=1) == ENUM and f(param_dtype=4) == ENUM
    assert f(channels=0) == DIM and f(channels=(1 << 24) + 2) == DIM and f(sequences=-1) == DIM and f(rows=-1) == DIM
    assert f(groups=0) == SHAPE and f(groups=3) == SHAPE and f(eps=-1e-6) == SHAPE and f(eps=float("nan")) == SHAPE
    assert f(channels=65538) == SHAPE and f(channels=32769, groups=1) == SHAPE                # wider than a block holds
    assert f(x=Rows(None, 0, 0)) == NULL and f(out=Rows(None, 0, 0)) == NULL and f(residual=Rows(None, 0, 0)) == NULL        # a sum of one
    for n in ("x", "residual", "gate", "sum"):
        assert f(**{n: Rows(at(20) + 1, 1280, 128)}) == DIM and f(**{n: Rows(at(20), 1280, -1)}) == DIM, n
    assert f(weight=at(5) + 2) == DIM and f(param_dtype=3, weight=at(5) + 1) == DIM
    assert f(out=Rows(at(4), 1280, 127)) == DIM and f(sum=Rows(at(2), 1270, 128)) == DIM
    for d in (0, 1, 2, 3, 5):
        assert f(out=Rows(at(d), 1280, 128)) == ALIAS, d
    assert f(sum=Rows(at(0), 1280, 128)) == ALIAS and f(sum=Rows(at(3), 1280, 128)) == ALIAS
    assert f(sum=Rows(at(1) + 2, 1280, 128)) == ALIAS and f(sum=Rows(at(1), 2560, 256)) == ALIAS      # the residual's, in other places
    assert f(rows=0) == OK and f(sequences=0, x=Rows(None, 0, 0), out=Rows(None, 0, 0)) == OK


def test_rms_norm_e4m3_refusals(L):
    f = lambda **c: call(L, "ssam_rms_norm_e4m3", norm(**c))  # noqa: E731
    assert f(block=0) == SHAPE and f(block=48) == SHAPE and f(block=8) == SHAPE and f(block=128) == SHAPE
    assert f(scales=None) == NULL and f(scales=at(6) + 2) == DIM and f(scales=at(0)) == ALIAS and f(scales=at(1)) == ALIAS and f(scales=at(4)) == ALIAS
    assert f(rows=0, scales=None) == OK


def test_rms_norm_backward_refusals(L):
    def make(**change):
        s = NormBack(dtype=3, param_dtype=0, channels=128, groups=2, sequences=2, rows=10, eps=1e-6, x=Rows(at(0), 1280, 128), gate=Rows(at(1), 1280, 128),
                     grad_out=Rows(at(2), 1280, 128), grad_sum=Rows(at(3), 1280, 128), grad_in=Rows(at(4), 1280, 128), grad_gate=Rows(at(5), 1280, 128),
                     weight=at(6), grad_weight=at(7), work=at(8), work_bytes=1 << 20)
        return changed(s, change)
    f = lambda **c: call(L, "ssam_rms_norm_backward", make(**c))  # noqa: E731
    assert L.ssam_rms_norm_backward(None, None) == NULL
    assert f(dtype=1) == ENUM and f(param_dtype=4) == ENUM and f(channels=0) == DIM and f(groups=3) == SHAPE and f(eps=-1.0) == SHAPE
    assert f(channels=65538) == SHAPE
    assert f(x=Rows(None, 0, 0)) == NULL and f(grad_out=Rows(None, 0, 0)) == NULL and f(gate=Rows(None, 0, 0)) == NULL and f(work=None) == NULL
    for n in ("x", "gate", "grad_out", "grad_sum", "grad_in", "grad_gate"):
        assert f(**{n: Rows(at(20) + 1, 1280, 128)}) == DIM, n
    for n in ("grad_in", "grad_gate"):
        assert f(**{n: Rows(at(20), 1280, 127)}) == DIM, n
        for d in (0, 1, 2, 3, 6, 8):
            assert f(**{n: Rows(at(d), 1280, 128)}) == ALIAS, (n, d)
    need = size(L, "ssam_rms_norm_backward_workspace_bytes", make())
    assert need > 0 and need % (64 * 4) == 0 and f(work_bytes=need - 1) == DIM and f(work=at(8) + 8) == DIM and f(grad_weight=at(7) + 2) == DIM
    assert f(grad_weight=at(6)) == ALIAS and f(grad_weight=at(8)) == ALIAS
    assert size(L, "ssam_rms_norm_backward_workspace_bytes", make(grad_weight=None)) == 0
    wide = make(channels=32768, groups=1, sequences=1 << 20, rows=1 << 20)
    assert size(L, "ssam_rms_norm_backward_workspace_bytes", wide) == 1024 * 32768 * 4       # a bounded number of partial sums
    assert f(rows=0, grad_weight=None, work=None) == OK


def test_tensors_must_live_on_the_gpu():
    import torch
    x, r = torch.zeros(4, 2, 8), torch.zeros(4, 2)
    for f in (lambda: ssam.ssam_scan_delta(x, x, x, r, r), lambda: ssam.ssam_scan_delta_marks(x, x), lambda: ssam.ssam_rms_norm(x[:, 0]),
              lambda: ssam.ssam_scan_delta_step(x, x, x, r, r, torch.zeros(4, 2, 8, 8)), lambda: ssam.ssam_rms_norm_e4m3(x[:, 0]),
              lambda: ssam.ssam_rms_norm_backward(x[:, 0], x[:, 0]), lambda: ssam.ssam_scan_delta_backward(x, x, x, x, r, r, x)):
        with pytest.raises(ValueError, match="GPU"):
            f()
    with pytest.raises(TypeError, match="tensor"):
        ssam.ssam_rms_norm(None)
    with pytest.raises(TypeError):
        seq._fast.delta(x, x)


def test_the_references_gradients_against_differences():
    """In 64 bits, e = 1e-6: the differences are off by e^2 and 1e-16 / e."""
    rng = np.random.default_rng(3)
    n, H, K, V, e = 7, 2, 3, 4, 1e-6

    def slopes(loss, v):
        for k in v:
            g = np.zeros_like(v[k])
            for i in np.ndindex(*v[k].shape):
                up, down = dict(v), dict(v)
                up[k], down[k] = v[k].copy(), v[k].copy()
                up[k][i] += e
                down[k][i] -= e
                g[i] = (loss(up) - loss(down)) / (2 * e)
            yield k, g

    v = {"q": rng.normal(size=(n, H, K)), "k": rng.normal(size=(n, H, K)), "v": rng.normal(size=(n, H, V)), "g": -rng.uniform(0, 1, (n, H)),
         "beta": rng.uniform(0, 1, (n, H)), "state": rng.normal(size=(H, K, V))}
    r, rl = rng.normal(size=(n, H, V)), rng.normal(size=(H, K, V))

    def loss(v):
        y, last, _ = ref.delta(ref.unit(v["q"]), ref.unit(v["k"]), v["v"], v["g"], v["beta"], 0.7, v["state"])
        return (y * r).sum() + (last * rl).sum()
    q, k = ref.unit(v["q"]), ref.unit(v["k"])
    kept = ref.delta(q, k, v["v"], v["g"], v["beta"], 0.7, v["state"])[2]
    got = ref.delta_back(r, q, k, v["v"], v["g"], v["beta"], 0.7, kept, rl)
    got["q"], got["k"] = ref.through_unit(v["q"], got["q"]), ref.through_unit(v["k"], got["k"])
    for name, g in slopes(loss, v):
        assert np.allclose(g, got[name], atol=1e-7, rtol=1e-6), name

    for gate in (False, True):
        v = {"x": rng.normal(size=(n, 6)), "w": rng.normal(size=3)}
        if gate:
            v["gate"] = rng.normal(size=(n, 6))
        r, rs = rng.normal(size=(n, 6)), rng.normal(size=(n, 6))

        def loss(v):
            y, _ = ref.norm(v["x"], v["w"], v.get("gate"), 2, 1e-3)
            return (y * r).sum() + (v["x"] * rs).sum()
        dx, dw, dgate, *_ = ref.norm_back(r, v["x"], v["w"], v.get("gate"), rs, 2, 1e-3)
        for name, g in slopes(loss, v):
            assert np.allclose(g, {"x": dx, "w": dw, "gate": dgate}[name], atol=1e-7, rtol=1e-6), (gate, name)
