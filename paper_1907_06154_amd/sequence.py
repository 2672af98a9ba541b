"""Binding of the sequence operators (include/ssam_sequence.h): per-channel filters and selective scans along time,
their gradients and their single-row forms.  Argument checks and marshalling only, as in binding.py.

Tensors of rows are [rows, channels] (one sequence, or several packed one behind the other: `starts`, a device tensor of
sequences + 1 offsets) or [sequences, rows, channels] (`lengths`: how many rows of each count).  Rows and sequences may have
any stride, channels are contiguous.  A result that is allocated here holds zeros in rows that belong to no sequence; one that
is passed in keeps what it held there.  The kernels run on the device of their tensors, on its current stream or on `stream`.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple, Optional

from . import binding
from .binding import _check, _stream_ptr

SSAM_F16, SSAM_BF16 = 2, 3
MARK_ROWS = 16
MAX_TAPS, MAX_STATES = 8, 64

EXPORTS = ["ssam_conv1d", "ssam_conv1d_backward", "ssam_conv1d_backward_workspace_bytes", "ssam_conv1d_step", "ssam_scan_selective",
           "ssam_scan_selective_workspace_bytes", "ssam_scan_selective_marks", "ssam_scan_selective_backward",
           "ssam_scan_selective_backward_workspace_bytes", "ssam_scan_selective_step"]

# The C structs, field by field ("0q": padding up to 8 bytes).
_SEQ, _ROWS = "2i2P", "P2q"
_CONV1D = struct.Struct("@5i0q" + _SEQ + 2 * _ROWS + "4P0q")
_CONV1D_BACK = struct.Struct("@5i0q" + _SEQ + 3 * _ROWS + "8PN0q")
_CONV1D_STEP = struct.Struct("@7i0qP" + 2 * _ROWS + "3Pq0q")
_SCAN = struct.Struct("@5i0q" + _SEQ + 6 * _ROWS + "2q7PN0q")
_SCAN_BACK = struct.Struct("@5i0q" + _SEQ + 6 * _ROWS + "2q5P" + 5 * _ROWS + "5PN0q")
_SCAN_STEP = struct.Struct("@7i0qP" + 6 * _ROWS + "2q4Pq0q")

_NONE = (0, 0, 0)
_codes = None
_lib = None


class Conv1dGrads(NamedTuple):
    x: object
    weight: object
    bias: Optional[object]
    state: Optional[object]


class ScanSelectiveGrads(NamedTuple):
    x: object
    dt: object
    a: object
    b: object
    c: object
    skip: Optional[object]
    gate: Optional[object]
    dt_bias: Optional[object]
    state: Optional[object]


def _load():
    global _lib, _codes
    if _lib is None:
        import torch
        L = binding.lib()
        for name in EXPORTS:
            f = getattr(L, name)
            f.argtypes = [ctypes.c_char_p] if name.endswith(("bytes", "marks")) else [ctypes.c_char_p, ctypes.c_void_p]
            f.restype = ctypes.c_size_t if name.endswith("bytes") else ctypes.c_longlong if name.endswith("marks") else ctypes.c_int
        _codes = {torch.float32: 0, torch.float16: SSAM_F16, torch.bfloat16: SSAM_BF16}
        _lib = L
    return _lib


def _code(t, name: str) -> int:
    try:
        return _codes[t.dtype]
    except KeyError:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}") from None


def _call(name: str, args: bytes, t, stream) -> None:
    """The entry point on t's device, whichever device is current."""
    import torch
    f = getattr(_lib, name)
    index = t.device.index
    if torch.cuda.device_count() < 2 or index == torch.cuda.current_device():
        _check(f(args, _stream_ptr(stream)), name)
        return
    with torch.cuda.device(index):
        _check(f(args, _stream_ptr(stream)), name)


def _fail(name: str, what: str):
    raise ValueError(f"{name} {what}")


def _main(t, name: str):
    """The tensor the others are measured by: its leading extents and channels."""
    if not t.is_cuda:
        _fail(name, "must live in GPU memory")
    if t.dim() not in (2, 3):
        _fail(name, "must be [rows, channels] or [sequences, rows, channels]")
    return t.shape


def _rows(t, name: str, like, shape):
    """(address, batch stride, row stride) of a tensor of rows: like's element type and device, this shape, contiguous channels."""
    if t is None:
        return _NONE
    if t.shape != shape:
        _fail(name, f"must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype != like.dtype or t.device != like.device:
        _fail(name, f"must be {like.dtype} on {like.device}")
    s = t.stride()
    if s[-1] != 1 and shape[-1] != 1:
        _fail(name, "must have contiguous channels (stride 1)")
    return (t.data_ptr(), 0, s[0]) if len(s) == 2 else (t.data_ptr(), s[0], s[1])


def _group_rows(t, name: str, like, lead):
    """The same for [.., groups, states], and the stride from group to group."""
    if t.dtype != like.dtype or t.device != like.device:
        _fail(name, f"must be {like.dtype} on {like.device}")
    if t.dim() != len(lead) + 2 or t.shape[:-2] != lead:
        _fail(name, f"must have shape {tuple(lead)} + (groups, states), not {tuple(t.shape)}")
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] != 1:
        _fail(name, "must have contiguous states (stride 1)")
    return ((t.data_ptr(), 0, s[0]) if len(s) == 3 else (t.data_ptr(), s[0], s[1])), s[-2]


def _dense(t, name: str, like, dtype, shape) -> int:
    if t is None:
        return 0
    if t.shape != shape:
        _fail(name, f"must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype != dtype or t.device != like.device:
        _fail(name, f"must be {dtype} on {like.device}")
    if not t.is_contiguous():
        _fail(name, "must be contiguous")
    return t.data_ptr()


def _sequences(lead, like, starts, lengths):
    """ssam_sequences of a call: (sequences, rows, begin, end)."""
    if starts is not None and lengths is not None:
        _fail("starts", "and lengths exclude one another")
    if len(lead) == 1:
        if lengths is not None:
            _fail("lengths", "belongs to [sequences, rows, channels]")
        if starts is None:
            return 1, lead[0], 0, 0
        if starts.dim() != 1 or starts.numel() < 1 or not starts.is_contiguous():
            _fail("starts", "must be a contiguous 1D tensor of sequences + 1 offsets")
        _offsets(starts, "starts", like)
        p = starts.data_ptr()
        return starts.numel() - 1, lead[0], p, p + 4
    if starts is not None:
        _fail("starts", "belongs to packed [rows, channels]")
    if lengths is None:
        return lead[0], lead[1], 0, 0
    if lengths.shape != (lead[0],) or not lengths.is_contiguous():
        _fail("lengths", f"must be a contiguous 1D tensor of {lead[0]} lengths")
    _offsets(lengths, "lengths", like)
    return lead[0], lead[1], 0, lengths.data_ptr()


def _offsets(t, name: str, like):
    import torch
    if t.dtype != torch.int32 or t.device != like.device:
        _fail(name, f"must be torch.int32 on {like.device}")


def _new_rows(like, shape, ragged: bool):
    import torch
    return (torch.zeros if ragged else torch.empty)(shape, dtype=like.dtype, device=like.device)


def _workspace(nbytes: int, given, like, stream):
    """(tensor to keep, address, bytes)."""
    import torch
    if given is not None:
        if given.device != like.device or not given.is_contiguous():
            _fail("d_work", f"must be contiguous on {like.device}")
        return given, given.data_ptr(), given.numel() * given.element_size()
    if not nbytes:
        return None, 0, 0
    w = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    if stream is not None:
        w.record_stream(stream)      # it dies when the call returns, while kernels that use it are queued on `stream`
    return w, w.data_ptr(), nbytes


def _filter(d_in, weight, bias):
    """Element types, channels and taps of a filter's parameters, checked, and their addresses."""
    code = _code(d_in, "d_in")
    channels = d_in.shape[-1]
    if weight.dim() != 2 or weight.shape[0] != channels:
        _fail("weight", f"must have shape ({channels}, taps), not {tuple(weight.shape)}")
    if weight.dtype != d_in.dtype and _codes.get(weight.dtype) != 0:
        _fail("weight", f"must be {d_in.dtype} or torch.float32")
    w = _dense(weight, "weight", d_in, weight.dtype, weight.shape)
    b = _dense(bias, "bias", d_in, weight.dtype, (channels,))
    return code, _codes[weight.dtype], channels, weight.shape[1], w, b


def ssam_conv1d(d_in, weight, bias=None, silu: bool = False, d_state=None, d_final=None, starts=None, lengths=None, d_out=None, stream=None):
    """Per-channel causal filter along time: out[t] = f(bias + sum_j weight[:, j] * in[t - taps + 1 + j]), f the SiLU or nothing.
    weight [channels, taps], bias [channels]: d_in's type or float32.  d_state, d_final: [sequences, taps - 1, channels], the rows
    before each sequence's first (zeros without) and its last ones afterwards (may be the same tensor)."""
    L = _load()
    shape = _main(d_in, "d_in")
    code, pcode, channels, taps, w, b = _filter(d_in, weight, bias)
    seq = _sequences(shape[:-1], d_in, starts, lengths)
    if d_out is None:
        d_out = _new_rows(d_in, shape, starts is not None or lengths is not None)
    carried = (seq[0], taps - 1, channels)
    args = _CONV1D.pack(code, pcode, channels, taps, bool(silu), *seq, *_rows(d_in, "d_in", d_in, shape), *_rows(d_out, "d_out", d_in, shape), w, b,
                        _dense(d_state, "d_state", d_in, d_in.dtype, carried), _dense(d_final, "d_final", d_in, d_in.dtype, carried))
    _call("ssam_conv1d", args, d_in, stream)
    return d_out


def ssam_conv1d_backward(d_grad, d_in, weight, bias=None, silu: bool = False, d_state=None, d_grad_final=None, starts=None, lengths=None,
                         state_grad: bool = False, d_work=None, stream=None) -> Conv1dGrads:
    """Gradients of ssam_conv1d for d_grad, the gradient of its result, and d_grad_final, that of its d_final (none if absent).
    weight's and bias's come in their own type; state_grad: that of d_state (or of the zeros in its place) too."""
    import torch
    L = _load()
    shape = _main(d_in, "d_in")
    code, pcode, channels, taps, w, b = _filter(d_in, weight, bias)
    seq = _sequences(shape[:-1], d_in, starts, lengths)
    carried = (seq[0], taps - 1, channels)
    gx = _new_rows(d_in, shape, starts is not None or lengths is not None)
    gw = torch.empty_like(weight)
    gb = torch.empty_like(bias) if bias is not None else None
    gs = torch.empty(carried, dtype=d_in.dtype, device=d_in.device) if state_grad else None
    head = (code, pcode, channels, taps, bool(silu), *seq, *_rows(d_in, "d_in", d_in, shape), *_rows(d_grad, "d_grad", d_in, shape),
            *_rows(gx, "x", d_in, shape), w, b, _dense(d_state, "d_state", d_in, d_in.dtype, carried),
            _dense(d_grad_final, "d_grad_final", d_in, d_in.dtype, carried), gw.data_ptr(), gb.data_ptr() if gb is not None else 0,
            gs.data_ptr() if gs is not None else 0)
    need = L.ssam_conv1d_backward_workspace_bytes(_CONV1D_BACK.pack(*head, 0, 0))
    keep, wp, wb = _workspace(need, d_work, d_in, stream)
    _call("ssam_conv1d_backward", _CONV1D_BACK.pack(*head, wp, wb), d_in, stream)
    return Conv1dGrads(gx, gw, gb, gs)


def _slot_args(d_in, rows: int, slots, pool: int, stride: int):
    if slots is None:
        if pool < rows:
            _fail("d_state", f"must have a slot for each of {rows} rows")
        return 0
    if slots.shape != (rows,) or not slots.is_contiguous():
        _fail("slots", f"must be a contiguous 1D tensor of {rows} slots")
    _offsets(slots, "slots", d_in)
    return slots.data_ptr()


def _pool(t, name: str, like, dtype, shape):
    """[slots, *shape]: address, slots and elements from slot to slot."""
    if t.dim() != 1 + len(shape) or t.shape[1:] != shape:
        _fail(name, f"must have shape (slots,) + {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype != dtype or t.device != like.device:
        _fail(name, f"must be {dtype} on {like.device}")
    n = 1
    for extent, step in zip(reversed(shape), reversed(t.stride()[1:])):
        if extent != 1 and step != n:
            _fail(name, "must have contiguous slots")
        n *= extent
    stride = t.stride()[0] if t.shape[0] > 1 else n
    if stride < n:
        _fail(name, "must have slots of its own (no overlap)")
    return t.data_ptr(), t.shape[0], stride


def ssam_conv1d_step(d_in, weight, d_state, bias=None, silu: bool = False, slots=None, d_out=None, stream=None):
    """ssam_conv1d for one more row of each of d_in's [rows, channels] sequences.  d_state [pool, taps - 1, channels], in d_in's
    type, is updated in place; slots (int32, device) names each row's slot of it (row r: slot r without).  A row whose slot is
    outside the pool (-1, say) is passed over; rows of one slot are taken in order."""
    _load()
    shape = _main(d_in, "d_in")
    if len(shape) != 2:
        _fail("d_in", "must be [rows, channels]")
    code, pcode, channels, taps, w, b = _filter(d_in, weight, bias)
    sp, pool, stride = _pool(d_state, "d_state", d_in, d_in.dtype, (taps - 1, channels))
    at = _slot_args(d_in, shape[0], slots, pool, stride)
    if d_out is None:
        d_out = _new_rows(d_in, shape, slots is not None)
    args = _CONV1D_STEP.pack(code, pcode, channels, taps, bool(silu), shape[0], pool, at, *_rows(d_in, "d_in", d_in, shape),
                             *_rows(d_out, "d_out", d_in, shape), w, b, sp, stride)
    _call("ssam_conv1d_step", args, d_in, stream)
    return d_out


def _scan_inputs(d_in, shape, d_dt, a, b, c, skip, gate, dt_bias):
    """What the three scan calls have in common, checked: (type and sizes), (rows), (group strides), (addresses of the parameters)."""
    import torch
    f32 = torch.float32
    channels = shape[-1]
    if a.dim() != 2 or a.shape[0] != channels:
        _fail("a", f"must have shape ({channels}, states), not {tuple(a.shape)}")
    ap = _dense(a, "a", d_in, f32, a.shape)
    br, bg = _group_rows(b, "b", d_in, shape[:-1])
    cr, cg = _group_rows(c, "c", d_in, shape[:-1])
    groups, states = b.shape[-2:]
    if c.shape != b.shape or states != a.shape[1]:
        _fail("c", f"and b must have as many groups as one another and {a.shape[1]} states")
    rows = (*_rows(d_in, "d_in", d_in, shape), *_rows(d_dt, "d_dt", d_in, shape), *_rows(gate, "gate", d_in, shape))
    return ((_code(d_in, "d_in"), channels, states, groups), rows, (*br, *cr), (bg, cg),
            (ap, _dense(skip, "skip", d_in, f32, (channels,)), _dense(dt_bias, "dt_bias", d_in, f32, (channels,))))


def ssam_scan_selective_marks(d_in, a, starts=None, lengths=None):
    """A tensor for ssam_scan_selective's d_marks: the states before every 16th row, for ssam_scan_selective_backward."""
    import torch
    L = _load()
    shape = _main(d_in, "d_in")
    channels, states = a.shape
    seq = _sequences(shape[:-1], d_in, starts, lengths)
    n = L.ssam_scan_selective_marks(_SCAN.pack(_code(d_in, "d_in"), channels, states, 1, 0, *seq, *(_NONE * 6), 0, 0, *(0,) * 8))
    return torch.empty((n, channels, states), dtype=torch.float32, device=d_in.device)


def ssam_scan_selective(d_in, d_dt, a, b, c, skip=None, gate=None, dt_bias=None, softplus: bool = False, d_state=None, d_final=None,
                        d_marks=None, starts=None, lengths=None, d_out=None, d_work=None, stream=None):
    """h_t = exp(d_t a) h_{t-1} + d_t in_t b_t,  out_t = (c_t . h_t + skip in_t) * silu(gate_t),  with d = dt + dt_bias, through a
    softplus or as it is.  d_in, d_dt, gate: rows of channels; b, c: rows of [groups, states], channel k using group
    k // (channels // groups); a [channels, states], skip, dt_bias [channels], d_state, d_final [sequences, channels, states]: float32.
    d_final may be d_state.  d_marks (from ssam_scan_selective_marks) keeps what the gradients need."""
    import torch
    L = _load()
    shape = _main(d_in, "d_in")
    sizes, rows, bc, apart, params = _scan_inputs(d_in, shape, d_dt, a, b, c, skip, gate, dt_bias)
    seq = _sequences(shape[:-1], d_in, starts, lengths)
    if d_out is None:
        d_out = _new_rows(d_in, shape, starts is not None or lengths is not None)
    f32, carried = torch.float32, (seq[0], *a.shape)
    if d_marks is not None and (d_marks.dim() != 3 or d_marks.shape[1:] != a.shape):
        _fail("d_marks", "must come from ssam_scan_selective_marks")
    head = (*sizes, bool(softplus), *seq, *rows, *_rows(d_out, "d_out", d_in, shape), *bc, *apart, *params,
            _dense(d_state, "d_state", d_in, f32, carried), _dense(d_final, "d_final", d_in, f32, carried),
            _dense(d_marks, "d_marks", d_in, f32, d_marks.shape) if d_marks is not None else 0)
    query = _SCAN.pack(*head, 0, 0)
    if d_marks is not None and d_marks.shape[0] < L.ssam_scan_selective_marks(query):
        _fail("d_marks", "must come from ssam_scan_selective_marks for these sequences")
    keep, wp, wb = _workspace(L.ssam_scan_selective_workspace_bytes(query), d_work, d_in, stream)
    _call("ssam_scan_selective", _SCAN.pack(*head, wp, wb), d_in, stream)
    return d_out


def ssam_scan_selective_workspace_bytes(d_in, a, groups: int = 1, starts=None, lengths=None) -> int:
    """Bytes of d_work that ssam_scan_selective needs for such inputs."""
    L = _load()
    shape = _main(d_in, "d_in")
    seq = _sequences(shape[:-1], d_in, starts, lengths)
    return L.ssam_scan_selective_workspace_bytes(
        _SCAN.pack(_code(d_in, "d_in"), *a.shape, groups, 0, *seq, *(_NONE * 6), 0, 0, *(0,) * 8))


def ssam_scan_selective_backward(d_grad, d_in, d_dt, a, b, c, d_marks, skip=None, gate=None, dt_bias=None, softplus: bool = False,
                                 d_grad_final=None, starts=None, lengths=None, state_grad: bool = False, d_work=None,
                                 stream=None) -> ScanSelectiveGrads:
    """Gradients of ssam_scan_selective for d_grad, the gradient of its result, and d_grad_final, that of its d_final (none if absent),
    from the marks the forward call left.  Rows' gradients come in d_in's type, the parameters' in float32; state_grad: that of
    d_state (or of the zeros in its place) too."""
    import torch
    L = _load()
    shape = _main(d_in, "d_in")
    sizes, rows, bc, apart, params = _scan_inputs(d_in, shape, d_dt, a, b, c, skip, gate, dt_bias)
    seq = _sequences(shape[:-1], d_in, starts, lengths)
    ragged = starts is not None or lengths is not None
    f32, carried = torch.float32, (seq[0], *a.shape)
    if d_marks.dim() != 3 or d_marks.shape[1:] != a.shape:
        _fail("d_marks", "must come from ssam_scan_selective_marks")
    gx, gdt = _new_rows(d_in, shape, ragged), _new_rows(d_in, shape, ragged)
    gz = _new_rows(d_in, shape, ragged) if gate is not None else None
    gb, gc = _new_rows(d_in, b.shape, ragged), _new_rows(d_in, c.shape, ragged)
    ga = torch.empty_like(a)
    gk = torch.empty_like(skip) if skip is not None else None
    gd = torch.empty_like(dt_bias) if dt_bias is not None else None
    gs = torch.empty(carried, dtype=f32, device=d_in.device) if state_grad else None
    head = (*sizes, bool(softplus), *seq, *rows, *bc, *_rows(d_grad, "d_grad", d_in, shape), *apart, *params,
            _dense(d_marks, "d_marks", d_in, f32, d_marks.shape), _dense(d_grad_final, "d_grad_final", d_in, f32, carried),
            *_rows(gx, "x", d_in, shape), *_rows(gdt, "dt", d_in, shape), *_rows(gz, "gate", d_in, shape),
            *_group_rows(gb, "b", d_in, shape[:-1])[0], *_group_rows(gc, "c", d_in, shape[:-1])[0], ga.data_ptr(),
            gk.data_ptr() if gk is not None else 0, gd.data_ptr() if gd is not None else 0, gs.data_ptr() if gs is not None else 0)
    query = _SCAN_BACK.pack(*head, 0, 0)
    if d_marks.shape[0] < L.ssam_scan_selective_marks(_SCAN.pack(*sizes, 0, *seq, *(_NONE * 6), 0, 0, *(0,) * 8)):
        _fail("d_marks", "must come from ssam_scan_selective_marks for these sequences")
    keep, wp, wb = _workspace(L.ssam_scan_selective_backward_workspace_bytes(query), d_work, d_in, stream)
    _call("ssam_scan_selective_backward", _SCAN_BACK.pack(*head, wp, wb), d_in, stream)
    return ScanSelectiveGrads(gx, gdt, ga, gb, gc, gk, gz, gd, gs)


def ssam_scan_selective_step(d_in, d_dt, a, b, c, d_state, skip=None, gate=None, dt_bias=None, softplus: bool = False, slots=None, d_out=None,
                             stream=None):
    """ssam_scan_selective for one more row of each of d_in's [rows, channels] sequences; d_state [pool, channels, states], float32,
    is updated in place, slots as in ssam_conv1d_step."""
    import torch
    _load()
    shape = _main(d_in, "d_in")
    if len(shape) != 2:
        _fail("d_in", "must be [rows, channels]")
    sizes, rows, bc, apart, params = _scan_inputs(d_in, shape, d_dt, a, b, c, skip, gate, dt_bias)
    sp, pool, stride = _pool(d_state, "d_state", d_in, torch.float32, a.shape)
    at = _slot_args(d_in, shape[0], slots, pool, stride)
    if d_out is None:
        d_out = _new_rows(d_in, shape, slots is not None)
    args = _SCAN_STEP.pack(*sizes, bool(softplus), shape[0], pool, at, *rows, *_rows(d_out, "d_out", d_in, shape), *bc, *apart, *params, sp, stride)
    _call("ssam_scan_selective_step", args, d_in, stream)
    return d_out
