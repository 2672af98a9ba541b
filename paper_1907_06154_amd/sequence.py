"""Binding of the sequence operators (include/ssam_sequence.h): per-channel filters and selective scans along time, scans with a
matrix per head for a state, their gradients and their single-row forms, and the norm around them.  The extension module _sequence checks and marshals the arguments; there is no
fallback, as in binding.py.

Tensors of rows are [rows, channels] (one sequence, or several packed one behind the other: `starts`, a device tensor of
sequences + 1 offsets) or [sequences, rows, channels] (`lengths`: how many rows of each count).  Rows and sequences may have
any stride, channels are contiguous.  A result that is allocated here holds zeros in rows that belong to no sequence; one that
is passed in keeps what it held there.  The kernels run on the device of their tensors, on its current stream or on `stream`;
what a call allocates belongs to that stream, which orders its first use and its reuse.

The calls are not recorded by autograd: results never require gradients, whatever their inputs do.  Gradients come from the
`*_backward` calls, which a torch.autograd.Function's backward makes; d_final, d_state and pools are written in place unseen by it.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from . import binding

MARK_ROWS = 16
MAX_TAPS, MAX_STATES = 8, 64
DELTA_ROWS, MAX_KEY = 64, 256

EXPORTS = ["ssam_conv1d", "ssam_conv1d_backward", "ssam_conv1d_backward_workspace_bytes", "ssam_conv1d_step", "ssam_scan_selective",
           "ssam_scan_selective_workspace_bytes", "ssam_scan_selective_marks", "ssam_scan_selective_backward",
           "ssam_scan_selective_backward_workspace_bytes", "ssam_scan_selective_step", "ssam_scan_delta", "ssam_scan_delta_workspace_bytes",
           "ssam_scan_delta_marks", "ssam_scan_delta_step", "ssam_rms_norm", "ssam_rms_norm_e4m3", "ssam_rms_norm_backward",
           "ssam_rms_norm_backward_workspace_bytes", "ssam_scan_delta_backward", "ssam_scan_delta_backward_workspace_bytes"]

_torch = None
_fast = None          # the extension module, bound to the library's entry points
_raw_stream = None    # handle of a device's current stream, by the device's index
_several = False      # more than one GPU in the machine


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


class ScanDeltaGrads(NamedTuple):
    q: object
    k: object
    v: object
    g: Optional[object]
    beta: object
    state: Optional[object]


class RmsNormQuantized(NamedTuple):
    values: object
    scales: object


class RmsNormGrads(NamedTuple):
    x: object
    weight: Optional[object]
    gate: Optional[object]


def _load():
    """Loads the library and the extension module; raises if either is not there."""
    global _torch, _fast, _raw_stream, _several
    import torch
    L = binding.lib()
    for name in EXPORTS:
        f = getattr(L, name)
        f.argtypes = [ctypes.c_char_p] if name.endswith(("bytes", "marks")) else [ctypes.c_char_p, ctypes.c_void_p]
        f.restype = ctypes.c_size_t if name.endswith("bytes") else ctypes.c_longlong if name.endswith("marks") else ctypes.c_int
    from . import _sequence
    _sequence.bind(binding.SsamError, *(ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in EXPORTS))
    # (asked for by handle: building a torch.cuda.Stream object takes a microsecond; that way is not part of torch's interface)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _several = torch.cuda.device_count() > 1
    _torch, _fast = torch, _sequence
    return L


def _run(name: str, like, stream, args):
    """The extension module's function on like's device, whichever device is current, with a stream's handle as last argument."""
    if _fast is None:
        _load()
    f = getattr(_fast, name)
    if not isinstance(like, _torch.Tensor) or not like.is_cuda:
        return f(*args, 0)                       # refused there
    index = like.get_device()
    if stream is not None:
        if stream.device != like.device:
            raise ValueError(f"stream must belong to {like.device}, not {stream.device}")
        with _torch.cuda.stream(stream):         # results and workspaces too: made on another stream they could still be in use there
            return f(*args, stream.cuda_stream)
    if _several and index != _torch.cuda.current_device():
        with _torch.cuda.device(index):
            return f(*args, _raw_stream(index))
    return f(*args, _raw_stream(index))


def ssam_conv1d(d_in, weight, bias=None, silu: bool = False, d_state=None, d_final=None, starts=None, lengths=None, d_out=None, stream=None):
    """Per-channel causal filter along time: out[t] = f(bias + sum_j weight[:, j] * in[t - taps + 1 + j]), f the SiLU or nothing.
    weight [channels, taps], bias [channels]: d_in's type or float32.  d_state, d_final: [sequences, taps - 1, channels], the rows
    before each sequence's first (zeros without) and its last ones afterwards (may be the same tensor)."""
    return _run("conv1d", d_in, stream, (d_in, weight, bias, silu, d_state, d_final, starts, lengths, d_out))


def ssam_conv1d_backward(d_grad, d_in, weight, bias=None, silu: bool = False, d_state=None, d_grad_final=None, starts=None, lengths=None,
                         state_grad: bool = False, d_work=None, stream=None) -> Conv1dGrads:
    """Gradients of ssam_conv1d for d_grad, the gradient of its result, and d_grad_final, that of its d_final (none if absent).
    weight's and bias's come in their own type; state_grad: that of d_state (or of the zeros in its place) too."""
    return Conv1dGrads(*_run("conv1d_backward", d_in, stream,
                             (d_grad, d_in, weight, bias, silu, d_state, d_grad_final, starts, lengths, state_grad, d_work)))


def ssam_conv1d_step(d_in, weight, d_state, bias=None, silu: bool = False, slots=None, d_out=None, stream=None):
    """ssam_conv1d for one more row of each of d_in's [rows, channels] sequences.  d_state [pool, taps - 1, channels], in d_in's
    type, is updated in place; slots (int32, device) names each row's slot of it (row r: slot r without).  A row whose slot is
    outside the pool (-1, say) is passed over; rows of one slot are taken in order."""
    return _run("conv1d_step", d_in, stream, (d_in, weight, d_state, bias, silu, slots, d_out))


def ssam_scan_selective_marks(d_in, a, starts=None, lengths=None):
    """A tensor for ssam_scan_selective's d_marks: the states before every 16th row, for ssam_scan_selective_backward; made on
    the current stream."""
    if _fast is None:
        _load()
    return _fast.scan_marks(d_in, a, starts, lengths)


def ssam_scan_selective_workspace_bytes(d_in, a, groups: int = 1, starts=None, lengths=None) -> int:
    """Bytes of d_work that ssam_scan_selective needs for such inputs."""
    if _fast is None:
        _load()
    return _fast.scan_bytes(d_in, a, groups, starts, lengths)


def ssam_scan_selective(d_in, d_dt, a, b, c, skip=None, gate=None, dt_bias=None, softplus: bool = False, d_state=None, d_final=None,
                        d_marks=None, starts=None, lengths=None, d_out=None, d_work=None, stream=None):
    """h_t = exp(d_t a) h_{t-1} + d_t in_t b_t,  out_t = (c_t . h_t + skip in_t) * silu(gate_t),  with d = dt + dt_bias, through a
    softplus or as it is.  d_in, d_dt, gate: rows of channels; b, c: rows of [groups, states], channel k using group
    k // (channels // groups); a [channels, states], skip, dt_bias [channels], d_state, d_final [sequences, channels, states]: float32.
    d_final may be d_state.  d_marks (from ssam_scan_selective_marks) keeps what the gradients need."""
    return _run("scan", d_in, stream, (d_in, d_dt, a, b, c, skip, gate, dt_bias, softplus, d_state, d_final, d_marks, starts, lengths, d_out, d_work))


def ssam_scan_selective_backward(d_grad, d_in, d_dt, a, b, c, d_marks, skip=None, gate=None, dt_bias=None, softplus: bool = False,
                                 d_grad_final=None, starts=None, lengths=None, state_grad: bool = False, d_work=None,
                                 stream=None) -> ScanSelectiveGrads:
    """Gradients of ssam_scan_selective for d_grad, the gradient of its result, and d_grad_final, that of its d_final (none if absent),
    from the marks the forward call left.  Rows' gradients come in d_in's type, the parameters' in float32; state_grad: that of
    d_state (or of the zeros in its place) too."""
    return ScanSelectiveGrads(*_run("scan_backward", d_in, stream, (d_grad, d_in, d_dt, a, b, c, skip, gate, dt_bias, softplus, d_marks, d_grad_final,
                                                                    starts, lengths, state_grad, d_work)))


def ssam_scan_selective_step(d_in, d_dt, a, b, c, d_state, skip=None, gate=None, dt_bias=None, softplus: bool = False, slots=None, d_out=None,
                             stream=None):
    """ssam_scan_selective for one more row of each of d_in's [rows, channels] sequences; d_state [pool, channels, states], float32,
    is updated in place, slots as in ssam_conv1d_step."""
    return _run("scan_step", d_in, stream, (d_in, d_dt, a, b, c, skip, gate, dt_bias, softplus, d_state, slots, d_out))


def ssam_scan_delta_marks(d_k, d_v, starts=None, lengths=None):
    """A tensor for ssam_scan_delta's d_marks: the state before every 64 rows and what the rows correct it by, for
    ssam_scan_delta_backward; made on the current stream."""
    if _fast is None:
        _load()
    return _fast.delta_marks(d_k, d_v, starts, lengths)


def ssam_scan_delta_workspace_bytes(d_k, d_v, starts=None, lengths=None) -> int:
    """Bytes of d_work that ssam_scan_delta needs for such inputs."""
    if _fast is None:
        _load()
    return _fast.delta_bytes(d_k, d_v, starts, lengths)


def ssam_scan_delta(d_q, d_k, d_v, g, beta, scale=None, unit: bool = False, d_state=None, d_final=None, d_marks=None, starts=None, lengths=None,
                    d_out=None, d_work=None, stream=None):
    """Gated delta rule, per head with a matrix S [key, value]:  S' = exp(g_t) S,  u = beta_t (v_t - S'^T k_t),  S = S' + k_t u^T,
    out_t = scale S^T q_t.  d_q, d_k: rows of [key heads, key width] (at most 256), d_v and the result: of [heads, value width], head h using key head
    h // (heads // key heads); g (None: no decay), beta: float32 rows of heads.  unit: rows of q and k are divided by sqrt(their squares' sum
    + 1e-6).  scale: 1 / sqrt(key width) if None.  d_state, d_final [sequences, heads, key, value], float32; d_final may be d_state.  Rows are
    taken 64 at a time: a value that is not finite makes the other rows of its 64, of its head, NaN too, and
    rows more than 2^13 times smaller than others of their 64 keep fewer of fp32's bits (2^-35 of the largest is the error).
    d_marks (from ssam_scan_delta_marks) keeps what the gradients need."""
    return _run("delta", d_v, stream, (d_q, d_k, d_v, g, beta, scale, unit, d_state, d_final, d_marks, starts, lengths, d_out, d_work))


def ssam_scan_delta_backward(d_grad, d_q, d_k, d_v, g, beta, d_marks, scale=None, unit: bool = False, d_grad_final=None, starts=None, lengths=None,
                             state_grad: bool = False, d_work=None, stream=None) -> ScanDeltaGrads:
    """Gradients of ssam_scan_delta for d_grad, the gradient of its result, and d_grad_final, that of its d_final (none if absent), from the
    marks the forward call left.  q's, k's and v's come in d_v's type, g's and beta's in float32; state_grad: that of d_state (or of the
    zeros in its place) too."""
    return ScanDeltaGrads(*_run("delta_backward", d_v, stream, (d_grad, d_q, d_k, d_v, g, beta, scale, unit, d_marks, d_grad_final, starts, lengths,
                                                                state_grad, d_work)))


def ssam_scan_delta_step(d_q, d_k, d_v, g, beta, d_state, scale=None, unit: bool = False, slots=None, d_out=None, stream=None):
    """ssam_scan_delta for one more row of each of d_v's [rows, heads, value] sequences; d_state [pool, heads, key, value], float32, is
    updated in place, slots as in ssam_conv1d_step."""
    return _run("delta_step", d_v, stream, (d_q, d_k, d_v, g, beta, d_state, scale, unit, slots, d_out))


def ssam_rms_norm(d_in, weight=None, d_residual=None, d_sum=None, gate=None, groups: int = 1, eps: float = 1e-6, d_out=None, stream=None):
    """s = d_in + d_residual, rounded to their type (d_in alone without);  out = s / sqrt(mean(s^2) + eps) * weight * silu(gate), the mean over each of
    `groups` equal parts of a row (heads, say; at most 32768 channels each).  weight [channels / groups], d_in's type or float32 (None: ones); gate (None: absent): rows as
    d_in's.  d_sum receives s and may be d_residual itself; the gradients start from it."""
    return _run("norm", d_in, stream, (d_in, weight, d_residual, d_sum, gate, groups, eps, d_out))


def ssam_rms_norm_e4m3(d_in, weight=None, d_residual=None, d_sum=None, gate=None, groups: int = 1, eps: float = 1e-6, block: Optional[int] = None,
                       d_out=None, d_scales=None, stream=None) -> RmsNormQuantized:
    """ssam_rms_norm with its result as torch.float8_e4m3fn and a float32 scale for every `block` channels (16 at least; None: a group's),
    the largest magnitude among them / 448; [.., channels / block] scales."""
    return RmsNormQuantized(*_run("norm_e4m3", d_in, stream, (d_in, weight, d_residual, d_sum, gate, groups, eps, block, d_out, d_scales)))


def ssam_rms_norm_backward(d_grad, d_in, weight=None, d_grad_sum=None, gate=None, groups: int = 1, eps: float = 1e-6, d_work=None,
                           stream=None) -> RmsNormGrads:
    """Gradients of ssam_rms_norm for d_grad, the gradient of its result, and d_grad_sum, that of its sum (none if absent).  d_in is what was
    normalised: the sum, where there was a residual, whose gradient is x's too."""
    return RmsNormGrads(*_run("norm_backward", d_in, stream, (d_grad, d_in, weight, d_grad_sum, gate, groups, eps, d_work)))
