"""Sequence operators beside the layer: a short causal convolution of every channel by itself, and a selective scan.

Tensor-level marshalling of ``conv1d_causal_*`` and ``conv1d_scan_*`` (declared in ``include/conv1d.h``, which states the
formulas): every arithmetic step runs in the library's kernels.  Layout as for the layer: [N, channels, positions],
contiguous along the positions; samples and channels may be strided, so the halves of a projection need no copy.

All of them run on the device of their tensors, on its current stream or on `stream`; outputs and workspaces are then
allocated for that stream, and the caller sees to the order between it and the streams that the inputs come from.
"""
from __future__ import annotations

import functools
import struct
from typing import NamedTuple, Optional

import torch
from torch.autograd.graph import increment_version

from . import binding

CAUSAL_SILU = 1
SCAN_SOFTPLUS = 1
MOST_TAPS, MOST_STATES = 8, 64


# conv1d_causal_t and conv1d_scan_t, packed (a ctypes structure takes three times as long to fill)
_CAUSAL = struct.Struct("5P2l6i")
_SCAN = struct.Struct("10P12l7i4x")


class ScanGrads(NamedTuple):
    """Gradients of conv1d_scan_fwd; None for an input that was not there (dinit: that was not asked for)."""

    dx: torch.Tensor
    ddt: torch.Tensor
    dA: torch.Tensor
    dB: torch.Tensor
    dC: torch.Tensor
    dskip: Optional[torch.Tensor]
    dz: Optional[torch.Tensor]
    ddt_bias: Optional[torch.Tensor]
    dinit: Optional[torch.Tensor]


_device_now = torch._C._cuda_getDevice


def _on_device(fn):
    """Runs fn with the device of its first argument current and, if asked for, on `stream`."""
    name = fn.__code__.co_varnames[0]

    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        t = args[0] if args else kw[name]
        device = t.device
        if device.type != "cuda":
            raise ValueError("the tensors must be on the device")
        if stream is not None:
            if stream.device != device:
                raise ValueError("the stream belongs to another device than the tensors")
            with torch.cuda.stream(stream):
                return fn(*args, **kw)
        if device.index != _device_now():
            with torch.cuda.device(device):
                return fn(*args, **kw)
        return fn(*args, **kw)

    return call


def _rows(t, name, shape, dtype, device):
    """A tensor of that shape whose last axis is contiguous."""
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} on {device}: got {t.dtype} {list(t.shape)} on {t.device}")
    if t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous along its last axis")
    return t


def _whole(t, name, shape, dtype, device):
    if t.shape != shape or t.dtype != dtype or t.device != device:
        _rows(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _like(x):
    return torch.empty_like(x) if x.is_contiguous() else torch.empty_like(x, memory_format=torch.contiguous_format)


def _output(out, x, ins):
    """The caller's `out`, checked, or a new tensor as x."""
    if out is None:
        return _like(x)
    increment_version(_apart(_spread(_rows(out, "out", x.shape, x.dtype, x.device), "out"), ins))
    return out


def _room(workspace, nbytes, device):
    """The caller's workspace, checked (its size by the call), or a new one; None for no bytes."""
    if workspace is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous, on the device of the tensors")
    return workspace


def _bytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _spread(t, name):
    """An output: no two of its elements in one place."""
    if t.is_contiguous():
        return t
    last, strides = 1, sorted((t.stride(i), t.shape[i]) for i in range(t.dim()) if t.shape[i] > 1)
    for stride, size in strides:
        if stride < last:
            raise ValueError(f"elements of {name} share memory")
        last = stride * size
    return t


def _span(t):
    first = t.data_ptr()
    return first, first + (t.nbytes if t.is_contiguous() else t.element_size() * (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))))


def _arc(t, period):
    """Bytes that t takes up modulo `period`: axes that step by whole periods add none."""
    size = t.element_size()
    return size * (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()) if s * size % period))


def _interleaved(out, t):
    """Whether the two lie in different parts of a period of out's strides, as the halves of a projection do."""
    for stride in out.stride():
        period = stride * out.element_size()
        if period:
            gap = (t.data_ptr() - out.data_ptr()) % period
            if _arc(out, period) <= gap and gap + _arc(t, period) <= period:
                return True
    return False


def _apart(out, ins):
    """An output given by the caller: its elements may not lie where an input's do."""
    first, last = _span(out)
    for t in ins:
        if t is not None:
            t0, t1 = _span(t)
            if first < t1 and t0 < min(last, t1) and not _interleaved(out, t):
                raise ValueError("out shares memory with an input")
    return out


# ---- depthwise causal convolution --------------------------------------------------------------------------------------
def _causal(x, w, bias, silu, init, lengths, step=False):
    if x.dim() != (2 if step else 3) or 0 in x.shape:
        raise ValueError(f"x must have the shape {'[N, C]' if step else '[N, C, L]'}, none of it 0")
    N, C, L = (*x.shape, 1) if step else x.shape
    if w.dim() != 2 or w.shape[0] != C or w.shape[1] < 1:
        raise ValueError("w must have the shape [C, S]")
    S, dev, t, code = w.shape[1], x.device, x.dtype, binding._dtype_code(x)
    _rows(x, "x", x.shape, t, dev)
    _whole(w, "w", (C, S), t, dev)
    if bias is not None:
        _whole(bias, "bias", (C,), torch.float32, dev)
    if init is not None:
        _whole(init, "init", (N, C, S - 1), t, dev)
    if lengths is not None:
        _whole(lengths, "lengths", (N,), torch.int32, dev)
    return _CAUSAL.pack(x.data_ptr(), w.data_ptr(), _ptr(bias), _ptr(init), _ptr(lengths), x.stride(0), 0 if step else x.stride(1), N, C, L, S, code,
                        CAUSAL_SILU if silu else 0), N, C, L, S


@_on_device
def conv1d_causal_fwd(x, w, bias=None, silu: bool = False, init=None, lengths=None, want_final: bool = False, out=None):
    """y[N, C, L] of x[N, C, L] and w[C, S], in x's type; (y, final) with want_final.

    init, final [N, C, S - 1]: the inputs before the sequence, and those that the position behind it needs.
    lengths int32 [N]: positions from there on are not part of the sequence, y is 0 there.
    """
    p, N, C, _, S = _causal(x, w, bias, silu, init, lengths)
    y = _output(out, x, (x, w, bias, init, lengths))
    final = x.new_empty((N, C, S - 1)) if want_final else None
    binding._check(binding.load().conv1d_causal_fwd(p, y.data_ptr(), y.stride(0), y.stride(1), _ptr(final), binding._current_stream()))
    return (y, final) if want_final else y


@_on_device
def conv1d_causal_bwd(dy, x, w, bias=None, silu: bool = False, init=None, lengths=None, dfinal=None, want_init: bool = False, workspace=None):
    """(dx, dw, dbias, dinit) of conv1d_causal_fwd(x, w, bias, silu, init, lengths): dx and dinit in x's type, dw [C, S] and dbias [C]
    in float32.  dbias is None without a bias, dinit unless wanted."""
    (p, N, C, L, S), dev = _causal(x, w, bias, silu, init, lengths), x.device
    _rows(dy, "dy", x.shape, x.dtype, dev)
    if dfinal is not None:
        _whole(dfinal, "dfinal", (N, C, S - 1), x.dtype, dev)
    lib = binding.load()
    workspace = _room(workspace, lib.conv1d_causal_bwd_workspace_bytes(N, C, L, S), dev)
    dx = _like(x)
    dw = _like(w) if w.dtype == torch.float32 else torch.empty((C, S), dtype=torch.float32, device=dev)
    db = None if bias is None else _like(bias)
    di = x.new_empty((N, C, S - 1)) if want_init else None
    binding._check(lib.conv1d_causal_bwd(p, dy.data_ptr(), dy.stride(0), dy.stride(1), _ptr(dfinal), dx.data_ptr(), dw.data_ptr(),
                                         _ptr(db), _ptr(di), _ptr(workspace), _bytes(workspace), binding._current_stream()))
    return dx, dw, db, di


@_on_device
def conv1d_causal_step(x, w, state, bias=None, silu: bool = False, out=None):
    """y[N, C] for one position x[N, C] of every sequence; state [N, C, S - 1], as conv1d_causal_fwd leaves it in `final`, is
    moved on by that position."""
    p, N, C, _, S = _causal(x, w, bias, silu, None, None, step=True)
    _whole(state, "state", (N, C, S - 1), x.dtype, x.device)
    y = _output(out, x, (x, w, bias, state))
    binding._check(binding.load().conv1d_causal_step(p, state.data_ptr(), y.data_ptr(), y.stride(0), binding._current_stream()))
    increment_version(state)
    return y


# ---- selective scan ----------------------------------------------------------------------------------------------------
def _scan(x, dt, A, B, C, skip, z, dt_bias, softplus, init, lengths, step=False):
    if x.dim() != (2 if step else 3) or 0 in x.shape:
        raise ValueError(f"x must have the shape {'[N, D]' if step else '[N, D, L]'}, none of it 0")
    shape = x.shape
    N, D, L = (*shape, 1) if step else shape
    if A.dim() != 2 or A.shape[0] != D or A.shape[1] < 1:
        raise ValueError("A must have the shape [D, S]")
    S, dev, t, code = A.shape[1], x.device, x.dtype, binding._dtype_code(x)
    if B.dim() != (3 if step else 4) or B.shape[1] < 1 or D % B.shape[1]:
        raise ValueError(f"B must have the shape {'[N, G, S]' if step else '[N, G, S, L]'}, G a divisor of D")
    G = B.shape[1]
    states = (N, G, S) if step else (N, G, S, L)
    _rows(x, "x", shape, t, dev)
    _rows(dt, "dt", shape, t, dev)
    _whole(A, "A", (D, S), torch.float32, dev)
    _rows(B, "B", states, t, dev)
    _rows(C, "C", states, t, dev)
    if skip is not None:
        _whole(skip, "skip", (D,), torch.float32, dev)
    if z is not None:
        _rows(z, "z", shape, t, dev)
    if dt_bias is not None:
        _whole(dt_bias, "dt_bias", (D,), torch.float32, dev)
    if init is not None:
        _whole(init, "init", (N, D, S), torch.float32, dev)
    if lengths is not None:
        _whole(lengths, "lengths", (N,), torch.int32, dev)
    xs, ds, bs, cs = x.stride(), dt.stride(), B.stride(), C.stride()
    zs = (0, 0) if z is None else z.stride()
    return _SCAN.pack(x.data_ptr(), dt.data_ptr(), B.data_ptr(), C.data_ptr(), _ptr(z), A.data_ptr(), _ptr(skip), _ptr(dt_bias), _ptr(init), _ptr(lengths),
                      xs[0], xs[1], ds[0], ds[1], zs[0], zs[1], bs[0], bs[1], bs[2], cs[0], cs[1], cs[2], N, D, L, S, G, code,
                      SCAN_SOFTPLUS if softplus else 0), N, D, L, S, G


@_on_device
def conv1d_scan_fwd(x, dt, A, B, C, skip=None, z=None, dt_bias=None, softplus: bool = False, init=None, lengths=None, want_final: bool = False,
                    save: bool = False, out=None, workspace=None):
    """(y, final, saved): the selective scan of x[N, D, L] with steps dt[N, D, L], rates A[D, S] (float32), B and C [N, G, S, L],
    gated by z[N, D, L]; y in x's type.

    init, final [N, D, S] float32: the state before and behind the sequence (final is None unless wanted).
    saved: what conv1d_scan_bwd needs of this call, with `save`; None without.
    lengths int32 [N]: positions from there on are not part of the sequence, y is 0 there and the state stays.
    """
    (p, N, D, L, S, G), dev = _scan(x, dt, A, B, C, skip, z, dt_bias, softplus, init, lengths), x.device
    lib = binding.load()
    y = _output(out, x, (x, dt, A, B, C, skip, z, dt_bias, init, lengths))
    final = A.new_empty((N, D, S)) if want_final else None
    saved = _room(None, lib.conv1d_scan_saved_bytes(N, D, L, S), dev) if save else None
    workspace = _room(workspace, lib.conv1d_scan_fwd_workspace_bytes(N, D, L, S, G), dev)
    binding._check(lib.conv1d_scan_fwd(p, y.data_ptr(), y.stride(0), y.stride(1), _ptr(final), _ptr(saved), _ptr(workspace),
                                       _bytes(workspace), binding._current_stream()))
    return y, final, saved


@_on_device
def conv1d_scan_bwd(dy, saved, x, dt, A, B, C, skip=None, z=None, dt_bias=None, softplus: bool = False, init=None, lengths=None, dfinal=None,
                    want_init: bool = False, workspace=None) -> ScanGrads:
    """Gradients of the call of conv1d_scan_fwd that had the same arguments and left `saved`: those of x, dt, B, C and z in their
    type, of A, skip, dt_bias and init in float32."""
    (p, N, D, L, S, G), dev, t = _scan(x, dt, A, B, C, skip, z, dt_bias, softplus, init, lengths), x.device, x.dtype
    lib = binding.load()
    _rows(dy, "dy", x.shape, t, dev)
    if dfinal is not None:
        _whole(dfinal, "dfinal", (N, D, S), torch.float32, dev)
    _whole(saved, "saved", (lib.conv1d_scan_saved_bytes(N, D, L, S),), torch.uint8, dev)
    workspace = _room(workspace, lib.conv1d_scan_bwd_workspace_bytes(N, D, L, S, G), dev)
    g = ScanGrads(_like(x), _like(x), _like(A), _like(B), _like(C), None if skip is None else _like(skip), None if z is None else _like(x),
                  None if dt_bias is None else _like(dt_bias), A.new_empty((N, D, S)) if want_init else None)
    binding._check(lib.conv1d_scan_bwd(p, dy.data_ptr(), dy.stride(0), dy.stride(1), _ptr(dfinal), saved.data_ptr(), *map(_ptr, g),
                                       _ptr(workspace), _bytes(workspace), binding._current_stream()))
    return g


@_on_device
def conv1d_scan_step(x, dt, A, B, C, state, skip=None, z=None, dt_bias=None, softplus: bool = False, out=None):
    """y[N, D] for one position of every sequence: x, dt, z [N, D], B and C [N, G, S]; state [N, D, S] float32, as conv1d_scan_fwd
    leaves it in `final`, is moved on by that position."""
    p, N, D, _, S, _ = _scan(x, dt, A, B, C, skip, z, dt_bias, softplus, None, None, step=True)
    _whole(state, "state", (N, D, S), torch.float32, x.device)
    y = _output(out, x, (x, dt, A, B, C, skip, z, dt_bias, state))
    binding._check(binding.load().conv1d_scan_step(p, state.data_ptr(), y.data_ptr(), y.stride(0), binding._current_stream()))
    increment_version(state)
    return y
