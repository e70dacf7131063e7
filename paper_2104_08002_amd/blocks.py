"""Operators around the layers of a network: the lookup of an embedding, group norm with an activation, dropout with the residual.

Tensor-level marshalling of ``conv1d_embed_*``, ``conv1d_norm_*`` and ``conv1d_dropout`` (declared in ``include/conv1d.h``, which states the
formulas): every arithmetic step runs in the library's kernels.  Activations are [N, channels, positions] as the layers take
them, contiguous along the positions; where a function says so also with the channels next to each other ("channels last", the
transposed view of a contiguous [N, positions, channels]).

Devices, streams, outputs and workspaces as in ``sequence``.
"""
from __future__ import annotations

import functools
import struct
from typing import Optional

import torch

from . import binding
from .sequence import _apart, _bytes, _on_device, _output, _ptr, _room, _rows, _spread, _whole, increment_version

EMBED_TOKENS64 = 1
NORM_RELU, NORM_SILU = 1, 2

# conv1d_embed_t, conv1d_norm_t and conv1d_dropout_t, packed
_EMBED = struct.Struct("2Pl6if4x")
_NORM = struct.Struct("4P3ld6i")
_DROPOUT = struct.Struct("4P4l2Ld4i")


# how much room a call of these sizes needs (a call into the library, each time, is 1 us)
@functools.lru_cache(maxsize=256)
def _room_for(what, *sizes):
    return getattr(binding.load(), what + "_workspace_bytes")(*sizes)


def _ordered(t, name, shape, dtype, device):
    """A tensor of that shape, positions or channels contiguous."""
    if t.shape != shape or t.dtype != dtype or t.device != device:
        _rows(t, name, shape, dtype, device)
    s = t.stride()
    if s[2] != 1 and s[1] != 1 and shape[1] > 1 and shape[2] > 1:
        raise ValueError(f"{name} must be contiguous along its positions or its channels")
    return s


def _channels_last(t) -> bool:
    """Whether channels lie next to each other, in one order with the library's (an axis of one element has no stride)."""
    _, C, L = t.shape
    _, sc, sl = t.stride()
    if L == 1:
        return C == 1 or sc == 1
    return sl != 1 and (C == 1 or sc == 1)


def _new(shape, last, like):
    N, C, L = shape
    return like.new_empty((N, L, C)).transpose(1, 2) if last else like.new_empty(shape)


def _ordered_output(out, shape, last, like, ins):
    """The caller's `out`, checked, or a new tensor, in the wanted order."""
    if out is None:
        return _new(shape, last, like)
    _, sc, sl = _ordered(out, "out", shape, like.dtype, like.device)
    if (sc != 1 and shape[1] > 1) if last else (sl != 1 and shape[2] > 1):
        raise ValueError("out must be contiguous along its " + ("channels" if last else "positions"))
    increment_version(_apart(_spread(out, "out"), ins))
    return out


# ---- embedding -----------------------------------------------------------------------------------------------------------
def _embed(tokens, lengths, V, D, dtype, scale, device, step=False):
    if tokens.dim() != (1 if step else 2) or 0 in tokens.shape:
        raise ValueError(f"tokens must have the shape {'[N]' if step else '[N, L]'}, none of it 0")
    if tokens.dtype != torch.int64 and tokens.dtype != torch.int32:
        raise TypeError(f"tokens must be int32 or int64: got {tokens.dtype}")
    N, L = (tokens.shape[0], 1) if step else tokens.shape
    if step:
        if tokens.device != device:
            raise ValueError("tokens must be on the device of the table")
    else:
        _rows(tokens, "tokens", tokens.shape, tokens.dtype, device)
    if lengths is not None:
        _whole(lengths, "lengths", (N,), torch.int32, device)
    return _EMBED.pack(tokens.data_ptr(), _ptr(lengths), tokens.stride(0), N, D, L, V, dtype, EMBED_TOKENS64 if tokens.dtype == torch.int64 else 0, scale)


def _table(table):
    if table.dim() != 2 or 0 in table.shape:
        raise ValueError("table must have the shape [V, D], none of it 0")
    code = binding._dtype_code(table)
    _whole(table, "table", table.shape, table.dtype, table.device)
    return (*table.shape, code)


@_on_device
def conv1d_embed_fwd(table, tokens, scale: float = 1.0, lengths=None, channels_last: bool = False, out=None):
    """y[N, D, L] = scale * table[tokens] of tokens[N, L] (int32 or int64) and table[V, D], in the table's type, contiguous along
    the positions or, with channels_last, the channels.

    lengths int32 [N]: y is 0 from there on; it is 0 too where a token is outside [0, V).
    """
    V, D, code = _table(table)
    p = _embed(tokens, lengths, V, D, code, scale, table.device)
    y = _ordered_output(out, (tokens.shape[0], D, tokens.shape[1]), channels_last, table, (table, tokens, lengths))
    binding._check(binding.load().conv1d_embed_fwd(p, table.data_ptr(), y.data_ptr(), *y.stride(), binding._current_stream()))
    return y


@_on_device
def conv1d_embed_step(table, tokens, scale: float = 1.0, out=None):
    """y[N, D] = scale * table[tokens] for one token of every sequence, tokens[N]."""
    V, D, code = _table(table)
    p = _embed(tokens, None, V, D, code, scale, table.device, step=True)
    if out is None:
        y = table.new_empty((tokens.shape[0], D))
    else:
        y = _rows(out, "out", (tokens.shape[0], D), table.dtype, table.device)
        increment_version(_apart(_spread(y, "out"), (table, tokens)))
    binding._check(binding.load().conv1d_embed_fwd(p, table.data_ptr(), y.data_ptr(), y.stride(0), 1, 1, binding._current_stream()))
    return y


@_on_device
def conv1d_embed_bwd(dy, tokens, V: int, scale: float = 1.0, lengths=None, workspace=None):
    """dtable [V, D] float32 for dy[N, D, L], positions or channels contiguous: scale times the sum of dy over the positions of each
    token, in an order that depends on the tokens, the sizes and dy's strides alone."""
    if dy.dim() != 3 or 0 in dy.shape or not 1 <= V < 1 << 31:
        raise ValueError("dy must have the shape [N, D, L], none of it 0, and V be at least 1 and below 2^31")
    (N, D, L), code, dev = dy.shape, binding._dtype_code(dy), dy.device
    p = _embed(tokens, lengths, V, D, code, scale, dev)
    if tokens.shape != (N, L):
        raise ValueError(f"tokens must have the shape {[N, L]}")
    sn, sd, sl = _ordered(dy, "dy", dy.shape, dy.dtype, dev)
    lib = binding.load()
    workspace = _room(workspace, _room_for("conv1d_embed_bwd", N, D, L, V, code, sd, sl), dev)
    dtable = torch.empty((V, D), dtype=torch.float32, device=dev)
    binding._check(lib.conv1d_embed_bwd(p, dy.data_ptr(), sn, sd, sl, dtable.data_ptr(), _ptr(workspace), _bytes(workspace), binding._current_stream()))
    return dtable


# ---- group norm ------------------------------------------------------------------------------------------------------------
def _norm(x, groups, weight, bias, relu, silu, eps, lengths):
    if x.dim() != 3 or 0 in x.shape:
        raise ValueError("x must have the shape [N, C, L], none of it 0")
    N, C, L = x.shape
    if groups < 1 or C % groups:
        raise ValueError("groups must divide the channels")
    if relu and silu:
        raise ValueError("relu or silu, not both")
    code, dev = binding._dtype_code(x), x.device
    strides = _ordered(x, "x", x.shape, x.dtype, dev)
    if weight is not None:
        _whole(weight, "weight", (C,), torch.float32, dev)
    if bias is not None:
        _whole(bias, "bias", (C,), torch.float32, dev)
    if lengths is not None:
        _whole(lengths, "lengths", (N,), torch.int32, dev)
    return _NORM.pack(x.data_ptr(), _ptr(weight), _ptr(bias), _ptr(lengths), *strides, eps, N, C, L, groups, code,
                      (NORM_RELU if relu else 0) | (NORM_SILU if silu else 0)), (N, C, L, groups, code, *strides[1:])


@_on_device
def conv1d_norm_fwd(x, groups: int, weight=None, bias=None, relu: bool = False, silu: bool = False, eps: float = 1e-5, lengths=None,
                    want_stats: bool = False, out=None, workspace=None):
    """y[N, C, L] of x[N, C, L], positions or channels contiguous (y then has the same order), in x's type: each of the `groups` groups
    of neighbouring channels of a sample brought to mean 0 and variance 1, times weight[C] plus bias[C] (float32), with ReLU or
    x * sigmoid(x) behind it; (y, stats) with want_stats: float64 [N, groups, 2], mean and 1 / sqrt(variance + eps).

    lengths int32 [N]: positions from there on are not part of the sequence, y is 0 there.
    """
    p, sizes = _norm(x, groups, weight, bias, relu, silu, eps, lengths)
    lib = binding.load()
    y = _ordered_output(out, x.shape, _channels_last(x), x, (x, weight, bias, lengths))
    stats = torch.empty((x.shape[0], groups, 2), dtype=torch.float64, device=x.device) if want_stats else None
    workspace = _room(workspace, _room_for("conv1d_norm_fwd", *sizes), x.device)
    binding._check(lib.conv1d_norm_fwd(p, y.data_ptr(), *y.stride(), _ptr(stats), _ptr(workspace), _bytes(workspace), binding._current_stream()))
    return (y, stats) if want_stats else y


@_on_device
def conv1d_norm_bwd(dy, stats, x, groups: int, weight=None, bias=None, relu: bool = False, silu: bool = False, eps: float = 1e-5, lengths=None,
                    workspace=None, want_weight: bool = True, want_bias: bool = True):
    """(dx, dweight, dbias) of the call of conv1d_norm_fwd that had the same arguments and left `stats`: dx in x's type and order, which
    is dy's too, dweight and dbias [C] float32, None for a parameter that was not there or whose gradient is not wanted."""
    (p, sizes), (N, C, L) = _norm(x, groups, weight, bias, relu, silu, eps, lengths), x.shape
    lib, dev, last = binding.load(), x.device, _channels_last(x)
    strides = _ordered(dy, "dy", x.shape, x.dtype, dev)
    if (strides[1] != 1 and C > 1) if last else (strides[2] != 1 and L > 1):
        raise ValueError("dy must be contiguous along its " + ("channels" if last else "positions") + ", as x is")
    _whole(stats, "stats", (N, groups, 2), torch.float64, dev)
    dx = _new(x.shape, last, x)
    dweight, dbias = (torch.empty_like(t) if want and t is not None else None for t, want in ((weight, want_weight), (bias, want_bias)))
    workspace = _room(workspace, _room_for("conv1d_norm_bwd", *sizes), dev)
    binding._check(lib.conv1d_norm_bwd(p, dy.data_ptr(), *strides, stats.data_ptr(), dx.data_ptr(), *dx.stride(), _ptr(dweight), _ptr(dbias),
                                       _ptr(workspace), _bytes(workspace), binding._current_stream()))
    return dx, dweight, dbias


# ---- dropout -----------------------------------------------------------------------------------------------------------------
@_on_device
def conv1d_dropout(x, p: float, key: int, call: int = 0, counter: Optional[torch.Tensor] = None, residual=None, lengths=None, out=None):
    """y[N, C, L] = residual + x / (1 - p) where an element is kept, residual where it is dropped, each with probability p, in x's type.

    What is dropped follows from the element's place, `key` and `call` (64 bits each, unsigned): the same call with the
    gradient in place of x, and no residual, is its backward pass.  Steps of a program take another `call` each.
    counter int64 [], on the device: a number added to `call` when the kernel runs; a captured step that is replayed needs one.
    lengths int32 [N]: y is 0 from there on.
    """
    if x.dim() != 3 or 0 in x.shape:
        raise ValueError("x must have the shape [N, C, L], none of it 0")
    if not 0 <= p <= 1:
        raise ValueError("p must lie between 0 and 1")
    if not (0 <= key < 1 << 64 and 0 <= call < 1 << 64):
        raise ValueError("key and call have 64 bits")
    (N, C, L), dev, code = x.shape, x.device, binding._dtype_code(x)
    _rows(x, "x", x.shape, x.dtype, dev)
    if residual is not None:
        _rows(residual, "residual", x.shape, x.dtype, dev)
    if lengths is not None:
        _whole(lengths, "lengths", (N,), torch.int32, dev)
    if counter is not None and (counter.dtype != torch.int64 or counter.numel() != 1 or counter.device != dev):
        raise ValueError("counter must be an int64 scalar on the device of x")
    y = _output(out, x, (x, residual, lengths, counter))
    rs = (0, 0) if residual is None else residual.stride()
    a = _DROPOUT.pack(x.data_ptr(), _ptr(residual), _ptr(lengths), _ptr(counter), x.stride(0), x.stride(1), rs[0], rs[1], key, call, p, N, C, L, code)
    binding._check(binding.load().conv1d_dropout(a, y.data_ptr(), y.stride(0), y.stride(1), binding._current_stream()))
    return y
