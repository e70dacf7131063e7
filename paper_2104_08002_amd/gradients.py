"""The norm over many gradient tensors, and clipping by it, without waiting for the device.

Tensor-level marshalling of ``conv1d_grad_norm`` and ``conv1d_grad_clip`` (declared in ``include/conv1d.h``): float32 and
bfloat16 tensors in one call, squares summed in 64 bits, in a fixed order.
"""
from __future__ import annotations

import array
import math

import torch
from torch.autograd.graph import increment_version

from . import binding

_CODES = {torch.float32: binding.CONV1D_FP32, torch.bfloat16: binding.CONV1D_BF16}
_NORMS = {2.0: 2, math.inf: 0}


def _dense(t) -> bool:
    """Every element of the span belongs to the tensor once: the order of its axes does not matter."""
    if t.is_contiguous():
        return True
    last = 1
    for stride, size in sorted((t.stride(i), t.shape[i]) for i in range(t.dim()) if t.shape[i] > 1):
        if stride != last:
            return False
        last = stride * size
    return True


class _Tensors:
    def __init__(self, grads):
        if isinstance(grads, torch.Tensor):
            grads = [grads]
        self.grads = grads = [g for g in grads if g is not None]
        n = len(grads)
        index = set(map(torch.Tensor.get_device, grads)) or {torch.cuda.current_device()}
        if len(index) > 1 or min(index) < 0 or (n and grads[0].device.type != "cuda"):
            raise ValueError("the gradients must be on one device")
        self.device = torch.device("cuda", index.pop())
        types = [g.dtype for g in grads]
        if any(t not in _CODES for t in set(types)):
            raise TypeError(f"unsupported dtype among {set(types)}")
        if not all(map(torch.Tensor.is_contiguous, grads)) and not all(map(_dense, grads)):
            raise ValueError("a gradient has gaps between its elements, or elements in one place")
        # (arrays of this kind are filled in half the time of ctypes' own)
        self.keep = (array.array("Q", list(map(torch.Tensor.data_ptr, grads))), array.array("Q", list(map(torch.Tensor.numel, grads))),
                     array.array("i", [_CODES[t] for t in types]))
        self.args = (*(a.buffer_info()[0] for a in self.keep), n)

    def norm(self, norm_type, workspace):
        kind = _NORMS.get(float(norm_type))
        if kind is None:
            raise ValueError("norm_type is 2 or inf")
        lib = binding.load()
        if workspace is None:
            workspace = torch.empty(max(lib.conv1d_grad_norm_workspace_bytes(*self.args[1::2]), 8), dtype=torch.uint8, device=self.device)
        elif workspace.device != self.device or not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous, on the device of the gradients")
        norm = torch.empty((), dtype=torch.float32, device=self.device)
        binding._check(lib.conv1d_grad_norm(*self.args, kind, norm.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                            binding._current_stream()))
        return norm


def _run(grads, stream, fn):
    t = _Tensors(grads)
    if stream is not None:
        if stream.device != t.device:
            raise ValueError("the stream belongs to another device than the gradients")
        with torch.cuda.stream(stream):
            return fn(t)
    if t.device.index != torch._C._cuda_getDevice():
        with torch.cuda.device(t.device):
            return fn(t)
    return fn(t)


def conv1d_grad_norm(grads, norm_type: float = 2.0, workspace=None, stream=None):
    """The norm over all elements of `grads` (None among them is passed over), a float32 scalar on their device: the root of the
    sum of squares, or with math.inf the largest magnitude; 0 for no elements."""
    return _run(grads, stream, lambda t: t.norm(norm_type, workspace))


def conv1d_grad_clip(grads, max_norm: float, norm_type: float = 2.0, norm=None, workspace=None, stream=None):
    """Scales `grads` in place by min(1, max_norm / (norm + 1e-6)) and returns the norm they had, a float32 scalar on their device.

    norm: a norm found before (conv1d_grad_norm, then joined over ranks, say) in the place of this call's own.
    Tensors that share memory, with each other or with `norm`, are refused.  An infinite norm scales by 0, NaN by NaN: look at the norm before the update.
    """
    max_norm = float(max_norm)
    if not max_norm >= 0:
        raise ValueError("max_norm must not be negative")

    def fn(t):
        total = norm
        if total is None:
            total = t.norm(norm_type, workspace)
        elif total.dtype != torch.float32 or total.numel() != 1 or total.device != t.device:
            raise ValueError("norm must be a float32 scalar on the gradients' device")
        binding._check(binding.load().conv1d_grad_clip(*t.args, total.data_ptr(), max_norm, binding._current_stream()))
        increment_version(t.grads)
        return total

    return _run(grads, stream, fn)
