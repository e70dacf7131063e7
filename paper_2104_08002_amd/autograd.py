"""The layer, the causal convolution and the selective scan as ``torch.autograd.Function``s on top of the C-ABI binding.

Glue only: every arithmetic step of the three passes and of the bias and ReLU around them runs in the library's kernels;
torch supplies device memory, the stream and the autograd graph.  This is the interface the
paper's single-layer measurements use (Section 4.3: ``net.forward(x)`` and ``out.sum().backward()``).

A step captured into a graph takes its gradients by ``torch.autograd.grad`` while no eager graph of the same leaves is
alive: the nodes that accumulate into ``.grad`` belong to the stream they were made on.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding, sequence


def _has_tangent(t) -> bool:
    # (unpack_dual asks for the level first too, but takes 2 us of a backward to say that there is none)
    return getattr(forward_ad, "_current_level", 0) >= 0 and forward_ad.unpack_dual(t).tangent is not None


class Conv1dFunction(torch.autograd.Function):
    """y = conv1d(x, w[, bias]) with dilation and zero padding; backward = one conv1d_bwd call."""

    @staticmethod
    def forward(ctx, x, w, bias, dilation: int, padding: int, relu: bool, bf16_out: bool):
        x, w = x.contiguous(), w.contiguous()
        ctx.save_for_backward(x, w)
        ctx.geometry = (int(dilation), int(padding))
        ctx.has_bias = bias is not None
        fused = bias is not None or relu or bf16_out
        if fused:
            y = binding.conv1d_fwd_ex(x, w, dilation, padding, bias=None if bias is None else bias.contiguous().float(),
                                      relu=relu, out_bf16=bf16_out)
        else:
            y = binding.conv1d_fwd(x, w, dilation, padding)
        ctx.relu = relu
        if relu and any(ctx.needs_input_grad):
            # not y itself: what follows the layer may change it in place
            ctx.y_positive = binding.conv1d_relu_mask(y)
        return y

    @staticmethod
    def backward(ctx, gy):
        x, w = ctx.saved_tensors
        d, P = ctx.geometry
        positive = ctx.y_positive if ctx.relu else None
        # create_graph or forward mode over this pass: the bias gradient is differentiable in gy
        if (gy.requires_grad and torch.is_grad_enabled()) or _has_tangent(gy):
            dy = gy
            if positive is not None:
                bit = torch.arange(8, dtype=torch.uint8, device=gy.device)
                dy = gy * ((positive[:, None] >> bit) & 1).bool().flatten()[:gy.numel()].view(gy.shape)
            gb = dy.float().sum(dim=(0, 2)) if ctx.has_bias else None
            dx, dw = binding.conv1d_bwd_ex(x, dy.to(x.dtype).contiguous(), w, d, P, out_bf16=x.dtype == torch.bfloat16)
        else:
            dx, dw, gb = binding.conv1d_layer_bwd(gy.resolve_neg().contiguous(), positive, x, w, d, P, ctx.has_bias)
        return dx, dw.to(w.dtype), gb, None, None, None, None


def conv1d(x, w, bias=None, dilation: int = 1, padding: int = 0, relu: bool = False, bf16_out: bool = False):
    return Conv1dFunction.apply(x, w, bias, dilation, padding, relu, bf16_out)


class Conv1d(torch.nn.Module):
    """Drop-in for ``torch.nn.Conv1d(C, K, S, dilation=d, padding=P)`` (stride 1, one group) on one MI355X."""

    def __init__(self, in_channels: int, out_channels: int, kernel_size: int, dilation: int = 1, padding: int = 0,
                 bias: bool = False, relu: bool = False, dtype=torch.float32, device="cuda"):
        super().__init__()
        self.dilation, self.padding, self.relu = dilation, padding, relu
        w = torch.empty(out_channels, in_channels, kernel_size, dtype=torch.float32, device=device)
        torch.nn.init.normal_(w, std=(in_channels * kernel_size) ** -0.5)
        self.weight = torch.nn.Parameter(w.to(dtype))
        self.bias = torch.nn.Parameter(torch.zeros(out_channels, dtype=torch.float32, device=device)) if bias else None

    def forward(self, x):
        return conv1d(x, self.weight, self.bias, self.dilation, self.padding, self.relu,
                      bf16_out=False)


def _along(t):
    """t with its last axis contiguous."""
    return t if t is None or t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


class CausalFunction(torch.autograd.Function):
    """(y, final) of sequence.conv1d_causal_fwd; its gradients are not differentiable again."""

    @staticmethod
    def forward(ctx, x, w, bias, init, lengths, silu: bool, want_final: bool):
        x, w = _along(x), w.contiguous()
        init = None if init is None else init.contiguous()
        b = None if bias is None else bias.contiguous().float()
        y = sequence.conv1d_causal_fwd(x, w, bias=b, silu=silu, init=init, lengths=lengths, want_final=want_final)
        ctx.save_for_backward(x, w, b, init, lengths)
        ctx.silu, ctx.bias_type = silu, None if bias is None else bias.dtype
        ctx.set_materialize_grads(False)
        return y if want_final else (y, None)

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gfinal):
        x, w, b, init, lengths = ctx.saved_tensors
        gy = torch.zeros_like(x, memory_format=torch.contiguous_format) if gy is None else _along(gy.resolve_neg().to(x.dtype))
        gfinal = None if gfinal is None else gfinal.resolve_neg().to(x.dtype).contiguous()
        dx, dw, db, di = sequence.conv1d_causal_bwd(gy, x, w, bias=b, silu=ctx.silu, init=init, lengths=lengths, dfinal=gfinal,
                                                    want_init=init is not None)
        return dx, dw.to(w.dtype), None if db is None else db.to(ctx.bias_type), di, None, None, None


def conv1d_causal(x, w, bias=None, silu: bool = False, init=None, lengths=None, want_final: bool = False):
    """y[N, C, L] of the depthwise causal convolution of x[N, C, L] with w[C, S]; (y, final) with want_final."""
    y, final = CausalFunction.apply(x, w, bias, init, lengths, silu, want_final)
    return (y, final) if want_final else y


class CausalConv1d(torch.nn.Module):
    """Depthwise causal convolution of `kernel_size` taps, one filter per channel, with a bias and (silu) x * sigmoid(x) behind it."""

    def __init__(self, channels: int, kernel_size: int, bias: bool = True, silu: bool = False, dtype=torch.float32, device="cuda"):
        super().__init__()
        self.silu = silu
        w = torch.empty(channels, kernel_size, dtype=torch.float32, device=device)
        torch.nn.init.normal_(w, std=kernel_size ** -0.5)
        self.weight = torch.nn.Parameter(w.to(dtype))
        self.bias = torch.nn.Parameter(torch.zeros(channels, dtype=torch.float32, device=device)) if bias else None

    def forward(self, x, init=None, lengths=None, want_final: bool = False):
        return conv1d_causal(x, self.weight, self.bias, self.silu, init, lengths, want_final)

    def step(self, x, state):
        """One position x[N, C] of every sequence; `state` is moved on."""
        with torch.no_grad():
            return sequence.conv1d_causal_step(x, self.weight, state, bias=self.bias, silu=self.silu)


class ScanFunction(torch.autograd.Function):
    """(y, final) of sequence.conv1d_scan_fwd; its gradients are not differentiable again."""

    @staticmethod
    def forward(ctx, x, dt, A, B, C, skip, z, dt_bias, init, lengths, softplus: bool, want_final: bool, graph: bool):
        x, dt, B, C, z = (_along(t) for t in (x, dt, B, C, z))
        ctx.types = [None if t is None else t.dtype for t in (A, skip, dt_bias, init)]
        A, skip, dt_bias, init = (None if t is None else t.contiguous().float() for t in (A, skip, dt_bias, init))
        y, final, saved = sequence.conv1d_scan_fwd(x, dt, A, B, C, skip=skip, z=z, dt_bias=dt_bias, softplus=softplus, init=init,
                                                   lengths=lengths, want_final=want_final, save=graph and any(ctx.needs_input_grad))
        ctx.save_for_backward(x, dt, A, B, C, skip, z, dt_bias, init, lengths, saved)
        ctx.softplus = softplus
        ctx.set_materialize_grads(False)
        return y, final

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gfinal):
        x, dt, A, B, C, skip, z, dt_bias, init, lengths, saved = ctx.saved_tensors
        gy = torch.zeros_like(x, memory_format=torch.contiguous_format) if gy is None else _along(gy.resolve_neg().to(x.dtype))
        gfinal = None if gfinal is None else gfinal.resolve_neg().float().contiguous()
        g = sequence.conv1d_scan_bwd(gy, saved, x, dt, A, B, C, skip=skip, z=z, dt_bias=dt_bias, softplus=ctx.softplus, init=init,
                                     lengths=lengths, dfinal=gfinal, want_init=init is not None)
        dA, dskip, ddt_bias, dinit = (None if v is None else v.to(t) for v, t in zip((g.dA, g.dskip, g.ddt_bias, g.dinit), ctx.types))
        return g.dx, g.ddt, dA, g.dB, g.dC, dskip, g.dz, ddt_bias, dinit, None, None, None, None


def conv1d_scan(x, dt, A, B, C, skip=None, z=None, dt_bias=None, softplus: bool = False, init=None, lengths=None, want_final: bool = False):
    """y[N, D, L] of the selective scan (sequence.conv1d_scan_fwd); (y, final) with want_final."""
    # (a parameter wants a gradient under no_grad too, as far as forward can see: the states are kept for a graph alone)
    y, final = ScanFunction.apply(x, dt, A, B, C, skip, z, dt_bias, init, lengths, softplus, want_final, torch.is_grad_enabled())
    return (y, final) if want_final else y
