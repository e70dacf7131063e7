"""Group norm whose weight or bias is frozen: its gradient is neither added up nor returned.  On the CPU which gradients autograd asks for (the
operator replaced by a stand-in), on the GPU the values of what is left."""
import itertools

import pytest
import torch

from paper_2104_08002_amd import autograd

FROZEN = pytest.mark.parametrize("weight,bias", list(itertools.product([False, True], repeat=2)))


@FROZEN
def test_autograd_asks_for_what_is_wanted(monkeypatch, weight, bias):
    asked = []

    def backward(dy, stats, x, groups, weight=None, bias=None, want_weight=True, want_bias=True, **_):
        asked.append((want_weight, want_bias))
        return dy.clone(), torch.ones_like(weight) if want_weight else None, torch.ones_like(bias) if want_bias else None

    monkeypatch.setattr(autograd.blocks, "conv1d_norm_fwd", lambda x, groups, **_: (x.clone(), torch.zeros(x.shape[0], groups, 2, dtype=torch.float64)))
    monkeypatch.setattr(autograd.blocks, "conv1d_norm_bwd", backward)
    layer = autograd.GroupNorm(2, 6, device="cpu")
    layer.weight.requires_grad_(weight)
    layer.bias.requires_grad_(bias)
    layer(torch.randn(2, 6, 5, requires_grad=True)).sum().backward()
    assert asked == [(weight, bias)] and (layer.weight.grad is not None, layer.bias.grad is not None) == (weight, bias)


@pytest.mark.gpu
@FROZEN
@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
@pytest.mark.parametrize("N,C,L,G", [(2, 12, 40, 3), (1100, 8, 5, 2), (2, 16, 9000, 2), (3, 1000, 50, 1)])
def test_values(weight, bias, last, N, C, L, G):
    """One launch a group and several: the wanted gradients are those of the whole call, bit for bit."""
    from paper_2104_08002_amd import blocks

    gen = torch.Generator(device="cuda").manual_seed(C)
    x, dy = (torch.randn((N, L, C) if last else (N, C, L), generator=gen, device="cuda") for _ in range(2))
    x, dy = (v.transpose(1, 2) if last else v for v in (x, dy))
    w, b = (torch.randn(C, generator=gen, device="cuda") for _ in range(2))
    how = {"weight": w, "bias": b, "silu": True}
    _, stats = blocks.conv1d_norm_fwd(x, G, want_stats=True, **how)
    whole = blocks.conv1d_norm_bwd(dy, stats, x, G, **how)
    for got, want, wanted in zip(blocks.conv1d_norm_bwd(dy, stats, x, G, want_weight=weight, want_bias=bias, **how), whole, (True, weight, bias)):
        assert torch.equal(got, want) if wanted else got is None
    leaves = [x.clone().requires_grad_(True), w.clone().requires_grad_(weight), b.clone().requires_grad_(bias)]
    autograd.conv1d_norm(leaves[0], G, *leaves[1:], silu=True).backward(dy)
    for leaf, want in zip(leaves, whole):
        assert torch.equal(leaf.grad, want) if leaf.requires_grad else leaf.grad is None
