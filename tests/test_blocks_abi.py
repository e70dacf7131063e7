"""Argument checks of the operators around the layers, without a GPU: no kernel is launched here."""
import ctypes

import pytest
import torch

from blocks_structs import Dropout, Embed, Norm
from paper_2104_08002_amd import binding, blocks

FAKE = 0x10000          # never dereferenced: every call below fails its checks
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_packed_arguments_are_the_structures():
    assert (blocks._EMBED.size, blocks._NORM.size, blocks._DROPOUT.size) == tuple(map(ctypes.sizeof, (Embed, Norm, Dropout)))


def _embed(**kw):
    f = dict(tokens=FAKE, lengths=None, tok_sn=100, N=2, D=6, L=100, V=50, dtype=0, flags=0, scale=1.0)
    f.update(kw)
    return ctypes.byref(Embed(**f))


@pytest.mark.parametrize("bad,status", [
    (dict(tokens=None), EINVAL), (dict(N=0), EINVAL), (dict(D=0), EINVAL), (dict(L=0), EINVAL), (dict(V=0), EINVAL), (dict(dtype=2), EINVAL), (dict(flags=2), EINVAL),
    (dict(tokens=FAKE + 2), EINVAL), (dict(tokens=FAKE + 4, flags=1), EINVAL), (dict(lengths=FAKE + 2), EINVAL), (dict(D=(1 << 20) + 1), EUNSUPPORTED),
    (dict(V=1 << 30), EUNSUPPORTED), (dict(N=1 << 16, L=(1 << 14) + 1), EUNSUPPORTED)])
def test_embedding_refusals(lib, bad, status):
    assert lib.conv1d_embed_fwd(_embed(**bad), FAKE, FAKE, 600, 100, 1, None) == status
    assert lib.conv1d_embed_bwd(_embed(**bad), FAKE, 600, 100, 1, FAKE, FAKE, 1 << 40, None) == status


def test_embedding_refusals_of_tensors(lib):
    fwd, bwd = lib.conv1d_embed_fwd, lib.conv1d_embed_bwd
    assert fwd(_embed(), None, FAKE, 600, 100, 1, None) == EINVAL
    assert fwd(_embed(), FAKE, None, 600, 100, 1, None) == EINVAL
    assert fwd(_embed(), FAKE + 2, FAKE, 600, 100, 1, None) == EINVAL
    assert fwd(_embed(), FAKE, FAKE, 600, 200, 2, None) == EINVAL                # neither positions nor channels contiguous
    assert bwd(_embed(), None, 600, 100, 1, FAKE, FAKE, 1 << 40, None) == EINVAL
    assert bwd(_embed(), FAKE, 600, 100, 1, None, FAKE, 1 << 40, None) == EINVAL
    assert bwd(_embed(), FAKE, 600, 200, 2, FAKE, FAKE, 1 << 40, None) == EINVAL
    assert bwd(_embed(), FAKE, 600, 100, 1, FAKE, FAKE + 128, 1 << 40, None) == EINVAL
    for V in (50, 5000):
        for s in ((600, 100, 1), (600, 1, 6)):
            need = lib.conv1d_embed_bwd_workspace_bytes(2, 6, 100, V, 0, *s[1:])
            assert need > 0
            assert bwd(_embed(V=V), FAKE, *s, FAKE, None, need, None) == EWORKSPACE and bwd(_embed(V=V), FAKE, *s, FAKE, FAKE, need - 1, None) == EWORKSPACE
    assert lib.conv1d_embed_bwd_workspace_bytes(0, 6, 100, 50, 0, 100, 1) == 0 and lib.conv1d_embed_bwd_workspace_bytes(2, 6, 100, 50, 3, 100, 1) == 0


def _norm(**kw):
    f = dict(x=FAKE, weight=None, bias=None, lengths=None, x_sn=600, x_sc=100, x_sl=1, eps=1e-5, N=2, C=6, L=100, G=3, dtype=0, flags=0)
    f.update(kw)
    return ctypes.byref(Norm(**f))


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), EINVAL), (dict(N=0), EINVAL), (dict(C=0), EINVAL), (dict(L=0), EINVAL), (dict(G=0), EINVAL), (dict(G=4), EINVAL), (dict(dtype=2), EINVAL),
    (dict(flags=4), EINVAL), (dict(flags=3), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(x=FAKE + 2), EINVAL),
    (dict(weight=FAKE + 2), EINVAL), (dict(bias=FAKE + 1), EINVAL), (dict(lengths=FAKE + 2), EINVAL), (dict(x_sc=200, x_sl=2), EINVAL),
    (dict(C=3 << 19, G=1), EUNSUPPORTED), (dict(L=(1 << 30) + 8), EUNSUPPORTED), (dict(N=1 << 23), EUNSUPPORTED), (dict(C=64, G=1, L=1 << 28), EUNSUPPORTED)])
def test_norm_refusals(lib, bad, status):
    assert lib.conv1d_norm_fwd(_norm(**bad), FAKE, 600, 100, 1, None, FAKE, 1 << 40, None) == status
    assert lib.conv1d_norm_bwd(_norm(**bad), FAKE, 600, 100, 1, FAKE, FAKE, 600, 100, 1, FAKE, FAKE, FAKE, 1 << 40, None) == status


def test_norm_refusals_of_tensors(lib):
    fwd, bwd = lib.conv1d_norm_fwd, lib.conv1d_norm_bwd
    big = dict(C=6, G=1, L=100000, x_sn=600000, x_sc=100000)
    assert fwd(_norm(), None, 600, 100, 1, None, FAKE, 1 << 40, None) == EINVAL
    assert fwd(_norm(), FAKE, 600, 1, 6, None, FAKE, 1 << 40, None) == EINVAL             # y in the other order
    assert fwd(_norm(), FAKE, 600, 100, 1, FAKE + 4, FAKE, 1 << 40, None) == EINVAL
    assert fwd(_norm(), FAKE, 600, 100, 1, None, FAKE + 8, 1 << 40, None) == EINVAL
    need = lib.conv1d_norm_fwd_workspace_bytes(2, 6, 100000, 1, 0, 100000, 1)
    assert need > 0 and lib.conv1d_norm_fwd_workspace_bytes(2, 6, 100, 3, 0, 100, 1) == 0   # small groups: one launch
    assert fwd(_norm(**big), FAKE, 600000, 100000, 1, None, FAKE, 0, None) == EWORKSPACE
    assert fwd(_norm(**big), FAKE, 600000, 100000, 1, None, None, need, None) == EWORKSPACE
    rest = (FAKE, FAKE, FAKE, 1 << 40, None)
    assert bwd(_norm(), None, 600, 100, 1, FAKE, FAKE, 600, 100, 1, *rest) == EINVAL
    assert bwd(_norm(), FAKE, 600, 1, 6, FAKE, FAKE, 600, 100, 1, *rest) == EINVAL
    assert bwd(_norm(), FAKE, 600, 100, 1, None, FAKE, 600, 100, 1, *rest) == EINVAL
    assert bwd(_norm(), FAKE, 600, 100, 1, FAKE, None, 600, 100, 1, *rest) == EINVAL
    assert bwd(_norm(), FAKE, 600, 100, 1, FAKE, FAKE, 600, 1, 6, *rest) == EINVAL
    assert bwd(_norm(), FAKE, 600, 100, 1, FAKE, FAKE, 600, 100, 1, FAKE, FAKE, FAKE, 8, None) == EWORKSPACE
    assert lib.conv1d_norm_bwd_workspace_bytes(2, 6, 100, 4, 0, 100, 1) == 0 and lib.conv1d_norm_bwd_workspace_bytes(2, 6, 100, 3, 2, 100, 1) == 0


def _dropout(**kw):
    f = dict(x=FAKE, residual=None, lengths=None, counter=None, x_sn=600, x_sc=100, r_sn=0, r_sc=0, key=1, call=2, p=0.5, N=2, C=6, L=100, dtype=0)
    f.update(kw)
    return ctypes.byref(Dropout(**f))


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), EINVAL), (dict(N=0), EINVAL), (dict(C=0), EINVAL), (dict(L=0), EINVAL), (dict(dtype=2), EINVAL), (dict(p=-0.1), EINVAL), (dict(p=1.1), EINVAL),
    (dict(p=float("nan")), EINVAL), (dict(x=FAKE + 2), EINVAL), (dict(residual=FAKE + 2), EINVAL), (dict(lengths=FAKE + 2), EINVAL), (dict(counter=FAKE + 4), EINVAL),
    (dict(L=(1 << 30) + 1), EUNSUPPORTED), (dict(N=1 << 16, C=1 << 16), EUNSUPPORTED)])
def test_dropout_refusals(lib, bad, status):
    assert lib.conv1d_dropout(_dropout(**bad), FAKE, 600, 100, None) == status


def test_dropout_refusals_of_outputs(lib):
    assert lib.conv1d_dropout(_dropout(), None, 600, 100, None) == EINVAL
    assert lib.conv1d_dropout(_dropout(), FAKE + 2, 600, 100, None) == EINVAL


def test_tensors_of_the_host_are_refused():
    x, t = torch.zeros(2, 6, 10), torch.zeros(2, 10, dtype=torch.int64)
    for call in (lambda: blocks.conv1d_embed_fwd(torch.zeros(5, 6), t), lambda: blocks.conv1d_embed_bwd(x, t, 5), lambda: blocks.conv1d_embed_step(torch.zeros(5, 6), t[0]),
                 lambda: blocks.conv1d_norm_fwd(x, 3), lambda: blocks.conv1d_norm_bwd(x, x, x, 3), lambda: blocks.conv1d_dropout(x, 0.5, 1)):
        with pytest.raises(ValueError):
            call()


def test_orders():
    """Which order a tensor is taken in, as the library does."""
    x = torch.zeros(2, 6, 10)
    assert not blocks._channels_last(x) and blocks._channels_last(x.transpose(1, 2)) and not blocks._channels_last(torch.zeros(2, 1, 10))
    assert blocks._channels_last(torch.zeros(2, 6, 1)) and blocks._channels_last(torch.zeros(2, 1, 1)) and not blocks._channels_last(x[:, :, :1])
    assert blocks._new((2, 6, 10), True, x).stride() == (60, 1, 6) and blocks._new((2, 6, 10), False, x).stride() == (60, 10, 1)
