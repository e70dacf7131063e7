"""Argument checks and plans of the sequence operators, without a GPU: no kernel is launched here."""
import ctypes

import pytest

from paper_2104_08002_amd import binding, sequence
from sequence_structs import Causal, Scan

FAKE = 0x10000          # never dereferenced: every call below fails its checks
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _causal(**kw):
    f = dict(x=FAKE, w=FAKE, bias=None, init=None, lengths=None, x_sn=1000, x_sc=100, N=2, C=3, L=100, S=4, dtype=0, flags=0)
    f.update(kw)
    return ctypes.byref(Causal(**f))


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(N=0), EINVAL), (dict(C=0), EINVAL), (dict(L=0), EINVAL), (dict(S=0), EINVAL), (dict(L=-5), EINVAL),
    (dict(dtype=2), EINVAL), (dict(flags=2), EINVAL), (dict(x=FAKE + 2), EINVAL), (dict(x=FAKE + 1, dtype=1), EINVAL), (dict(bias=FAKE + 2), EINVAL),
    (dict(init=FAKE + 2), EINVAL), (dict(lengths=FAKE + 1), EINVAL), (dict(S=9), EUNSUPPORTED), (dict(L=(1 << 30) + 1), EUNSUPPORTED),
    (dict(N=1 << 20, C=1 << 20), EUNSUPPORTED)])
def test_causal_refusals(lib, bad, status):
    assert lib.conv1d_causal_fwd(_causal(**bad), FAKE, 1, 1, None, None) == status
    assert lib.conv1d_causal_bwd(_causal(**bad), FAKE, 1, 1, None, FAKE, None, None, None, None, 0, None) == status
    if bad.get("L", 1) == 1:
        assert lib.conv1d_causal_step(_causal(**{"L": 1, **bad}), FAKE, FAKE, 1, None) in (status, EINVAL)


def test_causal_refusals_of_outputs(lib):
    assert lib.conv1d_causal_fwd(_causal(), None, 1, 1, None, None) == EINVAL
    assert lib.conv1d_causal_fwd(_causal(), FAKE + 2, 1, 1, None, None) == EINVAL
    assert lib.conv1d_causal_fwd(_causal(), FAKE, 1, 1, FAKE + 2, None) == EINVAL
    bwd = lib.conv1d_causal_bwd
    assert bwd(_causal(), None, 1, 1, None, FAKE, FAKE, None, None, FAKE, 1 << 20, None) == EINVAL
    assert bwd(_causal(), FAKE, 1, 1, None, None, FAKE, None, None, FAKE, 1 << 20, None) == EINVAL
    assert bwd(_causal(), FAKE, 1, 1, None, FAKE, None, FAKE, None, FAKE, 1 << 20, None) == EINVAL   # a bias gradient needs dw
    assert bwd(_causal(), FAKE, 1, 1, None, FAKE, FAKE, None, None, None, 0, None) == EWORKSPACE
    need = lib.conv1d_causal_bwd_workspace_bytes(2, 3, 100, 4)
    assert need == 4 * 3 * 5 * 2 * 1
    assert bwd(_causal(), FAKE, 1, 1, None, FAKE, FAKE, None, None, FAKE, need - 1, None) == EWORKSPACE
    assert lib.conv1d_causal_bwd_workspace_bytes(2, 3, 100, 9) == 0
    step = lib.conv1d_causal_step
    assert step(_causal(L=2), FAKE, FAKE, 1, None) == EINVAL
    assert step(_causal(L=1), None, FAKE, 1, None) == EINVAL
    assert step(_causal(L=1, init=FAKE), FAKE, FAKE, 1, None) == EINVAL
    assert step(_causal(L=1), FAKE, None, 1, None) == EINVAL


def _scan(**kw):
    f = dict(x=FAKE, dt=FAKE, B=FAKE, C=FAKE, z=None, A=FAKE, skip=None, dt_bias=None, init=None, lengths=None, N=2, D=6, L=100, S=16, G=2, dtype=0, flags=1)
    f.update(kw)
    return ctypes.byref(Scan(**f))


def _scan_bwd(lib, p, *, dy=FAKE, saved=FAKE, dx=FAKE, dA=FAKE, dskip=None, dz=None, ddt_bias=None, ws=FAKE, ws_bytes=1 << 40):
    return lib.conv1d_scan_bwd(p, dy, 1, 1, None, saved, dx, FAKE, dA, FAKE, FAKE, dskip, dz, ddt_bias, None, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), EINVAL), (dict(dt=None), EINVAL), (dict(A=None), EINVAL), (dict(B=None), EINVAL), (dict(C=None), EINVAL), (dict(N=0), EINVAL),
    (dict(D=0), EINVAL), (dict(L=0), EINVAL), (dict(S=0), EINVAL), (dict(G=0), EINVAL), (dict(G=4), EINVAL), (dict(dtype=3), EINVAL), (dict(flags=4), EINVAL),
    (dict(dt=FAKE + 2), EINVAL), (dict(B=FAKE + 1, dtype=1), EINVAL), (dict(A=FAKE + 2), EINVAL), (dict(skip=FAKE + 2), EINVAL), (dict(init=FAKE + 1), EINVAL),
    (dict(S=65), EUNSUPPORTED), (dict(N=1 << 15, D=1 << 11), EUNSUPPORTED), (dict(L=(1 << 30) + 1), EUNSUPPORTED)])
def test_scan_refusals(lib, bad, status):
    assert lib.conv1d_scan_fwd(_scan(**bad), FAKE, 1, 1, None, None, FAKE, 1 << 40, None) == status
    assert _scan_bwd(lib, _scan(**bad)) == status
    if bad.get("L", 1) == 1:
        assert lib.conv1d_scan_step(_scan(**{"L": 1, **bad}), FAKE, FAKE, 1, None) in (status, EINVAL)


def test_scan_refusals_of_outputs(lib):
    fwd = lib.conv1d_scan_fwd
    assert fwd(_scan(), None, 1, 1, None, None, FAKE, 1 << 40, None) == EINVAL
    assert fwd(_scan(), FAKE, 1, 1, None, FAKE + 4, FAKE, 1 << 40, None) == EINVAL          # saved: 16-byte aligned
    assert fwd(_scan(), FAKE, 1, 1, None, None, FAKE + 16, 1 << 40, None) == EINVAL         # workspace: 256-byte aligned
    need = lib.conv1d_scan_fwd_workspace_bytes(2, 6, 1000, 16, 2)
    assert need > 0 and fwd(_scan(L=1000), FAKE, 1, 1, None, None, FAKE, need - 1, None) == EWORKSPACE
    assert fwd(_scan(L=1000), FAKE, 1, 1, None, None, None, 0, None) == EWORKSPACE
    assert _scan_bwd(lib, _scan(), dy=None) == EINVAL
    assert _scan_bwd(lib, _scan(), saved=None) == EINVAL
    assert _scan_bwd(lib, _scan(), dA=None) == EINVAL
    assert _scan_bwd(lib, _scan(), dskip=FAKE) == EINVAL                                    # no skip in the call
    assert _scan_bwd(lib, _scan(), ddt_bias=FAKE) == EINVAL
    assert _scan_bwd(lib, _scan(), dz=FAKE) == EINVAL                                       # no gate, and a gate without its gradient
    assert _scan_bwd(lib, _scan(z=FAKE)) == EINVAL
    assert _scan_bwd(lib, _scan(), ws_bytes=lib.conv1d_scan_bwd_workspace_bytes(2, 6, 100, 16, 2) - 1) == EWORKSPACE
    step = lib.conv1d_scan_step
    assert step(_scan(L=1), None, FAKE, 1, None) == EINVAL
    assert step(_scan(L=2), FAKE, FAKE, 1, None) == EINVAL
    assert step(_scan(L=1, lengths=FAKE), FAKE, FAKE, 1, None) == EINVAL


def test_scan_sizes(lib):
    assert lib.conv1d_scan_saved_bytes(2, 6, 100, 16) == 4 * 2 * 13 * 6 * 16                # every 8 steps
    assert lib.conv1d_scan_saved_bytes(2, 6, 8, 5) == 4 * 2 * 1 * 6 * 8                     # states padded to 4, 8, 16, 32 or 64
    assert lib.conv1d_scan_fwd_workspace_bytes(64, 2048, 1000, 16, 1) == 0                  # rows enough: not cut
    assert lib.conv1d_scan_fwd_workspace_bytes(1, 3, 100, 16, 1) == 0                       # a few tiles
    for bad in ((0, 6, 100, 16, 2), (2, 6, 100, 65, 2), (2, 6, 100, 16, 4)):
        assert lib.conv1d_scan_fwd_workspace_bytes(*bad) == 0 and lib.conv1d_scan_bwd_workspace_bytes(*bad) == 0


def test_gradient_refusals(lib):
    data, counts, types = (ctypes.c_void_p * 2)(FAKE, FAKE + 400), (ctypes.c_size_t * 2)(100, 100), (ctypes.c_int * 2)(0, 0)
    norm, clip = lib.conv1d_grad_norm, lib.conv1d_grad_clip
    assert lib.conv1d_grad_norm_workspace_bytes(counts, 2) == 16 and lib.conv1d_grad_norm_workspace_bytes(counts, 0) == 0
    assert norm(data, counts, types, -1, 2, FAKE, FAKE, 1 << 20, None) == EINVAL
    assert norm(None, counts, types, 2, 2, FAKE, FAKE, 1 << 20, None) == EINVAL
    assert norm(data, counts, types, 2, 1, FAKE, FAKE, 1 << 20, None) == EINVAL             # kinds: 2 and the maximum
    assert norm(data, counts, types, 2, 2, None, FAKE, 1 << 20, None) == EINVAL
    assert norm(data, counts, types, 2, 2, FAKE, FAKE + 4, 1 << 20, None) == EINVAL
    assert norm(data, counts, types, 2, 2, FAKE, FAKE, 15, None) == EWORKSPACE
    assert norm((ctypes.c_void_p * 2)(FAKE, None), counts, types, 2, 2, FAKE, FAKE, 1 << 20, None) == EINVAL
    assert norm((ctypes.c_void_p * 2)(FAKE, FAKE + 401), counts, types, 2, 2, FAKE, FAKE, 1 << 20, None) == EINVAL
    assert norm(data, counts, (ctypes.c_int * 2)(0, 5), 2, 2, FAKE, FAKE, 1 << 20, None) == EINVAL
    assert norm(data, (ctypes.c_size_t * 2)(1, (1 << 37) + 1), types, 2, 2, FAKE, FAKE, 1 << 50, None) == EINVAL
    assert clip(data, counts, types, 2, None, 1.0, None) == EINVAL
    assert clip(data, counts, types, 2, FAKE, -1.0, None) == EINVAL
    assert clip(data, counts, types, 2, FAKE, float("nan"), None) == EINVAL
    assert clip((ctypes.c_void_p * 2)(FAKE, FAKE + 396), counts, types, 2, FAKE, 1.0, None) == EINVAL   # the last element of one is the first of the other
    assert clip(data, counts, types, 0, FAKE, 1.0, None) == 0


def test_tensors_on_the_host_are_refused():
    import torch

    from paper_2104_08002_amd import gradients

    x, w = torch.zeros(2, 3, 10), torch.zeros(3, 4)
    for call in (lambda: sequence.conv1d_causal_fwd(x, w), lambda: sequence.conv1d_causal_bwd(x, x, w), lambda: sequence.conv1d_causal_step(x[:, :, 0], w, x),
                 lambda: sequence.conv1d_scan_fwd(x, x, w, x, x), lambda: gradients.conv1d_grad_norm([x]), lambda: gradients.conv1d_grad_clip([x], 1.0)):
        with pytest.raises(ValueError):
            call()


def test_workspaces_elsewhere_are_refused():
    import torch

    room, here, there = sequence._room, torch.device("cpu"), torch.device("meta")
    assert room(None, 0, here) is None and room(None, 8, here).numel() == 8
    assert sequence._bytes(room(torch.empty(3), 8, here)) == 12
    for bad in (torch.empty(64, device=there), torch.empty(8, 8)[:, 0]):
        with pytest.raises(ValueError):
            room(bad, 8, here)


def test_structures_are_packed_as_declared():
    """The binding packs the structures by itself: the same size and places as a C compiler's."""
    for packed, declared in ((sequence._CAUSAL, Causal), (sequence._SCAN, Scan)):
        values = [1000 + i for i in range(len(declared._fields_))]
        made = declared.from_buffer_copy(packed.pack(*values))
        assert packed.size == ctypes.sizeof(declared) and [getattr(made, k) for k, _ in declared._fields_] == values
