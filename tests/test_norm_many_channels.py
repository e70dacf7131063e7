"""Group norm of as many channels as the header admits, channels next to each other and positions: on the CPU that every gradient is written,
every launch is finite and every access within its tensor (the host model); on the GPU the values."""
import ctypes
import os
import signal
import sys

import pytest
import torch

from blocks_structs import Norm
from test_sequence_bounds_model import Memory, _in_child

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "hostmodel"))

SIZES = [(1, 262144, 3, 1), (1, 300000, 2, 1), (2, 262145, 2, 5), (1, 1 << 20, 2, 2), (1, (1 << 20) - 3, 1, 1)]
MARK = 0xA5


@pytest.fixture(scope="module")
def model():
    import build as hostmodel_build
    from paper_2104_08002_amd import binding

    lib, real = ctypes.CDLL(hostmodel_build.build()), binding.load()
    for name in binding.EXPORTS:
        if name.startswith("conv1d_norm"):
            getattr(lib, name).restype, getattr(lib, name).argtypes = getattr(real, name).restype, getattr(real, name).argtypes
    return lib


def _case(lib, c):
    signal.alarm(60)  # (ends the child: a call of these sizes takes a second or two)
    N, C, L, G, dtype, last, at_end = c
    mem, e = Memory(at_end), 2 if dtype else 4
    rows, strides = N * C * L * e, (C * L, 1, C) if last else (C * L, L, 1)
    x, y, dy, dx, stats = mem.tensor(rows, e), mem.tensor(rows, e), mem.tensor(rows, e), mem.tensor(rows, e), mem.tensor(16 * N * G, 8)
    weight, bias, dweight, dbias = (mem.tensor(4 * C, 4) for _ in range(4))
    p = Norm(x, weight, bias, None, *strides, 1e-5, N, C, L, G, dtype, 0)
    written = ((y, rows), (dx, rows), (dweight, 4 * C), (dbias, 4 * C))
    for at, n in written:
        ctypes.memset(at, MARK, n)
    n = lib.conv1d_norm_fwd_workspace_bytes(N, C, L, G, dtype, *strides[1:])
    st = lib.conv1d_norm_fwd(ctypes.byref(p), y, *strides, stats, mem.tensor(n, 256), n, None)
    n = lib.conv1d_norm_bwd_workspace_bytes(N, C, L, G, dtype, *strides[1:])
    st = st or lib.conv1d_norm_bwd(ctypes.byref(p), dy, *strides, stats, dx, *strides, dweight, dbias, mem.tensor(n, 256), n, None)
    for i, (at, n) in enumerate(written):
        left = torch.frombuffer((ctypes.c_uint8 * n).from_address(at), dtype=torch.uint8) == MARK
        st = st or (100 + i if left.view(-1, 4 if i > 1 else e).all(1).any() else 0)
    return st


@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
def test_all_is_written_and_nothing_else(model, last):
    _in_child([(*s, i % 2, last, i % 2 == 0) for i, s in enumerate(SIZES)], lambda c: _case(model, c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("last", [False, True], ids=["positions", "channels"])
@pytest.mark.parametrize("N,C,L,G", SIZES)
def test_values(dtype, last, N, C, L, G):
    from paper_2104_08002_amd import blocks
    from test_gpu_blocks import _check_norm, _gen, _lengths, _norm_inputs

    x, dy, weight, bias = _norm_inputs(_gen(C), N, C, L, dtype)
    _check_norm(blocks, x, dy, G, weight, bias, "relu", None, last)
    _check_norm(blocks, x, dy, G, None, bias, "silu", _lengths("ragged", N, L), last)
