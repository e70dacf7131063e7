"""Bounds of the operators around the layers without a GPU: their kernels, compiled as CPU code by the host model (tests/hostmodel),
run thread by thread with every tensor of a call between inaccessible pages.  An access outside its tensor ends the child
process that makes the call, which has named the case before.  Strided inputs are the halves of larger tensors."""
import ctypes
import os
import random
import sys

import pytest

from blocks_structs import Dropout, Embed, Norm
from test_sequence_bounds_model import Memory, _in_child, _lengths

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "hostmodel"))


@pytest.fixture(scope="module")
def model():
    import build as hostmodel_build
    from paper_2104_08002_amd import binding

    lib, real = ctypes.CDLL(hostmodel_build.build()), binding.load()
    for name in binding.EXPORTS:
        if name.startswith(("conv1d_embed", "conv1d_norm", "conv1d_dropout")):
            getattr(lib, name).restype, getattr(lib, name).argtypes = getattr(real, name).restype, getattr(real, name).argtypes
    return lib


def _embed_case(lib, c):
    N, D, L, V, dtype, wide, last, kind, at_end = c
    mem, e = Memory(at_end), 2 if dtype else 4
    size, number = (8, ctypes.c_long) if wide else (4, ctypes.c_int)
    tokens = mem.tensor(N * L * size, size)
    rnd = random.Random(N * L + V)
    (number * (N * L)).from_address(tokens)[:] = [rnd.choice((0, V - 1, rnd.randrange(V), rnd.randrange(V), -1, V, 2 ** 31 - 1)) for _ in range(N * L)]
    p = Embed(tokens, _lengths(mem, N, L, kind), L, N, D, L, V, dtype, int(wide), 2.0)
    y = mem.tensor(2 * N * D * L * e, e)       # the halves of a wider tensor
    strides = (2 * D * L, 1, 2 * D) if last else (2 * D * L, L, 1)
    y += (D if last else D * L) * e
    st = lib.conv1d_embed_fwd(ctypes.byref(p), mem.tensor(V * D * e, e), y, *strides, None)
    n = lib.conv1d_embed_bwd_workspace_bytes(N, D, L, V, dtype, *strides[1:])
    return st or lib.conv1d_embed_bwd(ctypes.byref(p), y, *strides, mem.tensor(4 * V * D, 4), mem.tensor(n, 256), n, None)


def test_embedding_stays_in_bounds(model):
    rnd = random.Random(5)
    cases = [(N, D, L, V, dt, wide, last, kind, at_end)
             for N, D, L, V in ((1, 1, 1, 1), (2, 3, 1, 5), (3, 64, 1, 300), (1, 15, 515, 5), (2, 17, 130, 256), (1, 65, 129, 70000), (1, 2100, 9, 3), (2, 8, 1100, 2), (2, 9, 30, 20000))
             for dt, wide in ((0, True), (1, False)) for last in (False, True) for kind in (0, 2) for at_end in (True, False)]
    for _ in range(150):
        cases.append((rnd.randint(1, 5), rnd.choice((1, 2, 7, 8, 15, 16, 17, 40, 64, 70, 130)), rnd.choice((1, 2, 7, 8, 33, 127, 128, 300, 513, 700)),
                      rnd.choice((1, 2, 5, 64, 255, 256, 257, 5000)), rnd.randint(0, 1), rnd.random() < 0.5, rnd.random() < 0.5, rnd.randint(0, 2), rnd.random() < 0.5))
    _in_child(cases, lambda c: _embed_case(model, c))


def _norm_case(lib, c):
    N, C, L, G, dtype, last, act, kind, opt, at_end = c
    mem, e = Memory(at_end), 2 if dtype else 4
    rows = N * C * L * e
    wide, dense = ((2 * C * L, 1, 2 * C), (C * L, 1, C)) if last else ((2 * C * L, L, 1), (C * L, L, 1))
    at = (C if last else C * L) * e
    x, y, dy, dx = mem.tensor(2 * rows, e) + at, mem.tensor(rows, e), mem.tensor(2 * rows, e) + at, mem.tensor(rows, e)
    p = Norm(x, mem.tensor(4 * C, 4) if opt else None, mem.tensor(4 * C, 4) if opt else None, _lengths(mem, N, L, kind), *wide, 1e-5, N, C, L, G, dtype, act)
    n = lib.conv1d_norm_fwd_workspace_bytes(N, C, L, G, dtype, *wide[1:])
    stats = mem.tensor(16 * N * G, 8)
    st = lib.conv1d_norm_fwd(ctypes.byref(p), y, *dense, stats if opt else None, mem.tensor(n, 256), n, None)
    n = lib.conv1d_norm_bwd_workspace_bytes(N, C, L, G, dtype, *wide[1:])
    return st or lib.conv1d_norm_bwd(ctypes.byref(p), dy, *wide, stats, dx, *dense, mem.tensor(4 * C, 4) if opt else None, mem.tensor(4 * C, 4) if opt else None,
                                     mem.tensor(n, 256), n, None)


def test_norm_stays_in_bounds(model):
    rnd = random.Random(6)
    cases = [(N, C, L, G, dt, last, act, kind, 1, at_end)
             for N, C, L, G in ((1, 1, 1, 1), (2, 6, 1, 3), (1, 15, 2100, 3), (3, 8, 7, 2), (2, 70, 65, 1), (1, 2100, 3, 4), (1, 3, 20001, 1), (600, 4, 9, 4), (2, 2050, 17, 2), (1, 24, 5, 1), (2, 48, 40, 2), (1030, 24, 3, 1), (1, 120, 1, 5))
             for dt, act in ((0, 1), (1, 2)) for last in (False, True) for kind in (0, 2) for at_end in (True, False)]
    for _ in range(150):
        G = rnd.choice((1, 2, 3, 4))
        cases.append((rnd.randint(1, 5), G * rnd.choice((1, 2, 5, 8, 16, 33)), rnd.choice((1, 2, 7, 8, 33, 127, 128, 300, 513, 2049)), G, rnd.randint(0, 1),
                      rnd.random() < 0.5, rnd.randint(0, 2), rnd.randint(0, 2), rnd.randint(0, 1), rnd.random() < 0.5))
    _in_child(cases, lambda c: _norm_case(model, c))


def _dropout_case(lib, c):
    N, C, L, dtype, kind, opt, at_end = c
    mem, e = Memory(at_end), 2 if dtype else 4
    rows = N * C * L * e
    p = Dropout(mem.tensor(2 * rows, e) + C * L * e, mem.tensor(rows, e) if opt else None, _lengths(mem, N, L, kind), mem.tensor(8, 8) if opt else None, 2 * C * L, L,
                C * L, L, 2 ** 64 - 1, 2 ** 63, 0.3, N, C, L, dtype)
    return lib.conv1d_dropout(ctypes.byref(p), mem.tensor(rows, e), C * L, L, None)


def test_dropout_stays_in_bounds(model):
    rnd = random.Random(7)
    cases = [(rnd.randint(1, 5), rnd.randint(1, 9), rnd.choice((1, 2, 3, 4, 7, 8, 9, 33, 511, 513, 2100)), rnd.randint(0, 1), rnd.randint(0, 2), rnd.randint(0, 1),
              rnd.random() < 0.5) for _ in range(200)]
    _in_child(cases, lambda c: _dropout_case(model, c))
