"""Bounds of the sequence operators without a GPU: their kernels, compiled as CPU code by the host model (tests/hostmodel),
run thread by thread with every tensor of a call between inaccessible pages.  An access outside its tensor ends the child
process that makes the call, which has named the case before.  Strided inputs are the halves of larger tensors."""
import ctypes
import mmap
import os
import random
import sys

import pytest

from sequence_structs import Causal, Scan

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "hostmodel"))

PAGE, GUARD = mmap.PAGESIZE, 1 << 24


@pytest.fixture(scope="module")
def model():
    import build as hostmodel_build
    from paper_2104_08002_amd import binding

    lib, real = ctypes.CDLL(hostmodel_build.build()), binding.load()
    for name in binding.EXPORTS:
        if name.startswith(("conv1d_causal", "conv1d_scan", "conv1d_grad")):
            getattr(lib, name).restype, getattr(lib, name).argtypes = getattr(real, name).restype, getattr(real, name).argtypes
    return lib


class Memory:
    """Tensors that end (at_end) or begin at an inaccessible page."""

    def __init__(self, at_end):
        self.at_end, self.libc = at_end, ctypes.CDLL(None, use_errno=True)
        self.libc.mmap.restype = ctypes.c_void_p
        self.libc.mmap.argtypes = [ctypes.c_void_p, ctypes.c_size_t] + [ctypes.c_int] * 3 + [ctypes.c_long]
        self.libc.mprotect.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]

    def tensor(self, nbytes, align=1):
        body = max(PAGE, -(-nbytes // PAGE) * PAGE)
        at = self.libc.mmap(None, body + 2 * GUARD, 0, mmap.MAP_PRIVATE | mmap.MAP_ANONYMOUS | 0x4000, -1, 0)
        assert at not in (None, ctypes.c_void_p(-1).value)
        assert self.libc.mprotect(at + GUARD, body, mmap.PROT_READ | mmap.PROT_WRITE) == 0
        return at + GUARD + ((body - nbytes) // align * align if self.at_end else 0)


def _in_child(cases, call):
    """Runs call(case) for every case in a child process; fails with the case that ended it."""
    r, w = os.pipe()
    pid = os.fork()
    if pid == 0:
        code = 3
        try:
            os.close(r)
            for i, c in enumerate(cases):
                os.write(w, b"%d\n" % i)
                st = call(c)
                if st != 0:
                    os.write(w, b"status %d\n" % st)
                    os._exit(4)
            code = 0
        finally:
            os._exit(code)
    os.close(w)
    said = b""
    while chunk := os.read(r, 1 << 16):
        said += chunk
    os.close(r)
    _, status = os.waitpid(pid, 0)
    lines = said.decode().splitlines()
    last = [s for s in lines if s.isdigit()]
    assert status == 0, f"wait status {status} ({lines[-1:]}): {cases[int(last[-1])] if last else 'before the first case'}"


def _lengths(mem, N, L, kind):
    if kind == 0:
        return None
    at = mem.tensor(4 * N, 4)
    values = [L if kind == 1 else (0, L, L // 2, 1, -5, L + 9)[i % 6] for i in range(N)]
    (ctypes.c_int * N).from_address(at)[:] = values
    return at


def _causal_case(lib, c):
    N, C, L, S, dtype, kind, opt, at_end = c
    mem, e = Memory(at_end), 2 if dtype else 4
    x_all = mem.tensor(2 * N * C * L * e, e)
    state = [mem.tensor(N * C * (S - 1) * e, e) if opt and S > 1 else None for _ in range(4)]
    p = Causal(x_all + C * L * e, mem.tensor(C * S * e, e), mem.tensor(4 * C, 4) if opt else None, state[0], _lengths(mem, N, L, kind), 2 * C * L, L,
                  N, C, L, S, dtype, opt)
    y, dy, dx = mem.tensor(N * C * L * e, e), mem.tensor(N * C * L * e, e), mem.tensor(N * C * L * e, e)
    st = lib.conv1d_causal_fwd(ctypes.byref(p), y, C * L, L, state[1], None)
    n = lib.conv1d_causal_bwd_workspace_bytes(N, C, L, S)
    st = st or lib.conv1d_causal_bwd(ctypes.byref(p), dy, C * L, L, state[2], dx, mem.tensor(4 * C * S, 4), mem.tensor(4 * C, 4), state[3],
                                     mem.tensor(n, 4), n, None)
    if L == 1:
        p.init = p.lengths = None
        st = st or lib.conv1d_causal_step(ctypes.byref(p), mem.tensor(N * C * (S - 1) * e, e) if S > 1 else None, y, C, None)
    return st


def test_causal_stays_in_bounds(model):
    rnd = random.Random(5)
    cases = [(N, C, L, S, dt, kind, 1, at_end) for N, C, L, S in ((1, 1, 1, 1), (2, 3, 1, 4), (1, 2, 7, 8), (3, 5, 8, 4), (2, 3, 9, 3), (1, 2, 512, 4),
                                                                  (2, 2, 513, 2), (1, 2, 2049, 8), (1, 1100, 4097, 4))
             for dt in (0, 1) for kind in (0, 2) for at_end in (True, False)]
    for _ in range(300):
        cases.append((rnd.randint(1, 7), rnd.randint(1, 9), rnd.choice((1, 2, 5, 31, 64, 100, 511, 700, 2100)), rnd.randint(1, 8), rnd.randint(0, 1),
                      rnd.randint(0, 2), rnd.randint(0, 1), rnd.random() < 0.5))
    _in_child(cases, lambda c: _causal_case(model, c))


def test_causal_of_many_rows_stays_in_bounds(model):
    """Rows enough for four steps a lane backwards, and for eight."""
    cases = [(N, C, L, S, dt, kind, 1, at_end) for N, C, L, S in ((2, 1100, 2049, 2), (2, 1030, 2060, 8), (1, 4096, 600, 5), (2, 1100, 4099, 3), (1, 1400, 8200, 8))
             for dt, kind, at_end in ((0, 0, True), (1, 2, True), (0, 2, False))]
    _in_child(cases, lambda c: _causal_case(model, c))


def _scan_case(lib, c):
    N, Dg, L, S, G, dtype, kind, opt, at_end = c
    D, mem, e = G * Dg, Memory(at_end), 2 if dtype else 4
    rows = N * D * L * e

    def floats(n, want=True):
        return mem.tensor(4 * n, 4) if want else None

    xz, bc, dt = mem.tensor(2 * rows, e), mem.tensor(2 * N * G * S * L * e, e), mem.tensor(rows, e)
    gate = bool(opt & 1)
    p = Scan(xz, dt, bc, bc + G * S * L * e, xz + D * L * e if gate else None, floats(D * S), floats(D, opt & 2), floats(D, opt & 2),
                floats(N * D * S, opt & 4), _lengths(mem, N, L, kind), 2 * D * L, L, D * L, L, 2 * D * L, L, 2 * G * S * L, S * L, L, 2 * G * S * L,
                S * L, L, N, D, L, S, G, dtype, 1)
    y, ns = mem.tensor(rows, e), lib.conv1d_scan_saved_bytes(N, D, L, S)
    saved, n = mem.tensor(ns, 16), lib.conv1d_scan_fwd_workspace_bytes(N, D, L, S, G)
    st = lib.conv1d_scan_fwd(ctypes.byref(p), y, D * L, L, floats(N * D * S, opt & 4), saved, mem.tensor(n, 256) if n else None, n, None)
    n = lib.conv1d_scan_bwd_workspace_bytes(N, D, L, S, G)
    grad = [mem.tensor(rows, e) for _ in range(3)]
    states = [mem.tensor(N * G * S * L * e, e) for _ in range(2)]
    st = st or lib.conv1d_scan_bwd(ctypes.byref(p), mem.tensor(rows, e), D * L, L, floats(N * D * S, opt & 4), saved, grad[0], grad[1], floats(D * S),
                                   *states, floats(D, opt & 2), grad[2] if gate else None, floats(D, opt & 2), floats(N * D * S, opt & 4),
                                   mem.tensor(n, 256), n, None)
    if L == 1:
        p.init = p.lengths = None
        p.b_sg = p.c_sg = S  # one position: states contiguous
        p.b_sn = p.c_sn = 2 * G * S
        p.x_sn = p.z_sn = 2 * D
        p.dt_sn = D
        st = st or lib.conv1d_scan_step(ctypes.byref(p), floats(N * D * S), y, D, None)
    return st


def test_scan_stays_in_bounds(model):
    rnd = random.Random(6)
    cases = [(N, Dg, L, S, G, dt, kind, 7, at_end)
             for N, Dg, L, S, G in ((1, 1, 1, 1, 1), (2, 3, 1, 16, 2), (1, 65, 17, 16, 1), (2, 16, 64, 16, 1), (1, 9, 33, 5, 3), (1, 70, 16, 64, 1),
                                    (1, 5, 600, 16, 1), (2, 3, 1025, 3, 2), (1, 1, 2000, 33, 1))
             for dt in (0, 1) for kind in (0, 2) for at_end in (True, False)]
    for _ in range(120):
        cases.append((rnd.randint(1, 4), rnd.choice((1, 2, 4, 5, 16, 17, 64, 70)), rnd.choice((1, 2, 15, 16, 31, 63, 64, 65, 130, 300, 777)),
                      rnd.choice((1, 4, 5, 8, 16, 17, 32, 64)), rnd.randint(1, 3), rnd.randint(0, 1), rnd.randint(0, 2), rnd.randint(0, 7),
                      rnd.random() < 0.5))
    _in_child(cases, lambda c: _scan_case(model, c))


def test_scan_of_many_segments_stays_in_bounds(model):
    """More segments than are joined at once."""
    cases = [(N, Dg, L, S, 1, dt, kind, 7, at_end) for N, Dg, L, S in ((1, 1, 40000, 16), (2, 1, 20000, 64), (1, 1, 36000, 24))
             for dt, kind, at_end in ((0, 0, True), (1, 2, True), (0, 2, False))]
    _in_child(cases, lambda c: _scan_case(model, c))


def _grad_case(lib, c):
    sizes, max_norm, at_end = c
    mem, n = Memory(at_end), len(sizes)
    dtypes = [i % 2 for i in range(n)]
    data = (ctypes.c_void_p * n)(*[mem.tensor(s * (2 if d else 4), 2 if d else 4) for s, d in zip(sizes, dtypes)])
    counts, types = (ctypes.c_size_t * n)(*sizes), (ctypes.c_int * n)(*dtypes)
    need = lib.conv1d_grad_norm_workspace_bytes(counts, n)
    norm = mem.tensor(4, 4)
    st = lib.conv1d_grad_norm(data, counts, types, n, 2 * max_norm, norm, mem.tensor(need, 8), need, None)
    ctypes.c_float.from_address(norm).value = 5.0
    return st or lib.conv1d_grad_clip(data, counts, types, n, norm, 1.0, None)


def test_gradients_stay_in_bounds(model):
    rnd = random.Random(7)
    cases = [([], 1, True), ([1], 1, True), ([0, 0], 0, True), ([16384, 16385, 7, 0, 8], 1, True), ([3] * 161, 0, False), ([5] * 330, 1, True)]
    cases += [([rnd.choice((0, 1, 7, 8, 9, 100, 2047, 2048, 20000)) for _ in range(rnd.randint(1, 9))], rnd.randint(0, 1), rnd.random() < 0.5)
              for _ in range(40)]
    _in_child(cases, lambda c: _grad_case(model, c))
