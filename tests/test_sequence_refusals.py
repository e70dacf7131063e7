"""Calls that would race on memory are refused, calls that would not are taken, without a GPU: no kernel is launched here."""
import ctypes
import random

import pytest
import torch

from paper_2104_08002_amd import binding, sequence

FAKE = 0x10000          # never dereferenced: every call below fails its checks
EINVAL = -1


@pytest.mark.parametrize("norm,types", [(FAKE, (0, 0)), (FAKE + 396, (0, 0)), (FAKE + 800, (0, 0)), (FAKE + 4, (1, 1)), (FAKE + 196, (1, 0))])
def test_a_norm_within_a_gradient_is_refused(norm, types):
    """Every workgroup reads the norm while others scale what lies there."""
    lib = binding.load()
    data, counts = (ctypes.c_void_p * 2)(FAKE, FAKE + 500), (ctypes.c_size_t * 2)(100, 100)
    assert lib.conv1d_grad_clip(data, counts, (ctypes.c_int * 2)(*types), 2, norm, 1.0, None) == EINVAL
    one = 0 if norm < FAKE + 500 else 1
    assert lib.conv1d_grad_clip((ctypes.c_void_p * 1)(data[one]), (ctypes.c_size_t * 1)(100), (ctypes.c_int * 1)(types[one]), 1, norm, 1.0, None) == EINVAL


def test_a_norm_beside_a_gradient_is_taken():
    lib = binding.load()
    empty = (ctypes.c_size_t * 1)(0)
    assert lib.conv1d_grad_clip((ctypes.c_void_p * 1)(FAKE), empty, (ctypes.c_int * 1)(0), 1, FAKE, 1.0, None) == 0   # nothing there: nothing is launched


def _bytes_of(t):
    at = t.data_ptr() + t.element_size() * sum((torch.arange(n) * s).view([-1] + [1] * (t.dim() - 1 - i)) for i, (n, s) in enumerate(zip(t.shape, t.stride())))
    return {int(a) + k for a in at.flatten() for k in range(t.element_size())}


def _refused(out, t):
    try:
        sequence._apart(out, (None, t))
    except ValueError:
        return True
    return False


def test_an_output_beside_an_input_in_one_projection_is_taken():
    """The halves of a projection, of channels that lie between each other, of the rows of single positions."""
    for dtype in (torch.float32, torch.bfloat16):
        xz = torch.zeros(3, 8, 10, dtype=dtype)
        assert not _refused(xz[:, :4], xz[:, 4:]) and not _refused(xz[:, 4:], xz[:, :4]) and not _refused(xz[:, 2:4], xz[:, 4:5])
        assert not _refused(xz[:, :4], xz.view(3, 2, 4, 10)[:, 1])
        pairs = xz.view(3, 4, 2, 10)
        assert not _refused(pairs[:, :, 0], pairs[:, :, 1]) and not _refused(pairs[:, 1:3, 1], pairs[:, :, 0])
        one = torch.zeros(3, 8, dtype=dtype)
        assert not _refused(one[:, :4], one[:, 4:]) and not _refused(one[:, 4:], one[:, :4].view(3, 2, 2))
        for out, t in ((xz[:, :5], xz[:, 4:]), (xz[:, 4:], xz[:, :5]), (xz[:, :4], xz), (xz[1:], xz[:2]), (xz, xz), (pairs[:, :, 0], xz[:, 1:3]),
                       (xz[:, :4], xz[0, 0]), (one[:, :5], one[:, 4:]), (xz[:, :4], xz[:, 3:4])):
            assert _refused(out, t)


def test_no_output_within_an_input_is_taken():
    rnd = random.Random(3)
    flat, taken = torch.zeros(4096, dtype=torch.float32), 0
    for _ in range(3000):
        views = []
        for dtype in (torch.float32, rnd.choice((torch.float32, torch.bfloat16))):
            shape = [rnd.randint(1, 4) for _ in range(rnd.randint(2, 3))]
            strides = [rnd.choice((0, 1, 2, 3, 4, 8, 16, 24)) for _ in shape[:-1]] + [1]
            views.append(flat.view(dtype).as_strided(shape, strides, rnd.randint(0, 24)))
        out, t = views
        if not _refused(out, t):
            taken += 1
            assert not _bytes_of(out) & _bytes_of(t), (out.shape, out.stride(), out.storage_offset(), t.shape, t.stride(), t.storage_offset(), t.dtype)
    assert taken > 300
