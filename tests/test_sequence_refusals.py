"""Calls that would race on memory are refused, calls that would not are taken, without a GPU: no kernel is launched here."""
import ctypes

import pytest

from paper_2104_08002_amd import binding

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
