"""Frequencies and gains without a finite value in the kernel's types: the library refuses them before it touches the device or the
context's contents (a blank block of memory stands in for a context)."""
import ctypes as C

import pytest

from paper_2302_00787_b200 import binding as fb

BADARG, CUDA = -1, -9
P = 1 << 20        # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__ as ge
    ge.build()
    return fb.load_library()


@pytest.mark.parametrize("bad", (dict(gain=1e39), dict(gain=-1e39), dict(base=1e-320),
                                 dict(scaling="linear", factor=1e-310), dict(scaling="ntk", factor=1e-300),
                                 dict(scaling="parts", factor=1e-310, original=4096)))
def test_no_finite_value(lib, bad):
    dm = fb.fsharp_rotate_dims()
    dm.B, dm.L, dm.H, dm.Hk, dm.d = 1, 4, 2, 2, 32
    ctx = C.create_string_buffer(4096)
    rope = fb.make_rope(32, **bad)
    assert lib.fsharp_rotate(ctx, P, 2 * P, None, 0, 0, C.byref(rope), C.byref(dm), 0, 0, 3 * P, 4 * P) == BADARG


def test_large_ones_are_taken(lib):
    """Behind the checks the call looks for its device.  (base 1e-300: the last pair's frequency is its 15/16th power, 1e281, and 2^64 / 2 pi
    times that is finite.)"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are none of the device's")
    dm = fb.fsharp_rotate_dims()
    dm.B, dm.L, dm.H, dm.Hk, dm.d = 1, 4, 2, 2, 32
    ctx = C.create_string_buffer(4096)
    for good in (dict(gain=1e38), dict(base=1e-280), dict(base=1e-300), dict(base=1e300), dict(scaling="ntk", factor=1e300),
                 dict(scaling="ntk", factor=1e-200), dict(scaling="linear", factor=1e300)):
        rope = fb.make_rope(32, **good)
        assert lib.fsharp_rotate(ctx, P, 2 * P, None, 0, 0, C.byref(rope), C.byref(dm), 0, 0, 3 * P, 4 * P) == CUDA, good
