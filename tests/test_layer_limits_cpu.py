"""Arguments of the layer operators at the ends of their ranges are refused before anything is queued (no GPU: the
pointers below are never dereferenced)."""

import ctypes

import pytest

FAKE = 0x7F0000000000
EINVAL = -1


@pytest.fixture(scope="module")
def b():
    import torch  # noqa: F401
    from paper_2606_05613_amd import bkmoo
    return bkmoo


def at(i):
    return FAKE + (i << 40)


def adamw(b, places, eps=1e-8, dt=0):
    """bkmoo_adamw over tensors at (first byte, elements) of memory of their own."""
    t = (b._Tensor * len(places))(*[(at(0) + p, n, 1) for p, n in places])
    hp = b._AdamwHparams(0.1, 0.9, 0.99, eps, 0.0, 1, 0)
    return b._lib.bkmoo_adamw(len(places), t, dt, sum(n for _, n in places), at(1), 0, 0, at(2), at(3), None, 0, None,
                              ctypes.byref(hp), None, None)


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1.17e-38])
def test_eps_below_the_normal_numbers(b, eps):
    """The step's reciprocal takes a denormal number for zero."""
    assert adamw(b, [(0, 64)], eps=eps) == EINVAL
