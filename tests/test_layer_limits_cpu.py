"""Arguments of the layer operators at the ends of their ranges are refused before anything is queued (no GPU: the
pointers below are never dereferenced)."""

import ctypes
import random

import pytest

FAKE = 0x7F0000000000
EINVAL, EUNSUPPORTED = -1, -2


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


def apart(sizes, gap=0, es=4):
    """Places of tensors one after another, `gap` bytes apart."""
    out, p = [], 0
    for n in sizes:
        out.append((p, n))
        p += n * es + gap
    return out


def test_tensors_over_one_another(b):
    """Two tensors that share an element would be stepped at once: refused, in whatever order they come and
    however many there are; neighbours are not."""
    gen = random.Random(5)
    for many in (2, 3, 50, 1024, 1025, 3000):
        sizes = [gen.choice([0, 1, 2, 300]) for _ in range(many - 2)]
        far = sum(sizes) * 4 + 4096
        for first, second in (((far, 64), (far, 64)),             # one tensor twice
                              ((far, 64), (far + 63 * 4, 5)),     # its last element
                              ((far, 64), (far + 8, 1)),          # one within another
                              ((far + 40, 64), (far, 11))):
            for where in ("as they come", "behind", "mixed"):
                places = apart(sizes)
                places = [first] + places + [second] if where == "as they come" else places + [first, second]
                if where == "mixed":
                    gen.shuffle(places)
                assert adamw(b, places) == EINVAL, (many, first, second, where)


def test_empty_tensors_lie_over_nothing(b):
    t = (b._Tensor * 3)((at(0), 0, 1), (at(0), 0, 1), (0, 0, 1))
    hp = b._AdamwHparams(0.1, 0.9, 0.99, 1e-8, 0.0, 1, 0)
    assert b._lib.bkmoo_adamw(3, t, 0, 0, None, 0, 0, None, None, None, 0, None, ctypes.byref(hp), None, None) == 0


def test_norm_sizes_past_the_limits(b):
    """More rows or columns than the norms take, up to the ends of int64: refused by the size query too."""
    L, size = b._lib, ctypes.c_size_t(0)
    for M, D in ((255 << 32, 64), (1 << 31, 64), ((1 << 63) - 1, 64), (4, 32769), (4, 1 << 61), (4, (1 << 63) - 1)):
        assert L.bkmoo_residual_norm_workspace_size(M, D, 1, ctypes.byref(size)) == EUNSUPPORTED, (M, D)
    assert L.bkmoo_residual_norm_workspace_size((1 << 31) - 1, 32768, 16, ctypes.byref(size)) == 0
    assert size.value <= (256 + 16) * 2 * 32768 * 4 + 256
    for dt, D in ((0, 1 << 61), (0, 1 << 62), (1, 1 << 62), (1, (1 << 63) - 1), (0, (1 << 63) - 1)):
        assert L.bkmoo_residual_norm_forward(0, D, dt, at(0), at(1), at(2), None, None, 1.0, 1e-6, at(3), at(4),
                                             None) == EUNSUPPORTED, D


def test_adamw_sizes_past_the_limits(b):
    """Elements whose blocks of 256 or bytes would overflow 64 bits are refused, in the count of blocks too."""
    blocks = ctypes.c_int64(0)
    for n in ((1 << 63) - 1, (1 << 63) - 255, 1 << 48):
        t = (b._Tensor * 1)((at(0), n, 1))
        assert b._lib.bkmoo_adamw_blocks(1, t, ctypes.byref(blocks)) == EUNSUPPORTED, n
        hp = b._AdamwHparams(0.1, 0.9, 0.99, 1e-8, 0.0, 1, 0)
        assert b._lib.bkmoo_adamw(1, t, 0, n, at(1), 0, 0, at(2), at(3), None, 0, None, ctypes.byref(hp), None,
                                  None) == EUNSUPPORTED, n
    t = (b._Tensor * 1)((at(0), 1 << 35, 1))
    assert b._lib.bkmoo_adamw_blocks(1, t, ctypes.byref(blocks)) == 0 and blocks.value == 1 << 27


@pytest.mark.parametrize("scale,eps", [(1e39, 1e-6), (-1e300, 1e-6), (1.0, 1e39), (1.0, 1e-46)])
def test_norm_scalars_that_fp32_cannot_hold(b, scale, eps):
    """Finite in 64 bits, infinite (or zero, where it was not) in the kernels' 32."""
    assert b._lib.bkmoo_residual_norm_forward(0, 64, 0, at(0), at(1), at(2), None, None, scale, eps, at(3), at(4),
                                              None) == EINVAL


@pytest.mark.parametrize("bad", [dict(lr=1e39), dict(lr=1e20, wd=1e20), dict(lr=1e30, b1=1 - 1e-12)])
def test_adamw_scalars_that_fp32_cannot_hold(b, bad):
    """The rate, its product with the decay, or the rate over 1 - beta1^t."""
    v = dict(lr=0.1, b1=0.9, wd=0.0)
    v.update(bad)
    t = (b._Tensor * 1)((at(0), 64, 1))
    hp = b._AdamwHparams(v["lr"], v["b1"], 0.99, 1e-8, v["wd"], 1, 0)
    assert b._lib.bkmoo_adamw(1, t, 0, 64, at(1), 0, 0, at(2), at(3), None, 0, None, ctypes.byref(hp), None,
                              None) == EINVAL
