"""The layer operators refuse bad arguments before anything is queued (no GPU: the
pointers below are never dereferenced)."""

import ctypes

import pytest

FAKE = 0x7F0000000000


@pytest.fixture(scope="module")
def b():
    import torch  # noqa: F401
    from paper_2606_05613_amd import bkmoo
    return bkmoo


def at(i):
    return FAKE + (i << 32)


def rows(*r):
    return (ctypes.c_int64 * len(r))(*r)


def test_norm_arguments(b):
    L = b._lib
    f = lambda M=4, D=64, dt=0, r=at(0), y=at(1), w=at(2), p=None, g=None, c=1.0, e=1e-6, o=at(3), n=at(4): \
        L.bkmoo_residual_norm_forward(M, D, dt, r, y, w, p, g, c, e, o, n, None)  # noqa: E731
    assert f(M=0) == 0  # nothing to do
    for bad in (dict(M=-1), dict(D=0), dict(dt=2), dict(r=None), dict(y=None), dict(w=None), dict(o=None), dict(n=None),
                dict(c=float("inf")), dict(e=-1e-9), dict(e=float("nan")), dict(y=at(1) + 2), dict(g=at(5) + 1),
                dict(n=at(1)), dict(o=at(0) + 16), dict(n=at(3) + 64), dict(n=at(2))):
        assert f(**bad) == -1, bad
    assert f(D=16385) == -2 and f(D=16385, dt=1, M=0) == 0 and f(D=32769, dt=1) == -2
    size = ctypes.c_size_t(0)
    assert L.bkmoo_residual_norm_workspace_size(100, 64, 2, ctypes.byref(size)) == 0
    need = size.value
    assert need >= (100 + 2) * 2 * 64 * 4
    assert L.bkmoo_residual_norm_workspace_size(100, 64, 17, ctypes.byref(size)) == -2
    assert L.bkmoo_residual_norm_workspace_size(100, 64, 3, None) == -1
    assert L.bkmoo_residual_norm_workspace_size(1 << 24, 64, 3, ctypes.byref(size)) == 0
    assert size.value <= (512 + 3 + 1) * 2 * 64 * 4 + 256  # bounded: chunks, not rows
    g = lambda K=2, tr=rows(0, 40, 100), up=at(0), dn=at(1), r=at(2), y=at(3), w=at(4), p=None, ga=None, dr=at(5), \
        dy=at(6), dw=at(7), dp=None, dg=None, st=1000, ws=at(8), n=need: \
        L.bkmoo_residual_norm_backward(100, 64, 0, K, tr, up, dn, r, y, w, p, ga, 1.0, 1e-6, dr, dy, dw, dp, dg, st, ws,
                                       n, None)  # noqa: E731
    for bad in (dict(K=0), dict(tr=None), dict(tr=rows(0, 40, 99)), dict(tr=rows(1, 40, 100)), dict(tr=rows(0, 101, 100)),
                dict(dn=None), dict(r=None), dict(dw=None), dict(p=at(9)), dict(dp=at(9)), dict(ga=at(9)), dict(st=63),
                dict(ws=None), dict(ws=at(8) + 4), dict(dy=at(2)), dict(dr=at(0) + 64), dict(dr=at(3)), dict(dy=at(8))):
        assert g(**bad) == -1, bad
    assert g(K=17, tr=rows(*([0] * 17), 100)) == -2
    assert g(n=need - 1) == -3


def test_ffn_arguments(b):
    L = b._lib
    size = ctypes.c_size_t(0)
    ws = lambda back, M=70, D=64, F=96, dt=0: (L.bkmoo_ffn_workspace_size(M, D, F, dt, back, ctypes.byref(size)), size.value)  # noqa: E731
    ok, nf = ws(0)
    assert ok == 0 and nf >= 70 * 96 * 4
    ok, nb = ws(1)
    assert ok == 0 and nb >= 3 * 70 * 96 * 4
    assert ws(0, M=0)[0] == 0 and ws(0, M=-1)[0] == -1 and ws(0, D=0)[0] == -1 and ws(0, F=0)[0] == -1
    assert ws(0, dt=3)[0] == -1 and ws(2)[0] == -1 and ws(0, D=(1 << 20) + 1)[0] == -2
    f = lambda M=70, act=0, x=at(0), g=at(1), u=at(2), d=at(3), y=at(4), go=None, uo=None, w=at(5), n=nf: \
        L.bkmoo_ffn_forward(M, 64, 96, 0, act, x, g, u, d, y, go, uo, w, n, None)  # noqa: E731
    assert f(M=0) == 0
    for bad in (dict(M=-1), dict(act=2), dict(x=None), dict(g=None), dict(u=None), dict(d=None), dict(y=None),
                dict(go=at(6)), dict(uo=at(6)), dict(w=None), dict(w=at(5) + 8), dict(x=at(0) + 1), dict(y=at(0) + 16),
                dict(y=at(5)), dict(go=at(6), uo=at(6) + 64), dict(go=at(3), uo=at(6))):
        assert f(**bad) == -1, bad
    assert f(n=nf - 1) == -3
    g = lambda K=2, tr=rows(0, 40, 70), dy=at(0), x=at(1), u=at(2), v=at(3), wg=at(4), wu=at(5), wd=at(6), dx=at(7), \
        a=at(8), bb=at(9), c=at(10), st=20000, w=at(11), n=nb: \
        L.bkmoo_ffn_backward(70, 64, 96, 0, 0, K, tr, dy, x, u, v, wg, wu, wd, dx, a, bb, c, st, w, n, None)  # noqa: E731
    for bad in (dict(K=0), dict(tr=None), dict(tr=rows(0, 71, 70)), dict(tr=rows(0, 1, 2)), dict(dy=None), dict(x=None),
                dict(u=None), dict(v=None), dict(wg=None), dict(wd=None), dict(dx=None), dict(a=None), dict(bb=None),
                dict(c=None), dict(st=64 * 96 - 1), dict(w=None), dict(dx=at(0)), dict(dx=at(11) + 64), dict(c=at(10) + 2)):
        assert g(**bad) == -1, bad
    assert g(K=17, tr=rows(*([0] * 17), 70)) == -2
    assert g(n=nb - 1) == -3


def test_adamw_arguments(b):
    L = b._lib
    hp = lambda lr=0.1, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, t=1: ctypes.byref(b._AdamwHparams(lr, b1, b2, eps, wd, t, 0))  # noqa: E731

    def tensors(*n, base=at(0)):
        return (b._Tensor * len(n))(*[(base + (i << 24), k, 1) for i, k in enumerate(n)])
    blocks = ctypes.c_int64(0)
    assert L.bkmoo_adamw_blocks(3, tensors(1, 256, 257), ctypes.byref(blocks)) == 0 and blocks.value == 4
    assert L.bkmoo_adamw_blocks(0, tensors(1), ctypes.byref(blocks)) == -1
    assert L.bkmoo_adamw_blocks(1, tensors(-1), ctypes.byref(blocks)) == -1
    assert L.bkmoo_adamw_blocks(1, tensors(1), None) == -1
    f = lambda T=2, t=tensors(100, 300), dt=0, N=400, g=at(1), gd=0, s=0, m=at(2), v=at(3), sc=None, bl=0, ma=None, h=hp(), \
        gs=None: L.bkmoo_adamw(T, t, dt, N, g, gd, s, m, v, sc, bl, ma, h, gs, None)  # noqa: E731
    assert f(t=tensors(0, 0), N=0) == 0
    for bad in (dict(T=0), dict(t=None), dict(dt=2), dict(gd=-1), dict(s=2), dict(N=399), dict(N=401), dict(g=None),
                dict(m=None), dict(v=None), dict(sc=at(4), bl=3), dict(ma=at(5)), dict(h=None), dict(h=hp(lr=-1)),
                dict(h=hp(b1=1.0)), dict(h=hp(b2=float("nan"))), dict(h=hp(eps=0)), dict(h=hp(wd=-1)), dict(h=hp(t=0)),
                dict(g=at(1) + 2), dict(m=at(2) + 1), dict(gs=at(6) + 2), dict(v=at(2) + 64), dict(m=at(1)), dict(g=at(0)),
                dict(t=tensors(100, 300, base=0)), dict(t=tensors(100, 300, base=at(0) + 1)), dict(s=1, sc=at(4), bl=2),
                dict(s=1, bl=3), dict(v=at(0) + (1 << 24))):
        assert f(**bad) == -1, bad
