"""Every cut of the feed-forward block's products: tiles of 64, 128 and 256, whole and split sums (parts without a
step among them), workgroups that go through several tiles, sizes that end inside a tile and inside a step.

Tolerances against the 64-bit definition as in the block's other tests: fp32 sums of n products in any order of parts
4 sqrt(n) 2^-24 and 50 x 2^-24 for the activation; bf16 2^-8 x 1.5 more for the rounding between the products and of the
result.  Cuts with equal parts add in the same order: equal bits."""

import functools

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu

# rows at multiples of 16 bytes; of four bytes (bf16 of 130: 260); of two
SHAPES = {"even": (600, 520, 776, (0, 150, 150, 599, 600)), "four": (331, 130, 518, (0, 64, 331)),
          "odd": (300, 131, 265, (0, 299, 300))}


def tol(dtype, n):
    f32 = (4 * n ** 0.5 + 50) * 2.0 ** -24
    return f32 if dtype == torch.float32 else f32 + 1.5 * 2.0 ** -8


@functools.lru_cache(maxsize=None)
def case(M, D, F, rows, dtype):
    """Inputs, and what the definition gives."""
    g = torch.Generator().manual_seed(900 + M)
    t = {"x": ref.rand(g, M, D, dtype=dtype), "wg": ref.rand(g, F, D, dtype=dtype, scale=D ** -0.5),
         "wu": ref.rand(g, F, D, dtype=dtype, scale=D ** -0.5), "wd": ref.rand(g, D, F, dtype=dtype, scale=F ** -0.5),
         "dy": ref.rand(g, M, D, dtype=dtype), "u": ref.rand(g, M, F, dtype=dtype), "v": ref.rand(g, M, F, dtype=dtype)}
    w = {k: v.double() for k, v in t.items()}
    return t, ref.ffn_forward(w["x"], w["wg"], w["wu"], w["wd"], "gelu"), \
        ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], "gelu", list(rows))


def passes(lib, t, rows, cut):
    """y, u, v, dx and the gradient buffer of both passes, with the products cut so."""
    d = {k: v.cuda() for k, v in t.items()}
    (M, D), F, K = d["x"].shape, d["wg"].shape[0], len(rows) - 1
    n, lead = D * F, 3
    grads = torch.full((K, lead + 3 * n + 5), 77.0, dtype=d["x"].dtype, device="cuda")
    dw = [grads[:, lead + i * n:lead + (i + 1) * n] for i in range(3)]
    lib.set_ffn_tiles(*cut)
    try:
        out = lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], act="gelu", save=True)
        dx = lib.ffn_backward(d["dy"], d["x"], d["u"], d["v"], d["wg"], d["wu"], d["wd"], act="gelu", task_rows=rows,
                              dw_gate=dw[0], dw_up=dw[1], dw_down=dw[2])
        torch.cuda.synchronize()
    finally:
        lib.set_ffn_tiles()
    return *out, dx, grads


def check(dtype, got, want, M, D, F):
    y, u, v, dx, grads = got
    (wy, wu, wv), (wdx, *wdw) = want
    n, lead = D * F, 3
    assert ref.off(y, wy) <= tol(dtype, max(D, F))
    assert ref.off(u, wu) <= tol(dtype, D) and ref.off(v, wv) <= tol(dtype, D)
    assert ref.off(dx, wdx) <= tol(dtype, 2 * max(D, F))
    for i, w in enumerate(wdw):
        assert ref.off(grads[:, lead + i * n:lead + (i + 1) * n].reshape(w.shape), w) <= tol(dtype, max(M, D))
    assert bool((grads[:, :lead] == 77.0).all()) and bool((grads[:, lead + 3 * n:] == 77.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("splits", [1, 2, 7])
def test_every_tile(gpu_lib, dtype, shape, splits):
    M, D, F, rows = SHAPES[shape]
    t, *want = case(M, D, F, rows, dtype)
    first = None
    for side in (64, 128, 256):
        for workgroups in (0, 3, 17):
            print(f"case ffn tiles {shape} {dtype} side={side} splits={splits} workgroups={workgroups}", flush=True)
            got = passes(gpu_lib, t, rows, (side, splits, workgroups))
            if first is None:
                first = got
                check(dtype, got, want, M, D, F)
            assert all(torch.equal(a, b) for a, b in zip(first, got)), (side, workgroups)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("side", [64, 128, 256])
def test_more_parts_than_steps(gpu_lib, dtype, side):
    """Sums of one to three steps in 16 parts, and a task without rows."""
    M, D, F, rows = 70, 8, 72, (0, 70, 70)
    t, *want = case(M, D, F, rows, dtype)
    for workgroups in (0, 2):
        print(f"case ffn tiles parts {dtype} side={side} workgroups={workgroups}", flush=True)
        check(dtype, passes(gpu_lib, t, rows, (side, 16, workgroups)), want, M, D, F)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("side", [128, 256])
def test_non_finite_values_stay_in_their_rows(gpu_lib, dtype, side):
    """A step that a row ends in brings the next row's values: NaN there stays out, in tiles of every size."""
    M, D, F, rows = SHAPES["four"]
    t, (wy, _, _), (wdx, *_) = case(M, D, F, rows, dtype)
    t = {k: v.clone() for k, v in t.items()}
    for k in ("x", "dy", "u", "v"):
        t[k][260] = float("nan")
    y, _, _, dx, _ = passes(gpu_lib, t, rows, (side, 1, 2))
    others = [m for m in range(M) if m != 260]
    assert bool(torch.isnan(y[260]).all()) and bool(torch.isnan(dx[260]).all())
    assert ref.off(y[others], wy[others]) <= tol(dtype, F) and ref.off(dx[others], wdx[others]) <= tol(dtype, 2 * F)


def test_graph_replays_of_large_tiles(gpu_lib):
    """A captured pass over several tiles a workgroup gives the eager bits on every replay."""
    M, D, F, rows = SHAPES["even"]
    t, *_ = case(M, D, F, rows, torch.bfloat16)
    d = {k: v.cuda() for k, v in t.items()}
    step = lambda: gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], act="gelu")[0]  # noqa: E731
    gpu_lib.set_ffn_tiles(256, 2, 3)
    try:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = step()
        for i in range(3):
            d["x"].mul_(0.5)
            graph.replay()
            torch.cuda.synchronize()
            got, want = y.clone(), step()
            torch.cuda.synchronize()
            assert torch.equal(got, want), i
    finally:
        gpu_lib.set_ffn_tiles()


def test_refusals(gpu_lib):
    for bad in ((32,), (-64,), (512,), (0, -1), (0, 17), (0, 0, -1)):
        with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
            gpu_lib.set_ffn_tiles(*bad)
    d = {k: v.cuda() for k, v in case(*SHAPES["even"], torch.bfloat16)[0].items()}
    ws = torch.empty(gpu_lib.ffn_workspace_size(600, 520, 776, torch.bfloat16), dtype=torch.uint8, device="cuda")
    gpu_lib.set_ffn_tiles(0, 16)
    try:
        with pytest.raises(gpu_lib.BkmooError, match="EWORKSPACE"):
            gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], workspace=ws)
    finally:
        gpu_lib.set_ffn_tiles()
