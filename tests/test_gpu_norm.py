"""The residual norms against their definition in 64 bits.

Tolerances (2-norm of the difference over that of the result).  fp32: a result is
made by a few roundings of 2^-24 and a sum over a row, of which a thread adds at most 32
terms before a tree of 10 levels: 50 x 2^-24 = 3e-6.  A column sum adds at most M terms one
after another, errors of random sign: (4 + sqrt(M)) 2^-24 of the summands' norm; the sums
here do not cancel below a tenth of it.  bf16 adds one rounding of the result, 2^-8 at
most."""

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
EPS = 1e-6


def tol(dtype, M=0):
    f32 = 50 * 2.0 ** -24 + (10 * (4 + M ** 0.5) * 2.0 ** -24 if M else 0.0)
    return f32 if dtype == torch.float32 else f32 + 2.0 ** -8


def inputs(M, D, dtype, post, gate, seed=0):
    g = torch.Generator().manual_seed(1000 + seed)
    t = {"r": ref.rand(g, M, D, dtype=dtype, scale=2.0), "y": ref.rand(g, M, D, dtype=dtype, scale=0.7),
         "w": ref.rand(g, D, dtype=dtype, scale=0.1, mean=1.0),
         "p": ref.rand(g, D, dtype=dtype, scale=0.1, mean=1.0) if post else None,
         "g": ref.rand(g, D, dtype=dtype, scale=0.3, mean=0.5) if gate else None,
         "dn": ref.rand(g, M, D, dtype=dtype, mean=0.3), "up": ref.rand(g, M, D, dtype=dtype, mean=-0.2)}
    return t


def gpu(t):
    return {k: (v.cuda() if isinstance(v, torch.Tensor) else v) for k, v in t.items()}


def wide(t):
    return {k: (v.double() if isinstance(v, torch.Tensor) else v) for k, v in t.items()}


SHAPES = [(1, 4096), (1, 1), (3, 2), (5, 7), (64, 64), (33, 511), (17, 512), (9, 1024), (4, 1111), (7, 2056), (3, 4097),
          (2, 8192), (3, 16384), (260, 129)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,D", SHAPES + [(2, 32768)])
@pytest.mark.parametrize("post,gate", [(True, True), (False, False), (True, False), (False, True)])
def test_forward(gpu_lib, M, D, dtype, post, gate):
    if D * dtype.itemsize > 65536:
        pytest.skip("more than a row holds")
    print(f"case norm forward M={M} D={D} {dtype} post={post} gate={gate}", flush=True)
    t = inputs(M, D, dtype, post, gate)
    d, w = gpu(t), wide(t)
    r, n = gpu_lib.residual_norm_forward(d["r"], d["y"], d["w"], d["p"], d["g"], scale=0.7, eps=EPS)
    wr, wn = ref.norm_forward(w["r"], w["y"], w["w"], w["p"], w["g"], 0.7, EPS)
    assert ref.off(r, wr) <= tol(dtype) and ref.off(n, wn) <= tol(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,D", SHAPES + [(2, 32768)])
@pytest.mark.parametrize("post,gate,up", [(True, True, True), (False, False, True), (True, False, False),
                                          (False, True, False)])
def test_backward(gpu_lib, M, D, dtype, post, gate, up):
    if D * dtype.itemsize > 65536:
        pytest.skip("more than a row holds")
    print(f"case norm backward M={M} D={D} {dtype} post={post} gate={gate} up={up}", flush=True)
    t = inputs(M, D, dtype, post, gate, seed=1)
    if not up:
        t["up"] = None
    rows = [0, M // 3, M // 3, M]  # the second task has no row
    d, w = gpu(t), wide(t)
    lead, N = 3, 3 + 3 * D + 5
    grads = torch.full((3, N), 77.0, dtype=dtype, device="cuda")
    cut = [grads[:, lead + i * D:lead + (i + 1) * D] for i in range(3)]
    dr, dy = gpu_lib.residual_norm_backward(d["up"], d["dn"], d["r"], d["y"], d["w"], d["p"], d["g"], 0.7, EPS, rows,
                                            cut[0], cut[1] if post else None, cut[2] if gate else None)
    want = ref.norm_backward(w["up"], w["dn"], w["r"], w["y"], w["w"], w["p"], w["g"], 0.7, EPS, rows)
    # A gradient through a norm is what is left of d / rms when its part along the row is taken
    # out (nothing at D = 1): its error is measured against what there was, and what dr is off by
    # passes on to the others.
    had = (w["dn"] * w["w"] / ref.rms(w["r"], EPS)).norm().item() + (w["up"].norm().item() if up else 0.0)
    assert (dr.double().cpu() - want[0]).norm().item() <= tol(dtype) * had
    rest = 0.7 * tol(torch.float32) * had
    gg, pp = w["g"] if gate else torch.ones(1), w["p"] if post else torch.ones(1)
    size = ref.rms(w["y"], EPS) if post else torch.ones(1)
    z, e = (w["y"] / size).abs().max().item(), 0.7 * want[0] * gg * pp / size
    assert (dy.double().cpu() - want[1]).norm().item() <= tol(dtype) * e.norm().item() + \
        rest * ((gg * pp).abs().max() / size.min()).item()
    rest *= z * max(gg.abs().max().item(), pp.abs().max().item())
    for i, on in enumerate((True, post, gate)):
        if on:
            assert torch.equal(cut[i][1].float(), torch.zeros(D, device="cuda"))
            assert (cut[i].double().cpu() - want[2 + i]).norm().item() <= tol(dtype, M) * want[2 + i].norm().item() + \
                rest * M ** 0.5
        else:
            assert bool((cut[i] == 77.0).all())
    assert bool((grads[:, :lead] == 77.0).all()) and bool((grads[:, lead + 3 * D:] == 77.0).all())


def test_backward_against_differences(gpu_lib):
    """The gradients are those of the forward definition: central differences of
    L = <resid_out, A> + <normed, B> in 64 bits along random directions.  Their own error is
    h^2 times a third derivative (h = 1e-4, of order 1) and 1e-16 / h: far below the
    kernel's, a sum over all elements with relative error 3e-6 of the terms' norm."""
    M, D, rows = 13, 96, [0, 5, 13]
    t = inputs(M, D, torch.float32, True, True, seed=2)
    d, w = gpu(t), wide(t)
    out, _ = ref.norm_forward(w["r"], w["y"], w["w"], w["p"], w["g"], 0.7, EPS)
    # the kernel takes the rounded resid_out: 2^-24 of its input, as much of its results
    grads = torch.zeros((2, 3 * D), device="cuda")
    cut = [grads[:, i * D:(i + 1) * D] for i in range(3)]
    dr, dy = gpu_lib.residual_norm_backward(d["up"], d["dn"], out.float().cuda(), d["y"], d["w"], d["p"], d["g"], 0.7,
                                            EPS, rows, *cut)

    def loss(s):
        r, n = ref.norm_forward(s["r"], s["y"], s["w"], s["p"], s["g"], 0.7, EPS)
        return (r * w["up"]).sum() + (n * w["dn"]).sum()

    gen = torch.Generator().manual_seed(5)
    for name, grad in (("r", dr), ("y", dy), ("w", cut[0].sum(0)), ("p", cut[1].sum(0)), ("g", cut[2].sum(0))):
        for _ in range(4):
            v = torch.randn(w[name].shape, generator=gen, dtype=torch.float64)
            h = 1e-4
            diff = (loss({**w, name: w[name] + h * v}) - loss({**w, name: w[name] - h * v})).item() / (2 * h)
            got = (grad.double().cpu() * v).sum().item()
            assert abs(got - diff) <= 1e-5 * (grad.double().cpu().norm() * v.norm()).item() + 1e-6, name


def test_in_place_other_stream_and_repeatable(gpu_lib):
    t = gpu(inputs(130, 1000, torch.bfloat16, True, True, seed=3))
    args = (t["y"], t["w"], t["p"], t["g"])
    r1, n1 = gpu_lib.residual_norm_forward(t["r"], *args, scale=0.5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        r = t["r"].clone()
        r2, n2 = gpu_lib.residual_norm_forward(r, *args, scale=0.5, resid_out=r)
    torch.cuda.current_stream().wait_stream(s)
    assert r2.data_ptr() == r.data_ptr()
    assert torch.equal(r1, r2) and torch.equal(n1, n2)
    outs = []
    for _ in range(2):
        up = t["up"].clone()
        g = torch.empty((2, 3000), dtype=torch.bfloat16, device="cuda")
        dr, dy = gpu_lib.residual_norm_backward(up, t["dn"], r1, *args, scale=0.5, task_rows=[0, 50, 130],
                                                dweight=g[:, :1000], dpost_weight=g[:, 1000:2000], dgate=g[:, 2000:],
                                                dresid=up)
        assert dr.data_ptr() == up.data_ptr()
        outs.append((dr.clone(), dy, g))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_non_finite_rows_stay_alone(gpu_lib):
    """A row with a NaN or an infinity spoils itself and its own task's sums, nothing else."""
    t = inputs(8, 256, torch.float32, True, True, seed=4)
    t["y"][2, 5] = float("nan")
    t["r"][6, 9] = float("inf")
    d = gpu(t)
    r, n = gpu_lib.residual_norm_forward(d["r"], d["y"], d["w"], d["p"], d["g"])
    ok = torch.isfinite(n).all(1).cpu()
    assert ok.tolist() == [True, True, False, True, True, True, False, True]
    g = torch.empty((3, 768), device="cuda")
    dr, dy = gpu_lib.residual_norm_backward(d["up"], d["dn"], d["r"], d["y"], d["w"], d["p"], d["g"], task_rows=[0, 2, 5, 8],
                                            dweight=g[:, :256], dpost_weight=g[:, 256:512], dgate=g[:, 512:])
    assert torch.isfinite(dy).all(1).cpu().tolist() == ok.tolist()
    assert bool(torch.isfinite(g[0]).all()) and not bool(torch.isfinite(g[1]).all())


def test_no_rows(gpu_lib):
    D = 40
    z = torch.empty((0, D), device="cuda")
    w = torch.ones(D, device="cuda")
    r, n = gpu_lib.residual_norm_forward(z, z, w)
    assert r.shape == (0, D) and n.shape == (0, D)
    g = torch.full((2, D), 5.0, device="cuda")
    gpu_lib.residual_norm_backward(None, z, z, z, w, task_rows=[0, 0, 0], dweight=g)
    assert bool((g == 0).all())


def test_refusals(gpu_lib):
    r = torch.zeros((4, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    f = gpu_lib.residual_norm_forward
    for bad in (dict(y=r[:2]), dict(y=r.bfloat16()), dict(y=r.cpu()), dict(weight=w[:32]), dict(gate=w.bfloat16()),
                dict(post_weight=torch.ones((64, 1), device="cuda")), dict(y=torch.zeros((64, 4), device="cuda").t())):
        with pytest.raises(ValueError):
            f(**{**dict(resid=r, y=r.clone(), weight=w), **bad})
    with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
        f(r, r.clone(), w, eps=-1.0)
    with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
        f(r, r, w, normed=r)  # overlaps an input
    big = torch.zeros((1, 20000), device="cuda")
    with pytest.raises(gpu_lib.BkmooError, match="EUNSUPPORTED"):
        f(big, big.clone(), torch.ones(20000, device="cuda"))
    g = torch.zeros((2, 64), device="cuda")
    bwd = lambda **k: gpu_lib.residual_norm_backward(**{**dict(  # noqa: E731
        dresid_out=None, dnormed=r, resid_out=r.clone(), y=r.clone(), weight=w, task_rows=[0, 1, 4], dweight=g), **k})
    for rows in ([0, 3, 2], [0, 1, 5], [1, 2, 4]):
        with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
            bwd(task_rows=rows)
    with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
        bwd(dgate=g)  # no gate
    for bad in (dict(dweight=None), dict(dweight=g[:1]), dict(task_rows=[0]), dict(dweight=g.t().contiguous().t())):
        with pytest.raises(ValueError):
            bwd(**bad)
    with pytest.raises(gpu_lib.BkmooError, match="EWORKSPACE"):
        bwd(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
