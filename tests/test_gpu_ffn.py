"""The gated feed-forward block against its definition in 64 bits.

Tolerances (2-norm of the difference over that of the result).  fp32: a sum of n products in
fp32, errors of random sign, is off by about sqrt(n) 2^-24 of the products' norm, and
the sums here do not cancel on the whole; two or three such sums follow one another: 4 sqrt(n) 2^-24
with n the longest, and 50 x 2^-24 for the activation.  bf16: the same, and each of the two
roundings (of what lies between the products, and of the result) is 2^-8 at most and
2^-9 on average of its value: 2^-8 x 1.5 for both."""

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


def tol(dtype, n):
    f32 = (4 * n ** 0.5 + 50) * 2.0 ** -24
    return f32 if dtype == torch.float32 else f32 + 1.5 * 2.0 ** -8


def inputs(M, D, F, dtype, seed=0):
    g = torch.Generator().manual_seed(77 + seed)
    return {"x": ref.rand(g, M, D, dtype=dtype), "wg": ref.rand(g, F, D, dtype=dtype, scale=D ** -0.5),
            "wu": ref.rand(g, F, D, dtype=dtype, scale=D ** -0.5), "wd": ref.rand(g, D, F, dtype=dtype, scale=F ** -0.5),
            "dy": ref.rand(g, M, D, dtype=dtype), "u": ref.rand(g, M, F, dtype=dtype), "v": ref.rand(g, M, F, dtype=dtype)}


def gpu(t):
    return {k: v.cuda() for k, v in t.items()}


def wide(t):
    return {k: v.double() for k, v in t.items()}


SHAPES = [(1, 1, 1), (1, 64, 200), (1, 2048, 512), (2, 72, 136), (3, 7, 5), (8, 130, 258), (9, 130, 258), (16, 256, 384), (17, 256, 384), (24, 520, 264),
          (33, 128, 320), (64, 512, 96), (65, 512, 96), (130, 65, 131), (100, 1000, 72), (257, 136, 520), (300, 258, 514),
          (513, 768, 640), (1030, 264, 1000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,D,F", SHAPES)
@pytest.mark.parametrize("act,save", [("silu", True), ("gelu", False)])
def test_forward(gpu_lib, M, D, F, dtype, act, save):
    print(f"case ffn forward M={M} D={D} F={F} {dtype} {act} save={save}", flush=True)
    t = inputs(M, D, F, dtype)
    d, w = gpu(t), wide(t)
    y, u, v = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], act=act, save=save)
    wy, wu, wv = ref.ffn_forward(w["x"], w["wg"], w["wu"], w["wd"], act)
    assert ref.off(y, wy) <= tol(dtype, max(D, F))
    if save:
        assert ref.off(u, wu) <= tol(dtype, D) and ref.off(v, wv) <= tol(dtype, D)
    else:
        assert u is None and v is None


def backward(lib, d, dtype, rows, act, lead=3):
    M, D = d["x"].shape
    F, K = d["wg"].shape[0], len(rows) - 1
    n = D * F
    grads = torch.full((K, lead + 3 * n + 5), 77.0, dtype=dtype, device="cuda")
    cut = [grads[:, lead + i * n:lead + (i + 1) * n] for i in range(3)]
    dx = lib.ffn_backward(d["dy"], d["x"], d["u"], d["v"], d["wg"], d["wu"], d["wd"], act=act, task_rows=rows,
                          dw_gate=cut[0], dw_up=cut[1], dw_down=cut[2])
    return dx, grads, cut


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,D,F", SHAPES)
@pytest.mark.parametrize("act,lead", [("silu", 8), ("gelu", 3)])
def test_backward(gpu_lib, M, D, F, dtype, act, lead):
    print(f"case ffn backward M={M} D={D} F={F} {dtype} {act} lead={lead}", flush=True)
    t = inputs(M, D, F, dtype, seed=1)
    rows = [0, M // 3, M // 3, M]  # the second task has no row
    d, w = gpu(t), wide(t)
    dx, grads, cut = backward(gpu_lib, d, dtype, rows, act, lead)
    want = ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], act, rows)
    assert ref.off(dx, want[0]) <= tol(dtype, 2 * max(D, F))
    for k in range(3):
        assert ref.off(cut[k].reshape(want[1 + k].shape), want[1 + k]) <= tol(dtype, max(M, D))
        assert bool((cut[k][1] == 0).all())
    assert bool((grads[:, :lead] == 77.0).all()) and bool((grads[:, lead + 3 * D * F:] == 77.0).all())


def test_backward_against_differences(gpu_lib):
    """dx, dWg, dWu, dWd of the whole block are its central differences in 64 bits (h = 1e-4, second
    order, third derivatives of order 1: 1e-8) along random directions; the kernel's u and v are the
    forward kernel's own, fp32."""
    M, D, F = 21, 40, 56
    t = inputs(M, D, F, torch.float32, seed=2)
    d, w = gpu(t), wide(t)
    for act in ("silu", "gelu"):
        _, d["u"], d["v"] = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], act=act, save=True)
        dx, _, cut = backward(gpu_lib, d, torch.float32, [0, 9, M], act)
        loss = lambda s: (ref.ffn_forward(s["x"], s["wg"], s["wu"], s["wd"], act)[0] * w["dy"]).sum()  # noqa: E731
        gen = torch.Generator().manual_seed(6)
        for name, grad in (("x", dx), ("wg", cut[0].sum(0)), ("wu", cut[1].sum(0)), ("wd", cut[2].sum(0))):
            grad = grad.double().cpu().view(w[name].shape)
            for _ in range(4):
                v = torch.randn(w[name].shape, generator=gen, dtype=torch.float64)
                h = 1e-4
                diff = (loss({**w, name: w[name] + h * v}) - loss({**w, name: w[name] - h * v})).item() / (2 * h)
                assert abs((grad * v).sum().item() - diff) <= 1e-5 * (grad.norm() * v.norm()).item(), (act, name)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tasks_of_every_length(gpu_lib, dtype):
    """Sixteen tasks: empty, single rows, lengths around the kernels' steps of 32 and 64 rows."""
    lens = [0, 1, 2, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 5, 0, 200]
    rows = [0]
    for n in lens:
        rows.append(rows[-1] + n)
    t = inputs(rows[-1], 136, 200, dtype, seed=3)
    d, w = gpu(t), wide(t)
    dx, _, cut = backward(gpu_lib, d, dtype, rows, "silu")
    want = ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], "silu", rows)
    assert ref.off(dx, want[0]) <= tol(dtype, 400)
    for k in range(3):
        for task in range(16):
            assert ref.off(cut[k][task].reshape(want[1 + k][task].shape), want[1 + k][task]) <= tol(dtype, 200)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,D,F", [(1, 2048, 65), (37, 2048, 193), (66, 1025, 97)])
def test_backward_with_split_sums(gpu_lib, M, D, F, dtype):
    """Few rows of a wide model: the sums over D of the hidden gradient are split and joined (sizes that end inside
    the joining kernel's eight elements, rows off four bytes)."""
    print(f"case ffn backward split M={M} D={D} F={F} {dtype}", flush=True)
    t = inputs(M, D, F, dtype, seed=8)
    rows = [0, M // 2, M]
    d, w = gpu(t), wide(t)
    for act in ("silu", "gelu"):
        dx, _, cut = backward(gpu_lib, d, dtype, rows, act)
        want = ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], act, rows)
        assert ref.off(dx, want[0]) <= tol(dtype, 2 * max(D, F))
        for k in range(3):
            assert ref.off(cut[k].reshape(want[1 + k].shape), want[1 + k]) <= tol(dtype, max(M, D))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_unaligned_operands(gpu_lib, dtype, shift):
    """Contiguous operands that start off 16 bytes take the other loads: same results to rounding."""
    M, D, F = 70, 136, 264
    t = inputs(M, D, F, dtype, seed=4)
    w = wide(t)
    d = {}
    for k, v in t.items():
        buf = torch.empty(v.numel() + 8, dtype=dtype, device="cuda")
        d[k] = buf[shift:shift + v.numel()].view(v.shape)
        d[k].copy_(v)
    y, _, _ = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"])
    assert ref.off(y, ref.ffn_forward(w["x"], w["wg"], w["wu"], w["wd"], "silu")[0]) <= tol(dtype, F)
    dx, _, cut = backward(gpu_lib, d, dtype, [0, 30, M], "silu")
    want = ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], "silu", [0, 30, M])
    assert ref.off(dx, want[0]) <= tol(dtype, 2 * F)
    for k in range(3):
        assert ref.off(cut[k].reshape(want[1 + k].shape), want[1 + k]) <= tol(dtype, M)


@pytest.mark.parametrize("M", [3, 40, 600])
def test_extreme_and_non_finite_values(gpu_lib, M):
    """Large gates saturate (SiLU to u or to 0, derivative to 1 or 0) without NaN; a NaN in a row stays in it."""
    D, F = 64, 128
    t = inputs(M, D, F, torch.float32, seed=5)
    t["x"][0] *= 1e4
    t["u"][0, :64], t["u"][0, 64:] = 1e4, -1e4
    if M > 2:
        t["x"][2, 3] = float("nan")
    d = gpu(t)
    for act in ("silu", "gelu"):
        y, _, _ = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], act=act)
        fine = torch.isfinite(y).all(1).cpu()
        assert fine.tolist() == [i != 2 for i in range(M)]
        t2 = gpu(inputs(M, D, F, torch.float32, seed=5))
        t2["u"] = d["u"]
        dx, _, _ = backward(gpu_lib, t2, torch.float32, [0, M], act)
        w = {k: v.double().cpu() for k, v in t2.items()}
        want = ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], act, [0, M])[0]
        assert ref.off(dx, want) <= tol(torch.float32, 2 * F)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [5, 100, 300])
def test_rows_that_end_inside_a_step_keep_to_themselves(gpu_lib, M, dtype):
    """Rows whose last step of the sum runs into the next row: what is there (NaN) stays out."""
    D, F = 70, 90
    t = inputs(M, D, F, dtype, seed=9)
    w = wide(t)
    for k in ("x", "dy", "u", "v"):
        t[k][2] = float("nan")
    d = gpu(t)
    others = [m for m in range(M) if m != 2]
    y = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"])[0]
    dx, _, _ = backward(gpu_lib, d, dtype, [0, 2, M], "silu")
    want = ref.ffn_forward(w["x"], w["wg"], w["wu"], w["wd"], "silu")[0]
    grad = ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], "silu", [0, 2, M])[0]
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(dx[2]).all())
    assert ref.off(y[others], want[others]) <= tol(dtype, F)
    assert ref.off(dx[others], grad[others]) <= tol(dtype, 2 * F)


@pytest.mark.parametrize("M", [1, 20, 300])
def test_other_stream_workspace_and_repeatable(gpu_lib, M):
    """The same bits from a caller's own (dirty) workspace on another stream; outputs may be given."""
    D, F = 136, 520
    d = gpu(inputs(M, D, F, torch.bfloat16, seed=6))
    y1, u1, v1 = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], save=True)
    dx1, g1, _ = backward(gpu_lib, d, torch.bfloat16, [0, M // 2, M], "silu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ws = torch.full((gpu_lib.ffn_workspace_size(M, D, F, torch.bfloat16),), 0xff, dtype=torch.uint8, device="cuda")
        y2, u2, v2 = torch.empty_like(y1), torch.empty_like(u1), torch.empty_like(v1)
        gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], out=y2, gate_out=u2, up_out=v2, workspace=ws)
        dx2, g2, _ = backward(gpu_lib, d, torch.bfloat16, [0, M // 2, M], "silu")
    torch.cuda.current_stream().wait_stream(s)
    for a, b in ((y1, y2), (u1, u2), (v1, v2), (dx1, dx2), (g1, g2)):
        assert torch.equal(a, b)


def test_graph_replays(gpu_lib):
    """A captured forward and backward pass gives the eager bits on every replay."""
    M, D, F = 40, 136, 264
    d = gpu(inputs(M, D, F, torch.bfloat16, seed=7))
    grads = torch.zeros((2, 3 * D * F), dtype=torch.bfloat16, device="cuda")
    cut = [grads[:, i * D * F:(i + 1) * D * F] for i in range(3)]
    step = lambda: (gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"])[0],  # noqa: E731
                    gpu_lib.ffn_backward(d["dy"], d["x"], d["u"], d["v"], d["wg"], d["wu"], d["wd"],
                                         task_rows=[0, 11, M], dw_gate=cut[0], dw_up=cut[1], dw_down=cut[2]))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = step()
    for i in range(4):
        d["x"].mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = (y.clone(), dx.clone(), grads.clone())
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], grads), i


def test_no_rows(gpu_lib):
    D, F = 24, 40
    d = gpu(inputs(0, D, F, torch.float32))
    y, u, v = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], save=True)
    assert y.shape == (0, D) and u.shape == (0, F)
    _, grads, cut = backward(gpu_lib, d, torch.float32, [0, 0, 0], "silu")
    assert all(bool((c == 0).all()) for c in cut)


@pytest.mark.slow
def test_offsets_past_32_bits(gpu_lib):
    """Activations of more than 4 GiB: rows at the end equal those of a small call."""
    M, D, F = 160_003, 64, 14336
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("not enough memory")
    t = gpu(inputs(64, D, F, torch.bfloat16, seed=8))
    d = dict(t)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for k, n in (("x", D), ("dy", D), ("u", F), ("v", F)):
        d[k] = torch.randn((M, n), generator=gen, dtype=torch.bfloat16, device="cuda")
    y, u, v = gpu_lib.ffn_forward(d["x"], d["wg"], d["wu"], d["wd"], save=True)
    small = gpu_lib.ffn_forward(d["x"][-500:].contiguous(), d["wg"], d["wu"], d["wd"], save=True)
    w = {k: (x[-500:] if k in ("x", "dy", "u", "v") else x).double().cpu() for k, x in d.items()}
    wy, wu, wv = ref.ffn_forward(w["x"], w["wg"], w["wu"], w["wd"], "silu")
    for got, few, want in ((y, small[0], wy), (u, small[1], wu), (v, small[2], wv)):
        assert ref.off(got[-500:], want) <= tol(torch.bfloat16, F)
        assert ref.off(few, want) <= tol(torch.bfloat16, F)
    dx, _, cut = backward(gpu_lib, d, torch.bfloat16, [0, M - 500, M], "silu")
    want = ref.ffn_backward(w["dy"], w["x"], w["u"], w["v"], w["wg"], w["wu"], w["wd"], "silu", [0, 500])
    assert ref.off(dx[-500:], want[0]) <= tol(torch.bfloat16, 2 * F)
    for k in range(3):
        assert ref.off(cut[k][1].reshape(want[1 + k][0].shape), want[1 + k][0]) <= tol(torch.bfloat16, 500)


def test_refusals(gpu_lib):
    t = gpu(inputs(8, 32, 48, torch.float32))
    fwd = lambda **k: gpu_lib.ffn_forward(**{**dict(x=t["x"], w_gate=t["wg"], w_up=t["wu"], w_down=t["wd"]), **k})  # noqa: E731
    for bad in (dict(w_up=t["wu"][:40]), dict(w_down=t["wg"]), dict(x=t["x"].cpu()), dict(w_gate=t["wg"].bfloat16()),
                dict(x=t["x"][0]), dict(w_down=t["wd"].t().contiguous().t()), dict(out=t["x"][:4]),
                dict(workspace=torch.empty(4096, device="cuda")), dict(gate_out=t["u"][:4], up_out=t["v"])):
        with pytest.raises(ValueError):
            fwd(**bad)
    with pytest.raises(TypeError):
        fwd(x=t["x"].half())
    with pytest.raises(KeyError):
        fwd(act="relu")
    for bad in (dict(out=t["x"]), dict(gate_out=t["u"])):   # over an input; one product without the other
        with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
            fwd(**bad)
    with pytest.raises(gpu_lib.BkmooError, match="EWORKSPACE"):
        fwd(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    g = torch.zeros((2, 3 * 32 * 48), device="cuda")
    cut = [g[:, i * 1536:(i + 1) * 1536] for i in range(3)]
    bwd = lambda **k: gpu_lib.ffn_backward(**{**dict(  # noqa: E731
        dy=t["dy"], x=t["x"], gate_out=t["u"], up_out=t["v"], w_gate=t["wg"], w_up=t["wu"], w_down=t["wd"],
        task_rows=[0, 3, 8], dw_gate=cut[0], dw_up=cut[1], dw_down=cut[2]), **k})
    for rows in ([0, 9, 8], [0, 3, 9], [1, 3, 8], [0, 3, 7]):
        with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
            bwd(task_rows=rows)
    for bad in (dict(dw_up=None), dict(dw_gate=g[:, :1535]), dict(dw_gate=cut[0].contiguous()), dict(task_rows=[0]),
                dict(task_rows=[0, 8]), dict(dw_down=cut[2].bfloat16())):
        with pytest.raises(ValueError):
            bwd(**bad)
    with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
        bwd(dx=t["dy"])
    big = [torch.zeros((17, 1536), device="cuda") for _ in range(3)]
    with pytest.raises(gpu_lib.BkmooError, match="EUNSUPPORTED"):
        bwd(task_rows=[0] * 17 + [8], dw_gate=big[0], dw_up=big[1], dw_down=big[2])
