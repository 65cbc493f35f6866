"""The AdamW step against its definition in 64 bits.

Tolerances (2-norm of the difference over that of the terms that are added).  32-bit moments are
made by four roundings of 2^-24, the parameter by eight: 8 x 2^-24.  A bf16 parameter adds one
rounding, 2^-8 at most.  The first moment's terms b1 m and (1 - b1) g may cancel: an
error of 8 x 2^-24 of them is what the result, and the step made of it, may be off by.  8-bit moments are compared with the neighbours they may be
rounded to: equal to the definition's choice (same random bits) except where fp32 and 64 bits
fall on different sides of it: within 1e-4 of the distance between e4m3 values, and 8 x 2^-24 of
the first moment's terms, of the border either is right."""

import numpy as np
import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
SETS = [[1], [7, 1, 300], [256, 512], [4096, 4095, 4097, 8], [100_003], [0, 5, 0], [33] * 300]


def reference(p, g, m, v, sizes, decay, step, hp=HP):
    p, m, v = p.clone(), m.clone(), v.clone()
    at = 0
    for n, d in zip(sizes, decay):
        s = slice(at, at + n)
        p[s], m[s], v[s] = ref.adamw(p[s], g[s], m[s], v[s], step, hp["lr"], hp["beta1"], hp["beta2"], hp["eps"],
                                     hp["weight_decay"] if d else 0.0)
        at += n
    return p, m, v


def terms(g, m, hp=HP):
    """Size of what the first moment is added up from."""
    return hp["beta1"] * m.double().abs() + (1 - hp["beta1"]) * g.double().abs()


def step_terms(p, g, m, v, step, hp=HP):
    """The same for the parameter: itself, and the step with the first moment's terms."""
    one = torch.ones((), dtype=torch.float64)
    t, _, _ = ref.adamw(0 * one, g.double().abs(), m.double().abs(), v.double(), step, hp["lr"], hp["beta1"], hp["beta2"],
                        hp["eps"], 0.0)
    return p.double().abs() + t.abs()


def off_terms(got, want, size):
    return (got.double().cpu() - want).norm().item() / max(size.norm().item(), 1e-300)


def make(sizes, dtype, gdtype, seed=0):
    gen = torch.Generator().manual_seed(500 + seed)
    n = sum(sizes)
    return ref.rand(gen, n, dtype=dtype), ref.rand(gen, n, dtype=gdtype, scale=0.1), \
        ref.rand(gen, n, scale=0.03), ref.rand(gen, n, scale=0.1).square()


@pytest.mark.parametrize("sizes", SETS, ids=lambda s: f"{len(s)}t{sum(s)}")
@pytest.mark.parametrize("dtype,gdtype,master", [(torch.float32, torch.float32, False),
                                                 (torch.bfloat16, torch.bfloat16, False),
                                                 (torch.bfloat16, torch.float32, True),
                                                 (torch.float32, torch.bfloat16, False)])
def test_f32_states(gpu_lib, sizes, dtype, gdtype, master):
    print(f"case adamw {len(sizes)} tensors {sum(sizes)} {dtype} {gdtype} master={master}", flush=True)
    p, g, m, v = make(sizes, dtype, gdtype)
    decay = [i % 2 == 0 for i in range(len(sizes))]
    params = [t.clone().cuda() for t in torch.split(p, sizes)]  # each in memory of its own
    mm = (p.float() + 1e-3 * torch.arange(p.numel()) / max(1, p.numel())).cuda() if master else None
    want = reference(mm.cpu().double() if master else p.double(), 0.5 * g.double(), m.double(), v.double(), sizes, decay, 3)
    gm, gv = m.cuda(), v.cuda()
    gpu_lib.adamw(gpu_lib.adamw_table(params, decay), g.cuda(), gm, gv, step=3, master=mm,
                  grad_scale=torch.tensor([0.5], device="cuda"), **HP)
    got = torch.cat([t.reshape(-1) for t in params])
    f32 = 8 * 2.0 ** -24
    size = step_terms(p, 0.5 * g, m, v, 3)
    assert off_terms(gm, want[1], terms(0.5 * g, m)) <= f32 and ref.off(gv, want[2]) <= f32
    if master:
        assert off_terms(mm, want[0], size) <= f32
        assert torch.equal(got, mm.bfloat16())
    assert off_terms(got, want[0], size) <= f32 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)


def expected_f8(x, part_random, positive, size):
    """e4m3 values and the scale of one block (64 bits), by the definition: of the two values around
    it the upper where the part of the way there and a random number in (0, 1) reach one; and where fp32's
    error, of terms of `size`, may decide otherwise."""
    top = np.abs(x).max()
    if top < 2.0 ** -100:
        return np.zeros_like(x), 0.0, np.zeros(x.shape, bool)
    vals = ref.e4m3_values()
    y = np.minimum(np.abs(x) * (448.0 / top), 448.0)
    lo = np.searchsorted(vals, y, side="right") - 1
    hi = np.minimum(lo + 1, len(vals) - 1)
    part = np.where(hi > lo, (y - vals[lo]) / np.where(hi > lo, vals[hi] - vals[lo], 1.0), 0.0)
    up = part + part_random >= 1.0
    apart = np.where(hi > lo, vals[hi] - vals[lo], 1.0)
    near = np.abs(part + part_random - 1.0) < 1e-4 + 8 * 2.0 ** -24 * size * (448.0 / top) / apart
    out = np.where(up, vals[hi], vals[lo])
    if positive:
        out = np.where(x > 0, np.maximum(out, 2.0 ** -9), out)
    return np.where(x < 0, -out, out), top / 448.0, near


@pytest.mark.parametrize("sizes", SETS, ids=lambda s: f"{len(s)}t{sum(s)}")
@pytest.mark.parametrize("dtype,master,beta2", [(torch.float32, False, 0.95), (torch.bfloat16, True, 0.95),
                                                (torch.bfloat16, False, 0.99)])
def test_f8_states(gpu_lib, sizes, dtype, master, beta2):
    print(f"case adamw f8 {len(sizes)} tensors {sum(sizes)} {dtype} master={master} {beta2}", flush=True)
    hp = dict(HP, beta2=beta2)
    p, g, _, _ = make(sizes, dtype, dtype, seed=1)
    n, seed, step = sum(sizes), 1234, 7
    gen = np.random.default_rng(3)
    params = [t.clone().cuda() for t in torch.split(p, sizes)]
    table = gpu_lib.adamw_table(params)
    assert table.blocks == sum(-(-s // 256) for s in sizes)
    m8 = torch.from_numpy(gen.normal(0, 100, n).clip(-448, 448)).float().to(torch.float8_e4m3fn)
    q8 = torch.from_numpy(np.abs(gen.normal(0, 100, n)).clip(2.0 ** -9, 448)).float().to(torch.float8_e4m3fn)
    scales = torch.from_numpy(gen.uniform(1e-4, 3e-4, (2, table.blocks))).float()
    of = np.concatenate([np.full(s, 0) for s in sizes] or [[]]).astype(np.int64)
    at = blk = 0
    for s in sizes:
        of[at:at + s] = blk + np.arange(s) // 256
        at, blk = at + s, blk + -(-s // 256)
    m = m8.double() * scales[0].double()[of]
    q = q8.double() * scales[1].double()[of]
    mm = p.float().cuda() if master else None
    want = reference(p.double(), g.double(), m, q * q, sizes, [True] * len(sizes), step, hp)
    gm, gq, gs = m8.cuda(), q8.cuda(), scales.cuda()
    gpu_lib.adamw(table, g.cuda(), gm, gq, step=step, master=mm, scales=gs, seed=seed, **hp)
    got = torch.cat([t.reshape(-1) for t in params])
    f32 = 12 * 2.0 ** -24
    assert off_terms(mm if master else got, want[0], step_terms(p, g, m, q * q, step, hp)) <= f32 + (2.0 ** -8 if dtype == torch.bfloat16 and not master else 0)
    m1, q1 = want[1].numpy(), want[2].sqrt().numpy()
    size = (terms(g, m).numpy(), q1)
    gm, gq, gs = gm.double().cpu().numpy(), gq.double().cpu().numpy(), gs.double().cpu().numpy()
    at = blk = 0
    for s in sizes:
        for b in range(-(-s // 256)):
            i = np.arange(b * 256, min(s, (b + 1) * 256))
            if beta2 > 0.98:   # sixteen bits a moment
                h = ref.mix(blk * 256 + i % 256, seed)
                random = [((h >> np.uint32(k)) & np.uint32(0xffff)) / 65536 + 2.0 ** -17 for k in (0, 16)]
            else:              # eight, one mix for two elements
                h = ref.mix(blk * 128 + (i % 256) // 2, seed) >> (np.uint32(16) * (i % 2).astype(np.uint32))
                random = [((h >> np.uint32(k)) & np.uint32(255)) / 256 + 2.0 ** -9 for k in (0, 8)]
            for k, (x, have) in enumerate(((m1, gm), (q1, gq))):
                vals, scale, near = expected_f8(x[at + i], random[k].astype(np.float64), k == 1, size[k][at + i])
                assert abs(gs[k, blk] - scale) * 448 <= 8 * 2.0 ** -24 * size[k][at + i].max()
                wrong = have[at + i] != vals
                assert not (wrong & ~near).any(), (s, b, k)
            blk += 1
        at += s


def test_f8_rounding_keeps_the_mean(gpu_lib):
    """A second moment that nearest rounding would hold in place decays: sqrt(v) after 400 steps
    without gradient is b2^200 of its start.  A step moves it by 0.0005, a 125th to a 250th of the
    distance d between e4m3 values (at most an eighth of it): 400 such choices have a deviation of
    sqrt(400 / 125) d, the mean of 65,280 elements one of 0.1%; 16 random bits bias a choice by 2^-17
    d, 400 of them by 0.04%.  Within 1%.  One element of each block has a gradient that
    keeps the block's scale at rest."""
    n, b2, steps = 65536, 0.999, 400
    p = torch.zeros(n, device="cuda")
    grad = torch.zeros(n, device="cuda")
    grad[::256] = 1.0
    m8 = torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)
    q = torch.full((n,), 100.0, device="cuda")
    q[::256] = 448.0
    q8, scales = q.to(torch.float8_e4m3fn), torch.zeros((2, n // 256), device="cuda")
    start = q8.float()
    scales[1] = 1.0 / 448.0
    table = gpu_lib.adamw_table([p])
    for t in range(1, steps + 1):
        gpu_lib.adamw(table, grad, m8, q8, step=t, lr=0.0, beta2=b2, scales=scales, seed=t)
    value = (q8.float().view(-1, 256) * scales[1][:, None])[:, 1:].mean().item()
    first = (start.view(-1, 256) / 448.0)[:, 1:].mean().item()
    assert abs(value / first - b2 ** (steps / 2)) <= 0.01 * b2 ** (steps / 2)


def test_zero_state_and_zero_gradient(gpu_lib):
    """The first step from zeros, with blocks whose gradient is zero: no NaN, parameters only decay."""
    n = 600
    p = torch.ones(n, device="cuda")
    g = torch.zeros(n, device="cuda")
    g[300] = 2.0
    m8 = torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)
    q8, scales = m8.clone(), torch.zeros((2, 3), device="cuda")
    gpu_lib.adamw(gpu_lib.adamw_table([p]), g, m8, q8, step=1, scales=scales, **HP)
    want = torch.full((n,), 1 - HP["lr"] * HP["weight_decay"], dtype=torch.float64)
    want[300] -= HP["lr"]
    assert ref.off(p, want) <= 8 * 2.0 ** -24
    assert scales[:, 0].abs().sum().item() == 0 and scales[:, 1].min().item() > 0


def test_non_finite_gradient_stays_in_its_block(gpu_lib):
    for bad in (float("nan"), float("inf")):
        p, g = torch.ones(1024, device="cuda"), torch.full((1024,), 0.1, device="cuda")
        g[300] = bad
        m, v = torch.zeros(1024, device="cuda"), torch.zeros(1024, device="cuda")
        gpu_lib.adamw(gpu_lib.adamw_table([p]), g, m, v, step=1, lr=0.1)
        assert (~torch.isfinite(p)).nonzero().view(-1).tolist() == [300]
        m8 = torch.zeros(1024, device="cuda").to(torch.float8_e4m3fn)
        q8, scales = m8.clone(), torch.zeros((2, 4), device="cuda")
        p = torch.ones(1024, device="cuda")
        gpu_lib.adamw(gpu_lib.adamw_table([p]), g, m8, q8, step=1, lr=0.1, scales=scales)
        held = torch.isfinite(q8.float() * scales[1].repeat_interleave(256))
        assert not held[300] and bool(held[:256].all()) and bool(held[512:].all())
        assert (~torch.isfinite(p)).nonzero().view(-1).tolist() == [300]


def test_non_finite_states_stay(gpu_lib):
    """A step with a finite gradient does not make a non-finite moment finite again."""
    m8 = torch.zeros(512, device="cuda")
    m8[7] = float("nan")
    m8, q8 = m8.to(torch.float8_e4m3fn), torch.ones(512, device="cuda")
    q8[9] = float("nan")
    q8 = q8.to(torch.float8_e4m3fn)
    scales = torch.full((2, 2), 0.01, device="cuda")
    p = torch.ones(512, device="cuda")
    gpu_lib.adamw(gpu_lib.adamw_table([p]), torch.ones(512, device="cuda"), m8, q8, step=2, lr=0.1, scales=scales)
    assert (~torch.isfinite(m8.float())).nonzero().view(-1).tolist() == [7]
    assert (~torch.isfinite(q8.float())).nonzero().view(-1).tolist() == [9]
    assert (~torch.isfinite(p)).nonzero().view(-1).tolist() == [7, 9]


def test_many_tensors(gpu_lib):
    """More tensors than a launch takes, empty ones among them, each with decay or not."""
    sizes = [(i * 37) % 300 for i in range(700)]
    p, g, m, v = make(sizes, torch.float32, torch.float32, seed=2)
    decay = [i % 3 == 0 for i in range(len(sizes))]
    params = [t.clone().cuda() for t in torch.split(p, sizes)]
    want = reference(p.double(), g.double(), m.double(), v.double(), sizes, decay, 5)
    gm, gv = m.cuda(), v.cuda()
    gpu_lib.adamw(gpu_lib.adamw_table(params, decay), g.cuda(), gm, gv, step=5, **HP)
    got = torch.cat([t.reshape(-1) for t in params])
    assert off_terms(got, want[0], step_terms(p, g, m, v, 5)) <= 8 * 2.0 ** -24
    assert off_terms(gm, want[1], terms(g, m)) <= 8 * 2.0 ** -24


def test_views_at_odd_places_and_repeatable(gpu_lib):
    """Parameters, gradient and states that start at odd elements of larger buffers; what lies
    between them stays; a second run from the same state gives the same bits; another stream."""
    sizes = [5, 513, 2, 4097]
    n = sum(sizes)
    outs = []
    for _ in range(2):
        gen = torch.Generator().manual_seed(9)
        buf = ref.rand(gen, n + 64, dtype=torch.bfloat16).cuda()
        params, at = [], 1
        for s in sizes:
            params.append(buf[at:at + s])
            at += s + 3
        keep = buf.clone()
        grad = ref.rand(gen, n + 1, dtype=torch.bfloat16).cuda()[1:]
        m8 = torch.zeros(n + 3, device="cuda").to(torch.float8_e4m3fn)
        q8 = m8.clone()
        table = gpu_lib.adamw_table(params)
        scales = torch.zeros((2, table.blocks), device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for t in (1, 2):
                gpu_lib.adamw(table, grad, m8[3:], q8[3:], step=t, scales=scales, seed=t, **HP)
        torch.cuda.current_stream().wait_stream(s)
        inside = torch.zeros(n + 64, dtype=torch.bool)
        at = 1
        for k in sizes:
            inside[at:at + k] = True
            at += k + 3
        assert torch.equal(buf.cpu()[~inside], keep.cpu()[~inside])
        assert not torch.equal(buf.cpu()[inside], keep.cpu()[inside])
        assert bool((m8[:3].float() == 0).all())
        outs.append((buf, m8.float(), q8.float(), scales))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.slow
def test_more_than_32_bit_offsets(gpu_lib):
    """One tensor of 2^32 + 777 elements: its last elements step like those of a small one."""
    n = (1 << 32) + 777
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough memory")
    p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-300:] = 0.25
    g[:300] = -0.25
    m8 = torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    q8 = torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    table = gpu_lib.adamw_table([p])
    scales = torch.zeros((2, table.blocks), device="cuda")
    gpu_lib.adamw(table, g, m8, q8, step=1, lr=0.5, weight_decay=0.0, scales=scales)
    assert torch.allclose(p[-300:].float(), torch.full((300,), 0.5, device="cuda"))
    assert torch.allclose(p[:300].float(), torch.full((300,), 1.5, device="cuda"))
    assert bool((p[300:-300] == 1).all())
    # 777 elements: 256, 256, 256 and a block of 9
    assert (scales[0, -4:] > 0).tolist() == [False, True, True, True]


def test_refusals(gpu_lib):
    p, g = torch.ones(512, device="cuda"), torch.ones(512, device="cuda")
    m, v = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda")
    table = gpu_lib.adamw_table([p])
    ok = dict(table=table, grad=g, moment1=m, moment2=v, step=1, lr=0.1)
    for bad in (dict(step=0), dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0),
                dict(eps=1e-60), dict(weight_decay=float("inf"))):
        with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
            gpu_lib.adamw(**{**ok, **bad})
    with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
        gpu_lib.adamw(**{**ok, "moment2": m})   # the same memory twice
    with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
        gpu_lib.adamw(**{**ok, "grad": p})      # the parameters themselves
    with pytest.raises(gpu_lib.BkmooError, match="EINVAL"):
        gpu_lib.adamw(**{**ok, "master": torch.zeros(512, device="cuda")})  # of fp32 parameters
    m8 = m.to(torch.float8_e4m3fn)
    for bad in (dict(grad=g[:511]), dict(moment1=m8), dict(moment1=m8, moment2=m8.clone()), dict(grad=g.cpu()),
                dict(scales=torch.zeros((2, 2), device="cuda")), dict(grad_scale=torch.ones(2, device="cuda")),
                dict(moment1=m8, moment2=m8.clone(), scales=torch.zeros((2, 3), device="cuda"))):
        with pytest.raises(ValueError):
            gpu_lib.adamw(**{**ok, **bad})
    for bad in ([], [p, p.bfloat16()], [p[::2]], [p.cpu()]):
        with pytest.raises(ValueError):
            gpu_lib.adamw_table(bad)
    with pytest.raises(ValueError):
        gpu_lib.adamw_table([p], [True, False])
    assert bool((p == 1).all())
