"""Tables of adamw(): tensors in any order in memory."""

import random

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("many,order", [(300, "descending"), (300, "mixed"), (1500, "mixed"), (2300, "descending")])
def test_neighbours_in_any_order(gpu_lib, many, order):
    """Views of one buffer, one directly after another, listed in another order than they lie in.  fp32: eight
    roundings of 2^-24 of the parameter and of a step of at most lr."""
    gen = random.Random(many)
    sizes = [gen.choice([0, 1, 3, 40, 300]) for _ in range(many)]
    n = sum(sizes)
    tgen = torch.Generator().manual_seed(31)
    flat = ref.rand(tgen, n)
    buf = flat.cuda()
    views, spans, at = list(torch.split(buf, sizes)), [], 0
    for k in sizes:
        spans.append((at, k))
        at += k
    turn = list(range(many))
    turn.reverse() if order == "descending" else gen.shuffle(turn)
    g = ref.rand(tgen, n, scale=0.1)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    gpu_lib.adamw(gpu_lib.adamw_table([views[i] for i in turn]), g.cuda(), m, v, step=1, lr=0.01, weight_decay=0.1)
    place = torch.cat([torch.arange(spans[i][0], sum(spans[i])) for i in turn])
    want = flat.double()
    z = torch.zeros(n, dtype=torch.float64)
    want[place] = ref.adamw(want[place], g.double(), z, z, 1, 0.01, 0.9, 0.999, 1e-8, 0.1)[0]
    assert ((buf.double().cpu() - want).abs() <= 8 * 2.0 ** -24 * (flat.abs().double() + 0.01)).all()


def one_step(lib, table, n, **kw):
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    lib.adamw(table, torch.ones(n, device="cuda"), m, v, step=1, lr=0.1, weight_decay=0.0, **kw)


def test_a_parameter_that_moved_is_refused(gpu_lib):
    """A table holds addresses: after a parameter's storage was replaced, a step is refused, the memory of old stays
    allocated as long as the table, and a new table takes the parameters where they are."""
    for move in ("data", "module", "storage"):
        model = torch.nn.Linear(8, 8, device="cuda")
        params = list(model.parameters())
        n = sum(p.numel() for p in params)
        table = gpu_lib.adamw_table(params)
        old = params[0].data_ptr()
        one_step(gpu_lib, table, n)
        before = [p.detach().clone() for p in params]
        if move == "data":
            params[0].data = params[0].data.clone()
        elif move == "module":
            model.bfloat16()
        else:
            params[0].data.untyped_storage().resize_(0)
        others = [torch.zeros(64, device="cuda") for _ in range(50)]  # would take freed memory
        if move != "storage":
            assert old not in [t.data_ptr() for t in others]
        with pytest.raises(ValueError, match="adamw_table"):
            one_step(gpu_lib, table, n)
        torch.cuda.synchronize()
        assert all(bool((t == 0).all()) for t in others)
        if move == "data":
            assert all(torch.equal(p, q) for p, q in zip(params, before))
            one_step(gpu_lib, gpu_lib.adamw_table(params), n)
            assert not torch.equal(params[0], before[0])


def test_a_parameter_written_in_place_stays(gpu_lib):
    """Values may change between steps: loading a checkpoint into the parameters keeps the table."""
    p = torch.nn.Parameter(torch.ones(100, device="cuda"))
    table = gpu_lib.adamw_table([p])
    with torch.no_grad():
        p.copy_(torch.full((100,), 3.0))
    one_step(gpu_lib, table, 100)
    assert torch.allclose(p, torch.full((100,), 2.9, device="cuda"))
