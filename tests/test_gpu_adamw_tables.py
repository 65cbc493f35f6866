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
