"""Steps that give no seed draw other random bits each: 8-bit moments keep their mean."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def state(n):
    """No gradient but in one element of each block, which keeps the block's scale at rest."""
    grad = torch.zeros(n, device="cuda")
    grad[::256] = 1.0
    q = torch.full((n,), 100.0, device="cuda")
    q[::256] = 448.0
    scales = torch.zeros((2, n // 256), device="cuda")
    scales[1] = 1.0 / 448.0
    return grad, torch.zeros(n, device="cuda").to(torch.float8_e4m3fn), q.to(torch.float8_e4m3fn), scales


def test_steps_without_a_seed_keep_the_mean(gpu_lib):
    """sqrt(v) after 400 steps without gradient is b2^200 of its start.  400 choices, each within a 125th to a
    250th of the distance d of e4m3 values (an eighth of the value at most), have a deviation of sqrt(400 / 125) d, the
    mean of 65,280 elements one of 0.1%; 16 random bits bias 400 choices by 0.04%.  Within 1%."""
    n, b2, steps = 65536, 0.999, 400
    grad, m8, q8, scales = state(n)
    first = q8.float().view(-1, 256)[:, 1:].mean().item() / 448.0
    table = gpu_lib.adamw_table([torch.zeros(n, device="cuda")])
    for t in range(1, steps + 1):
        gpu_lib.adamw(table, grad, m8, q8, step=t, lr=0.0, beta2=b2, scales=scales)
    value = (q8.float().view(-1, 256) * scales[1][:, None])[:, 1:].mean().item()
    assert abs(value / first - b2 ** (steps / 2)) <= 0.01 * b2 ** (steps / 2)


def test_the_seed_of_a_step_is_its_number(gpu_lib):
    """Without a seed a step repeats bit for bit, and is the one whose seed is the step's number."""
    n = 4096
    outs = []
    for kw in (dict(), dict(), dict(seed=7), dict(seed=8)):
        grad, m8, q8, scales = state(n)
        gpu_lib.adamw(gpu_lib.adamw_table([torch.zeros(n, device="cuda")]), grad, m8, q8, step=7, lr=0.0, beta2=0.999,
                      scales=scales, **kw)
        outs.append(q8.view(torch.uint8).clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert not torch.equal(outs[0], outs[3])
