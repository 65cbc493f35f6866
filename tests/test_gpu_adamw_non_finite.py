"""What a non-finite gradient does to 8-bit moments: exactly the elements that bkmoo_adamw's description names."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("beta2", [0.95, 0.999])
def test_elements_that_become_non_finite(gpu_lib, bad, beta2):
    """A NaN: its own element alone.  An infinity: its block's moments, and its block's parameters with the next step."""
    n, at, block = 1000, 300, list(range(256, 512))
    gen = torch.Generator().manual_seed(11)
    g = (0.1 * torch.randn(n, generator=gen)).cuda()
    outs = []
    for value in (bad, 0.0):
        grad = g.clone()
        grad[at] = value
        p = torch.ones(n, device="cuda")
        m8 = torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)
        q8, scales = m8.clone(), torch.zeros((2, 4), device="cuda")
        table, seen = gpu_lib.adamw_table([p]), []
        for step in (1, 2):
            gpu_lib.adamw(table, grad if step == 1 else g, m8, q8, step=step, lr=0.1, beta2=beta2, scales=scales)
            of = torch.arange(n, device="cuda") // 256
            seen.append([p.clone(), m8.float() * scales[0][of], q8.float() * scales[1][of]])
        outs.append(seen)
    own = [at] if bad != bad else block
    for step, want_p in ((0, [at]), (1, own)):
        for name, t, want in zip(("p", "m", "q"), outs[0][step], (want_p, own, own)):
            assert (~torch.isfinite(t)).nonzero().view(-1).tolist() == want, (step, name)
    # the others are what they are with a zero in its place
    for step in (0, 1):
        for t, u in zip(outs[0][step], outs[1][step]):
            rest = torch.isfinite(t)
            assert torch.equal(t[rest], u[rest])
