"""Infinities of the down projection, and products at the end of bf16's range, in the block's forward pass: the
same for few rows, whose hidden values are held as two bf16, as for many."""

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("F", [136, 135])  # rows at multiples of four bytes, and not
@pytest.mark.parametrize("M", [1, 5, 8, 9, 64, 65])
def test_infinite_weights_of_the_down_projection(gpu_lib, M, F, dtype):
    """y[:, d] = sum_f h[:, f] w[d, f]: where one w[d, f] is infinite y[:, d] is infinite with its sign times h[:, f]'s,
    and the other columns are what they are without it (tolerance: sums of at most 136 products of fp32, and two bf16
    roundings, as in the block's other tests)."""
    D = 72
    gen = torch.Generator().manual_seed(21)
    x = ref.rand(gen, M, D, dtype=dtype)
    wg, wu = (ref.rand(gen, F, D, dtype=dtype, scale=D ** -0.5) for _ in range(2))
    wd = ref.rand(gen, D, F, dtype=dtype, scale=F ** -0.5)
    wd[3, 10], wd[5, 20], wd[70, F - 1] = float("inf"), float("-inf"), float("inf")
    y = gpu_lib.ffn_forward(x.cuda(), wg.cuda(), wu.cuda(), wd.cuda())[0].double().cpu()
    want = ref.ffn_forward(x.double(), wg.double(), wu.double(), wd.double(), "silu")[0]
    assert not bool(torch.isnan(want).any())
    inf = torch.isinf(want)
    assert inf.any(0).nonzero().view(-1).tolist() == [3, 5, 70]
    assert torch.equal(y[inf], want[inf])
    fine = [d for d in range(D) if d not in (3, 5, 70)]
    tol = (4 * 136 ** 0.5 + 50) * 2.0 ** -24 + (1.5 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    assert ref.off(y[:, fine], want[:, fine]) <= tol


@pytest.mark.parametrize("F", [16, 15])
@pytest.mark.parametrize("M", [1, 8])
def test_hidden_values_at_the_end_of_the_range(gpu_lib, M, F):
    """h = (129/128 2^64) (254/128 2^63) = 1.99988 2^127 is finite in fp32 and rounds to infinity in bf16.  Few
    rows hold it as two bf16: times an eighth it is 0.24998 2^127, one rounding to bf16 from there."""
    D = 8
    x = torch.zeros((M, D), dtype=torch.bfloat16)
    x[:, 0] = 1.0
    wg, wu = torch.zeros((F, D), dtype=torch.bfloat16), torch.zeros((F, D), dtype=torch.bfloat16)
    wg[0, 0], wu[0, 0], wu[1, 0], wg[1, 0] = 129 / 128 * 2.0 ** 64, 254 / 128 * 2.0 ** 63, -254 / 128 * 2.0 ** 63, \
        129 / 128 * 2.0 ** 64
    wd = torch.zeros((D, F), dtype=torch.bfloat16)
    wd[:, 0] = 0.125
    wd[4:, 0], wd[4:, 1] = 0.0, 0.125
    y = gpu_lib.ffn_forward(x.cuda(), wg.cuda(), wu.cuda(), wd.cuda())[0].double().cpu()
    want = ref.ffn_forward(x.double(), wg.double(), wu.double(), wd.double(), "silu")[0]
    assert bool(torch.isfinite(want).all())
    assert bool(((y - want).abs() <= 2.0 ** -8 * want.abs()).all())
