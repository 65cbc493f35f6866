"""The input gradient where its sum is split in many parts and workgroups go through several of them, at sizes that
choose this by themselves: du Wg + dv Wu is one sum of two segments, and a part ends before, at or behind the border.

Against the 64-bit definition (on the GPU, plain products).  fp32: two sums of at most 2 F products, 4 sqrt(2 F) 2^-24,
and 50 x 2^-24 for the activation; bf16: 2^-8 x 1.5 more for the two roundings."""

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,D,F,dtype", [(1, 4352, 1216, torch.float32), (257, 1024, 4096, torch.float32),
                                         (66, 5764, 10196, torch.float32), (1, 4480, 11648, torch.bfloat16),
                                         (280, 5440, 15104, torch.bfloat16), (1030, 4096, 14336, torch.bfloat16)])
def test_input_gradient_of_many_parts(gpu_lib, M, D, F, dtype):
    print(f"case ffn input gradient M={M} D={D} F={F} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(41)
    rand = lambda *s, scale=1.0: torch.randn(s, generator=gen, device="cuda").mul_(scale).to(dtype)  # noqa: E731
    x, dy, u, v = rand(M, D), rand(M, D), rand(M, F), rand(M, F)
    wg, wu, wd = rand(F, D, scale=D ** -0.5), rand(F, D, scale=D ** -0.5), rand(D, F, scale=F ** -0.5)
    grads = torch.empty((1, 3 * D * F), dtype=dtype, device="cuda")
    dw = list(torch.split(grads, D * F, dim=1))
    dx = gpu_lib.ffn_backward(dy, x, u, v, wg, wu, wd, dw_gate=dw[0], dw_up=dw[1], dw_down=dw[2])
    a, da = ref.act(u.double(), "silu")
    dh = dy.double() @ wd.double()
    want = (dh * v.double() * da) @ wg.double() + (dh * a) @ wu.double()
    tol = (4 * (2 * F) ** 0.5 + 50) * 2.0 ** -24 + (1.5 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    assert ref.off(dx, want.cpu()) <= tol
