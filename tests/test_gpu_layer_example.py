"""The example trains: every operator together, as a user runs them."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("feed_forward_training",
                                                  os.path.join(ROOT, "examples", "feed_forward_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("method,states", [("mgda", "f8"), ("mean", "f32")])
def test_losses_fall(gpu_lib, example, method, states):
    """Every language's loss ends at less than two thirds of where it started."""
    h = example.main(["--layers", "2", "--width", "128", "--inner", "352", "--languages", "3", "--tokens", "600",
                      "--steps", "60", "--method", method, "--states", states])
    assert bool(torch.isfinite(h).all())
    assert bool((h[-1] < h[0] * 2 / 3).all()), (h[0].tolist(), h[-1].tolist())


def test_one_pass_gives_every_languages_gradient(gpu_lib, example):
    """The gradient rows of one pass over the whole batch are those of a pass over each language's
    rows alone.  Both round activations and gradients to bf16 (2^-9 of a value on average); where the
    number of rows selects another kernel, h and sums differ in their last place, and so may the
    rounding of what follows: 2^-7 of the norm."""
    x, target, rows = example.data(3, 300, 64, 160, 2)
    model = example.Stack(2, 64, 160, seed=3)
    n, kept = model.forward(x)
    grads = torch.zeros((3, model.N), dtype=torch.bfloat16, device="cuda")
    dn = (n.float() - target.float()).to(torch.bfloat16)
    model.backward(dn, kept, rows, grads)
    for k in range(3):
        b, e = rows[k], rows[k + 1]
        nk, keptk = model.forward(x[b:e].contiguous())
        one = torch.zeros((1, model.N), dtype=torch.bfloat16, device="cuda")
        model.backward(dn[b:e].contiguous(), keptk, [0, e - b], one)
        d = (one[0].float() - grads[k].float()).norm() / grads[k].float().norm()
        assert d <= 2.0 ** -7, (k, d.item())
