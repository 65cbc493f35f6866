"""The Python example of a layer's step in README.md runs as written, step after step."""

import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_readme_layer_example_runs(gpu_lib):
    block = re.findall(r"```python\n(.*?)```", open(README).read(), re.S)[1]
    env = {}
    exec(compile(block, "README.md", "exec"), env)
    torch.cuda.synchronize()
    g, update, flat, master = env["g"], env["update"], env["flat"], env["master"]
    # every language has a gradient of every parameter, and the step moved the parameters
    assert g.shape == (env["K"], flat.numel()) and bool(torch.isfinite(g).all())
    assert bool((g.abs().amax(1) > 0).all())
    assert update.shape == flat.shape and bool(torch.isfinite(update).all())
    assert torch.equal(flat, master.to(flat.dtype)) and not torch.equal(flat, env["before"])
    assert bool((env["scales"] > 0).all()) and bool(torch.isfinite(env["v"].float()).all())
