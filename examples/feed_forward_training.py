"""Multilingual training steps of a small feed-forward stack, on the library alone.

    python examples/feed_forward_training.py [--layers 2] [--width 512] [--inner 1408]
        [--languages 4] [--tokens 2048] [--steps 60] [--method mgda] [--states f8]

Each step is one pass over a batch whose rows are sorted by language:

    forward    residual_norm_forward and ffn_forward, layer by layer
    backward   the same operators backwards; every language's weight gradients land in its
               row of the [K, N] gradient buffer
    resolve    one conflict-free update of the K rows, bucket by bucket
    AdamW      over all tensors at once, moments in 8 or 32 bits, a 32-bit copy of the bf16
               parameters, the gradient clipped by its norm on the device

The task is made up: a fixed random stack of the same shape labels the tokens, turned a little
differently for every language, so that the languages' gradients agree in part and conflict in
part.  Prints each language's loss as it falls.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_05613_amd import bkmoo  # noqa: E402

SCALE = 0.5  # of every block's contribution to the residual stream


class Stack:
    """Layers of (gated feed-forward block, norm after it, gate, residual, norm before the next) with
    their parameters one after another in one flat buffer, as the gradients are."""

    def __init__(self, layers: int, width: int, inner: int, dtype=torch.bfloat16, seed: int = 0):
        self.shapes = [("norm", (width,))]
        for i in range(layers):
            self.shapes += [(f"{i}.gate", (inner, width)), (f"{i}.up", (inner, width)), (f"{i}.down", (width, inner)),
                            (f"{i}.post", (width,)), (f"{i}.scale", (width,)), (f"{i}.norm", (width,))]
        self.layers, sizes = layers, [torch.Size(s).numel() for _, s in self.shapes]
        self.offsets = [0]
        for n in sizes:
            self.offsets.append(self.offsets[-1] + n)
        self.N = self.offsets[-1]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.flat = torch.ones(self.N, dtype=dtype, device="cuda")
        self.at = {}
        for (name, shape), o, n in zip(self.shapes, self.offsets, sizes):
            p = self.flat[o:o + n].view(shape)
            if len(shape) == 2:
                p.normal_(0.0, shape[1] ** -0.5, generator=gen)
            self.at[name] = p

    def forward(self, x: torch.Tensor):
        """The last norm's output, and what the backward pass needs."""
        p, kept = self.at, []
        r, n = bkmoo.residual_norm_forward(torch.zeros_like(x), x, p["norm"])
        kept.append((r, x))
        for i in range(self.layers):
            y, u, v = bkmoo.ffn_forward(n, p[f"{i}.gate"], p[f"{i}.up"], p[f"{i}.down"], save=True)
            inputs = n
            r, n = bkmoo.residual_norm_forward(r, y, p[f"{i}.norm"], p[f"{i}.post"], p[f"{i}.scale"], SCALE)
            kept.append((r, y, inputs, u, v))
        return n, kept

    def backward(self, dn: torch.Tensor, kept, rows, grads: torch.Tensor):
        """Every language's gradient of all parameters to its row of `grads` [K, N]."""
        p = self.at
        cut = {name: grads[:, o:e] for (name, _), o, e in zip(self.shapes, self.offsets, self.offsets[1:])}
        dr = None
        for i in reversed(range(self.layers)):
            r, y, inputs, u, v = kept[i + 1]
            dr, dy = bkmoo.residual_norm_backward(dr, dn, r, y, p[f"{i}.norm"], p[f"{i}.post"], p[f"{i}.scale"], SCALE,
                                                  task_rows=rows, dweight=cut[f"{i}.norm"],
                                                  dpost_weight=cut[f"{i}.post"], dgate=cut[f"{i}.scale"])
            dn = bkmoo.ffn_backward(dy, inputs, u, v, p[f"{i}.gate"], p[f"{i}.up"], p[f"{i}.down"], task_rows=rows,
                                    dw_gate=cut[f"{i}.gate"], dw_up=cut[f"{i}.up"], dw_down=cut[f"{i}.down"])
        r, x = kept[0]
        bkmoo.residual_norm_backward(dr, dn, r, x, p["norm"], task_rows=rows, dweight=cut["norm"])


class Trainer:
    def __init__(self, model: Stack, languages: int, method: str, states: str, lr: float):
        self.model, self.method, self.lr, self.steps = model, method, lr, 0
        N, f8 = model.N, states == "f8"
        self.grads = torch.zeros((languages, N), dtype=model.flat.dtype, device="cuda")
        # a bucket for every layer's tensors, and one for the first norm
        self.buckets = torch.tensor([0] + [o for (n, _), o in zip(model.shapes, model.offsets) if n.endswith(".gate")]
                                    + [N], dtype=torch.int64, device="cuda")
        self.table = bkmoo.adamw_table([model.at[n] for n, _ in model.shapes], [len(s) == 2 for _, s in model.shapes])
        kind = torch.float8_e4m3fn if f8 else torch.float32
        self.m = torch.zeros(N, device="cuda").to(kind)
        self.v = torch.zeros(N, device="cuda").to(kind)
        self.scales = torch.zeros((2, self.table.blocks), device="cuda") if f8 else None
        self.master = model.flat.float() if model.flat.dtype == torch.bfloat16 else None

    def step(self, x: torch.Tensor, target: torch.Tensor, rows) -> torch.Tensor:
        """One training step; the languages' losses before it."""
        self.steps += 1
        n, kept = self.model.forward(x)
        off = n.float() - target.float()
        count = torch.tensor([max(1, e - b) for b, e in zip(rows, rows[1:])], device="cuda")
        per_row = 0.5 * off.square().mean(1)
        losses = torch.stack([per_row[b:e].mean() for b, e in zip(rows, rows[1:])])
        weight = torch.repeat_interleave(1.0 / count, torch.tensor([e - b for b, e in zip(rows, rows[1:])],
                                                                   device="cuda"))
        dn = (off * (weight / off.shape[1])[:, None]).to(n.dtype)  # of every language's own mean loss
        self.model.backward(dn, kept, rows, self.grads)
        update = bkmoo.resolve(self.grads, self.buckets, self.method)
        clip = torch.clamp(1.0 / (torch.linalg.vector_norm(update.float()) + 1e-6), max=1.0).view(1)
        bkmoo.adamw(self.table, update, self.m, self.v, step=self.steps, lr=self.lr, beta2=0.95, master=self.master,
                    scales=self.scales, grad_scale=clip, seed=self.steps)
        return losses


def data(languages: int, tokens: int, width: int, inner: int, layers: int, seed: int = 1):
    """A batch sorted by language, in ragged shares, and its targets."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = [0]
    for k in range(languages):
        rows.append(tokens * (k + 1) * (k + 2) // (languages * (languages + 1)))
    x = torch.empty((tokens, width), device="cuda").normal_(0.0, 1.0, generator=gen).to(torch.bfloat16)
    teacher, _ = Stack(layers, width, inner, seed=99).forward(x)
    turn = torch.empty((languages, width), device="cuda").normal_(0.0, 0.3, generator=gen)
    language = torch.repeat_interleave(torch.arange(languages, device="cuda"),
                                       torch.tensor([e - b for b, e in zip(rows, rows[1:])], device="cuda"))
    return x, (teacher.float() + turn[language]).to(torch.bfloat16), rows


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--inner", type=int, default=1408)
    ap.add_argument("--languages", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--method", default="mgda", choices=["mgda", "pcgrad", "cagrad", "mean"])
    ap.add_argument("--states", default="f8", choices=["f32", "f8"])
    a = ap.parse_args(argv)
    x, target, rows = data(a.languages, a.tokens, a.width, a.inner, a.layers)
    trainer = Trainer(Stack(a.layers, a.width, a.inner, seed=0), a.languages, a.method, a.states, a.lr)
    history = []
    for t in range(a.steps):
        losses = trainer.step(x, target, rows)
        history.append(losses)
        if t % max(1, a.steps // 6) == 0 or t + 1 == a.steps:
            print(f"step {t + 1:4d}  " + "  ".join(f"{v:.4f}" for v in losses.tolist()), flush=True)
    return torch.stack(history)


if __name__ == "__main__":
    main()
