"""The layer operators in 64 bits, on the CPU: plain definitions, and inputs.

Written from the formulas alone; shares no code with the library."""

import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half the distance of neighbours, relative


def rms(x, eps):
    return torch.sqrt((x * x).mean(1, keepdim=True) + eps)


def norm_forward(r, y, w, p, g, c, eps):
    b = y if p is None else p * (y / rms(y, eps))
    b = b if g is None else g * b
    out = r + c * b
    return out, w * (out / rms(out, eps))


def by_task(x, rows):
    return torch.stack([x[a:b].sum(0) for a, b in zip(rows, rows[1:])])


def norm_backward(up, dn, r, y, w, p, g, c, eps, rows):
    """dresid, dy, and the tasks' dweight, dpost, dgate."""
    one = torch.ones(r.shape[1], dtype=torch.float64)
    pp, gg = one if p is None else p, one if g is None else g
    s = rms(r, eps)
    x = r / s
    a = w * dn
    dr = (a - x * (x * a).mean(1, keepdim=True)) / s + (0.0 if up is None else up)
    e = c * gg * pp * dr
    if p is None:
        z, dy = y, e
    else:
        t = rms(y, eps)
        z = y / t
        dy = (e - z * (z * e).mean(1, keepdim=True)) / t
    return dr, dy, by_task(dn * x, rows), by_task(c * gg * dr * z, rows), by_task(c * pp * dr * z, rows)


def act(u, name):
    """a(u), a'(u)"""
    if name == "silu":
        s = torch.sigmoid(u)
        return u * s, s + u * s * (1 - s)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (u + 0.044715 * u ** 3))
    return 0.5 * u * (1 + t), 0.5 * (1 + t) + 0.5 * u * (1 - t * t) * k * (1 + 3 * 0.044715 * u * u)


def ffn_forward(x, wg, wu, wd, name):
    u, v = x @ wg.T, x @ wu.T
    return (act(u, name)[0] * v) @ wd.T, u, v


def ffn_backward(dy, x, u, v, wg, wu, wd, name, rows):
    """dx and the tasks' dWg, dWu [K, F, D], dWd [K, D, F]."""
    a, da = act(u, name)
    dh = dy @ wd
    du, dv, h = dh * v * da, dh * a, a * v
    per = lambda m, n: torch.stack([m[b:e].T @ n[b:e] for b, e in zip(rows, rows[1:])])  # noqa: E731
    return du @ wg + dv @ wu, per(du, x), per(dv, x), per(dy, h)


def adamw(p, g, m, v, step, lr, b1, b2, eps, wd):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * wd) - lr * (m / (1 - b1 ** step)) / (torch.sqrt(v / (1 - b2 ** step)) + eps), m, v


def mix(pair, seed):
    """Four random bytes for each pair of elements (numpy uint32)."""
    k = np.uint32(0x9E3779B1)
    with np.errstate(over="ignore"):
        h = pair.astype(np.uint32) * k + np.uint32(seed)
        h = (h ^ (h >> np.uint32(16))) * k
        h = (h ^ (h >> np.uint32(15))) * k
    return h ^ (h >> np.uint32(16))


def e4m3_values():
    """The non-negative finite e4m3 values, ascending."""
    return np.array([m * 2.0 ** -9 for m in range(8)] +
                    [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)])


def rand(gen, *shape, dtype=torch.float32, scale=1.0, mean=0.0):
    return (torch.randn(*shape, generator=gen) * scale + mean).to(dtype)


def off(got, want):
    """2-norm of the difference over the 2-norm of what is wanted."""
    d = (got.double().cpu() - want).norm().item()
    n = want.norm().item()
    return d / n if n else (0.0 if d == 0 else math.inf)
