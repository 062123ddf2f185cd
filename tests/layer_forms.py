"""The stage's layers in plain torch and 64 bits, and what the kernels' results may be off by.

Half a step of a type, eps / 2 of it, is what one rounding may change.  Sums of n terms in fp32, in any
order, are off by at most (n + c) 2^-24 times the sum of the terms' magnitudes, c for the few operations before
and after (16 here); every other tolerance is added up from those two."""

import math

import numpy as np
import torch

F32 = 2.0 ** -24
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}
# largest second derivative of each activation (z phi'' ... at 0: 2 phi(0) for both gelus; silu 1/2; relu none)
CURVE = {None: 0.0, "relu": 0.0, "gelu": 0.8, "gelu_tanh": 0.81, "silu": 0.5}
# largest first derivative
STEEP = {None: 1.0, "relu": 1.0, "gelu": 1.13, "gelu_tanh": 1.13, "silu": 1.1}


def half(t):
    return torch.finfo(t).eps / 2


def kept(seed, n, p):
    """Dropout's factors of n entries, from splitmix64 as published, as float64 on the host."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed % 2 ** 64) + (np.arange((n + 3) // 4, dtype=np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z ^= z >> np.uint64(31)
    parts = np.stack([(z >> np.uint64(16 * i)) & np.uint64(0xFFFF) for i in range(4)], axis=1).reshape(-1)[:n]
    level = int(math.floor(p * 65536 + 0.5))
    factor = 65536.0 / (65536 - level) if level < 65536 else 0.0
    return torch.from_numpy((parts >= np.uint64(level)).astype(np.float64) * factor)


def act(z, name):
    if name == "relu":
        return torch.relu(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def linear(x, w, b=None, r=None, name=None, mask=None):
    z = x.double() @ w.double().t()
    if b is not None:
        z = z + b.double()
    y = act(z, name)
    if mask is not None:
        y = y * mask
    return y if r is None else y + r.double(), z


def linear_bound(x, w, b, r, name, mask, y, kind):
    """What y of the kernels may be off by, entry by entry."""
    k = x.shape[1]
    terms = x.double().abs() @ w.double().abs().t() + (0.0 if b is None else b.double().abs())
    e = (k + 16) * F32 * terms * STEEP[name]
    if name is not None:  # the activation in fp32: a few of its steps, and 1.5e-7 of z where erfc is a formula's
        e = e + terms * (8 * F32 + (3e-7 if kind == torch.bfloat16 else 0.0))
    if mask is not None:
        e = e * mask
    e = e + 4 * F32 * (y.abs() + (0.0 if r is None else 2 * r.double().abs()))
    return e + half(kind) * (y.abs() + e)


def linear_grads(dy, x, w, z, name=None, mask=None):
    g = dy.double() if mask is None else dy.double() * mask
    if name is not None:
        t = z.double().requires_grad_(True)
        g = g * torch.autograd.grad(act(t, name).sum(), t)[0]
    return g @ w.double(), g.t() @ x.double(), g.sum(0), g


def linear_grad_bounds(dy, x, w, z, g, dx, dw, db, name, mask, kind, z_off):
    """What the gradients may be off by: dz by its rounding, by that of z (half a step of it, and z_off that
    z's own sum may be off by) through the second derivative, and a few fp32 steps; then the sums."""
    d = dy.double().abs() if mask is None else dy.double().abs() * mask
    slope = 16 * F32 * (1.0 + z.double().abs()) + (1e-6 if kind == torch.bfloat16 else 0.0)
    off = d * (CURVE[name] * (half(kind) * z.double().abs() + z_off) + (slope if name is not None else 0.0)) + 4 * F32 * g.abs()
    sharp = off
    if kind == torch.bfloat16 and (name is not None):
        off = off + half(kind) * (g.abs() + off)
    m, n, k = x.shape[0], w.shape[0], x.shape[1]
    gm, xa, wa = g.abs() + off, x.double().abs(), w.double().abs()
    out = []
    for e, terms, count, v in ((off @ wa, gm @ wa, n, dx), (off.t() @ xa, gm.t() @ xa, m, dw),
                               (sharp.sum(0), gm.sum(0), m, db)):
        e = e + (count + 16) * F32 * terms
        out.append(e + half(kind) * (v.abs() + e))
    return out


def close(got, want, bound, what=""):
    """Every entry within its bound (a few 2^-53 of slack for the plain form itself)."""
    got, want = got.double().cpu(), want.cpu()
    bound = bound.cpu() + 1e-12 * want.abs() + 1e-300
    bad = (got - want).abs() > bound
    worst = ((got - want).abs() / bound).max().item() if got.numel() else 0.0
    assert not bad.any() and got.isfinite().all(), "%s: %d of %d entries out of bounds, worst %.3g times" % (
        what, int(bad.sum()), got.numel(), worst)
    return worst
