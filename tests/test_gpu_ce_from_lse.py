"""The gradient that is formed from lse (the backward call, and training in pieces) for more bf16 tokens
than a row tile, against the formulas in 64 bits: the bounds of test_gpu_linear_ce, and for dw one
rounding of 2^-8 more, that of the scaled hidden states."""

import pytest
import torch

from test_gpu_linear_ce import inputs, mpc, near, oracle  # noqa: F401

pytestmark = pytest.mark.gpu


def bounds(h, w, y, gloss):
    want = oracle(h, w, y, gloss)
    rows = (y != -100).nonzero()[:, 0]
    hd, wd = h[rows].double(), w.double()
    c = torch.softmax(hd @ wd.t(), 1)
    c[torch.arange(len(rows), device="cuda"), y[rows]] -= 1.0
    g = torch.full((len(rows),), 1.0 / max(len(rows), 1), device="cuda") if gloss is None else gloss[rows]
    c *= g.double()[:, None]
    want["dw"] = (want["dw"][0], want["dw"][1] + 2.0 ** -8 * (c.abs().t() @ hd.abs()))
    return want


@pytest.mark.parametrize("kind", ["plain", "sure", "hopeless", "both", "weights", "some weights 0", "same target"])
@pytest.mark.parametrize("T,D,V", [(257, 32, 600), (700, 72, 900), (1500, 33, 70)])
def test_gradient_from_lse(mpc, T, D, V, kind):  # noqa: F811
    h, w, y = inputs(T, D, V, torch.bfloat16, seed=60, ignored=0.1)
    gloss = None
    if kind in ("sure", "hopeless", "both"):
        w = (w.float() / w.float().norm(dim=1, keepdim=True)).bfloat16()
        lot = torch.arange(T, device="cuda") % 3 == 0
        sign = torch.full((T, 1), 400.0 if kind == "sure" else -400.0, device="cuda")
        if kind == "both":
            sign[::2] = 400.0
        h = torch.where((lot & (y >= 0))[:, None], (w.float()[y.clamp_min(0)] * sign).bfloat16(), h)
    elif kind in ("weights", "some weights 0"):
        gloss = torch.randn(T, device="cuda")
        if kind != "weights":
            gloss[::2] = 0.0
    elif kind == "same target":
        y[y >= 0] = 5
    want = bounds(h, w, y, gloss)
    _, lse = mpc.mpc_linear_ce_forward(h, w, y)
    for dh, dw in (mpc.mpc_linear_ce_backward(h, w, y, lse, gloss), mpc.mpc_linear_ce_backward(h, w, y, lse, gloss, piece=64),
                   mpc.mpc_linear_ce_train(h, w, y, gloss, piece=max(V // 2, 1))[1:]):
        near(dh, want["dh"], "dh")
        near(dw, want["dw"], "dw")
    assert mpc.mpc_get_status() == 0
