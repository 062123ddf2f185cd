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


def test_a_long_sum_of_one_sign_is_not_one_sided(mpc):  # noqa: F811
    """dh over 262144 entries that are positive (or negative) throughout a column, the largest first.  With
    hidden states of 0 all probabilities are equal and exact in bf16, which leaves the sums' truncation, at
    most 1.7e-7 of the sum in each of 512 steps, and the rounding of 4096 results: its mean along the
    result stays within 6 of its deviations of 2.5e-5."""
    T, D, V = 4096, 4096, 262144
    gen = torch.Generator(device="cuda").manual_seed(7)
    w = torch.rand(V, D, device="cuda", generator=gen).add_(0.5)
    w *= torch.exp2(torch.rand(D, device="cuda", generator=gen)) * (torch.arange(D, device="cuda") % 2 * 2 - 1)
    w *= torch.exp2(torch.linspace(8, 0, V, device="cuda"))[:, None]
    w = w.bfloat16()
    w[5] = 0.0
    want = torch.stack([x.double().sum(0) for x in w.split(8192)]).sum(0) / V / T
    h = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    dh = mpc.mpc_linear_ce_train(h, w, torch.full((T,), 5, device="cuda"))[1][T - 1].double()
    along = float((dh * want).sum() / (want * want).sum()) - 1.0
    assert abs(along) <= 512 * 1.7e-7 + 6 * 2.5e-5, along


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [65536, 65537, 140001])
def test_many_tokens(mpc, dtype, T):  # noqa: F811
    """More tokens than a CTA of the list counts by itself, a fifth of them ignored, some targets out of range."""
    h, w, y = inputs(T, 24, 40, dtype, seed=80)
    masked = y.clone()
    for i, bad in ((0, 40), (T // 2, -7), (T - 1, 1 << 40)):
        y[i], masked[i] = bad, -100
    want = bounds(h, w, masked, None)
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    near(loss, want["loss"], "loss")
    near(lse, want["lse"], "lse")
    assert mpc.mpc_get_status() == 6
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    near(loss, want["loss"], "loss (train)")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")
    assert mpc.mpc_get_status() == 6
