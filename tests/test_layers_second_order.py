"""Second derivatives of the linear layer by its bias: with an activation the gradients depend on the bias through z, so
they hang on it too, and differentiating them by it raises instead of leaving the term out.  On the CPU, with the
kernels' calls in plain torch."""

import pytest
import torch

import layer_stand_ins


@pytest.fixture
def mpc(monkeypatch):
    import paper_2401_07788_gb300 as m
    from paper_2401_07788_gb300 import layers

    layer_stand_ins.install(monkeypatch, layers)
    return m


@pytest.mark.parametrize("of", ["x", "w", "b"])
@pytest.mark.parametrize("alone", [False, True])
def test_by_the_bias(mpc, of, alone):
    """alone: nothing but `of` and the bias takes a gradient."""
    t = {n: torch.randn(*s, dtype=torch.float64) for n, s in (("x", (6, 8)), ("w", (5, 8)), ("b", (5,)))}
    for n in t:
        t[n].requires_grad_(n in (of, "b") or not alone)
    y = mpc.linear(t["x"], t["w"], t["b"], act="gelu")
    (g,) = torch.autograd.grad(y.sum(), t[of], create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable"):
        torch.autograd.grad(y.sum() + g.square().sum(), t["b"])


def test_without_an_activation(mpc):
    """Nothing depends on the bias: the other terms' derivative is handed out."""
    x, w, b = (torch.randn(*s, dtype=torch.float64, requires_grad=True) for s in ((6, 8), (5, 8), (5,)))
    y = mpc.linear(x, w, b)
    (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    (h,) = torch.autograd.grad((b * b).sum() + g.square().sum(), b)
    assert torch.equal(h, 2 * b)
