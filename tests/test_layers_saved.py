"""What the linear layer keeps for its gradient: x for that of w, and to refuse second derivatives through an
activation.  On the CPU, with the kernels' calls in plain torch."""

import pytest
import torch

import layer_forms as forms
import layer_stand_ins


@pytest.fixture
def mpc(monkeypatch):
    import paper_2401_07788_gb300 as m
    from paper_2401_07788_gb300 import layers

    layer_stand_ins.install(monkeypatch, layers)
    return m


@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("need", [(1, 1, 1), (1, 0, 0), (1, 0, 1), (0, 1, 0), (0, 0, 1), (0, 1, 1)])
def test_what_keeps_x(mpc, need, act):
    ops = [torch.randn(*s, dtype=torch.float64, requires_grad=bool(n)) for s, n in zip(((6, 8), (5, 8), (5,)), need)]
    x, w, b = ops
    dy = torch.randn(6, 5, dtype=torch.float64)
    y = mpc.linear(x, w, b, act=act)
    node = y.grad_fn if hasattr(y.grad_fn, "saved_tensors") else y.grad_fn.next_functions[0][0]
    held = [t for t in node.saved_tensors if t is not None]
    mine = [t for t in held if t.data_ptr() == x.data_ptr()]
    assert bool(mine) == bool(need[1] or act)
    got = torch.autograd.grad(y, [t for t in ops if t.requires_grad], dy)
    want = torch.autograd.grad(forms.linear(x, w, b, None, act)[0], [t for t in ops if t.requires_grad], dy)
    for a, c in zip(got, want):
        assert torch.allclose(a, c, rtol=1e-12, atol=1e-14)


def test_second_derivatives_with_a_frozen_w(mpc):
    """Through an activation they are not zero, and raise; without one the gradient depends on neither x nor z."""
    x, w = torch.randn(6, 8, dtype=torch.float64, requires_grad=True), torch.randn(5, 8, dtype=torch.float64)
    y = mpc.linear(x, w, act="gelu")
    (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable"):
        torch.autograd.grad(y.sum() + g.square().sum(), x)
    y = mpc.linear(x, w)
    (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    (h,) = torch.autograd.grad((x * x).sum() + g.square().sum(), x)
    assert torch.equal(h, 2 * x)
    (g,) = torch.autograd.grad(mpc.linear(x, w).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable"):
        torch.autograd.grad(g.sum(), x)
