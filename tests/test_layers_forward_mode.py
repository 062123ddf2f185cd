"""Forward-mode derivatives of the stage's layers are refused, whichever operand has the tangent and whether or not
gradients are recorded: a call that went by it would hand out a derivative of zero.  On the CPU, with the
kernels' calls in plain torch."""

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import layer_stand_ins


@pytest.fixture
def mpc(monkeypatch):
    import paper_2401_07788_gb300 as m
    from paper_2401_07788_gb300 import layers

    layer_stand_ins.install(monkeypatch, layers)
    return m


def calls(mpc):
    x, w, b, r = torch.randn(4, 8), torch.randn(5, 8), torch.randn(5), torch.randn(4, 5)
    linear = lambda *t: mpc.linear(*t, act="gelu", p=0.5, seed=1)  # noqa: E731
    drop = lambda *t: mpc.dropout(t[0], 0.5, 1, residual=t[1])  # noqa: E731
    return [(linear, [x, w, b, r]), (drop, [r, r + 1])]


@pytest.mark.parametrize("which,operand", [(0, 0), (0, 1), (0, 2), (0, 3), (1, 0), (1, 1)])
@pytest.mark.parametrize("recorded", [False, True])
def test_tangents_raise(mpc, which, operand, recorded):
    call, operands = calls(mpc)[which]
    with forward_ad.dual_level(), torch.set_grad_enabled(recorded):
        call(*operands)  # no tangent: as ever
        operands[operand] = forward_ad.make_dual(operands[operand], torch.ones_like(operands[operand]))
        with pytest.raises((RuntimeError, NotImplementedError), match="forward"):
            call(*operands)


@pytest.mark.parametrize("which", [0, 1])
def test_modules_and_views(mpc, which):
    module = [mpc.Linear(8, 4), mpc.Dropout(0.5, seed=1)][which]
    x = torch.randn(3, 5, 8)
    with forward_ad.dual_level(), torch.no_grad():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for t in (dual, dual.transpose(0, 1)):
            with pytest.raises((RuntimeError, NotImplementedError), match="forward"):
                module(t)
