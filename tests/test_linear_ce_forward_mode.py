"""Forward-mode derivatives of linear_cross_entropy are refused: a call that went by its autograd function would hand
out a derivative of zero.  On the CPU, with the kernels' calls in plain torch."""

import pytest
import torch
import torch.autograd.forward_ad as forward_ad


@pytest.fixture
def mpc(monkeypatch):
    import paper_2401_07788_gb300 as m
    from paper_2401_07788_gb300 import training

    def forward(h, w, targets, ignore_index=-100):
        logits = h @ w.t()
        lse = torch.logsumexp(logits, 1)
        return lse - logits.gather(1, targets[:, None])[:, 0], lse

    def train(h, w, targets, *_):
        return forward(h, w, targets)[0], torch.zeros_like(h), torch.zeros_like(w)

    monkeypatch.setattr(training, "mpc_linear_ce_forward", forward)
    monkeypatch.setattr(training, "mpc_linear_ce_train", train)
    return m


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("operand", [0, 1])
@pytest.mark.parametrize("recorded", [False, True])
def test_tangents_raise(mpc, reduction, operand, recorded):
    operands = [torch.randn(6, 8), torch.randn(10, 8)]
    targets = torch.arange(6)
    with forward_ad.dual_level(), torch.set_grad_enabled(recorded):
        mpc.linear_cross_entropy(*operands, targets, reduction=reduction)  # no tangent: as ever
        operands[operand] = forward_ad.make_dual(operands[operand], torch.ones_like(operands[operand]))
        with pytest.raises((RuntimeError, NotImplementedError), match="forward"):
            mpc.linear_cross_entropy(*operands, targets, reduction=reduction)
