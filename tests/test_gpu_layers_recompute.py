"""Recomputation (torch.utils.checkpoint) of the stage's layers with dropout: outputs and gradients are bit for bit
those of the run without it."""

import pytest
import torch
from torch.utils.checkpoint import checkpoint

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


class Body(torch.nn.Module):
    def __init__(self, mpc, dtype):
        super().__init__()
        on = {"device": "cuda", "dtype": dtype}
        self.norm = mpc.RMSNorm(64, **on)
        self.up = mpc.Linear(64, 160, act="gelu", p=0.5, seed=1, **on)
        self.down = mpc.Linear(160, 64, p=0.5, seed=2, **on)
        self.drop = mpc.Dropout(0.5, seed=3)

    def forward(self, x):
        y, h = self.norm(x, x)
        return self.drop(self.down(self.up(y)).square(), residual=h)


def run(mpc, kind, dtype, each):
    torch.manual_seed(4)
    body = Body(mpc, dtype)
    seen = []
    for _ in range(2):
        xs = [torch.randn(5, 7, 64, device="cuda").to(dtype).requires_grad_(True) for _ in range(each)]
        ys = [body(x) if kind is None else checkpoint(body, x, use_reentrant=kind == "reentrant") for x in xs]
        for y in ys:
            y.float().square().sum().backward()
        seen += [y.detach() for y in ys] + [x.grad for x in xs] + [p.grad for p in body.parameters()]
        body.zero_grad()
    return seen


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["reentrant", "not reentrant"])
@pytest.mark.parametrize("each", [1, 2])
def test_recomputation(mpc, each, kind, dtype):
    for a, b in zip(run(mpc, None, dtype, each), run(mpc, kind, dtype, each)):
        assert torch.equal(a, b)
    assert mpc.mpc_get_status() == 0
