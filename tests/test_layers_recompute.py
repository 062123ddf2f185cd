"""A module's masks under recomputation (torch.utils.checkpoint): the repeated forward pass takes the first one's, so
gradients are those of the run without it.  On the CPU, with the kernels' calls in plain torch."""

import pytest
import torch
from torch.utils.checkpoint import checkpoint

import layer_stand_ins

F64 = torch.float64


@pytest.fixture
def mpc(monkeypatch):
    import paper_2401_07788_gb300 as m
    from paper_2401_07788_gb300 import layers

    layer_stand_ins.install(monkeypatch, layers)
    return m


class Body(torch.nn.Module):
    """Layers that drop, with something between them that keeps their outputs for its gradient."""

    def __init__(self, mpc):
        super().__init__()
        self.up = mpc.Linear(12, 20, act="gelu", p=0.5, seed=1, dtype=F64)
        self.down = mpc.Linear(20, 12, p=0.5, seed=2, dtype=F64)
        self.drop = mpc.Dropout(0.5, seed=3)

    def forward(self, x):
        return self.drop(self.down(self.up(x)).square()).square() + x


def run(mpc, kind, calls=3, each=1, **options):
    """Outputs and gradients of `calls` steps of `each` passes before their backward pass."""
    torch.manual_seed(11)
    body = Body(mpc)
    seen = []
    for _ in range(calls):
        xs = [torch.randn(9, 12, dtype=F64, requires_grad=True) for _ in range(each)]
        ys = [body(x) if kind is None else checkpoint(body, x, use_reentrant=kind == "reentrant", **options) for x in xs]
        for y in ys:
            y.square().sum().backward()
        seen += [y.detach() for y in ys] + [x.grad for x in xs] + [p.grad for p in body.parameters()]
        body.zero_grad()
    return seen


@pytest.mark.parametrize("kind", ["reentrant", "not reentrant"])
@pytest.mark.parametrize("each", [1, 3])
def test_recomputation_takes_the_same_masks(mpc, kind, each):
    """Several steps, and several passes in flight before the first backward pass."""
    for a, b in zip(run(mpc, None, each=each), run(mpc, kind, each=each)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["reentrant", "not reentrant"])
def test_a_recomputation_inside_another(mpc, kind):
    def both(x, inner):
        body = Body(mpc)
        def middle(t):
            return checkpoint(body, t, use_reentrant=kind == "reentrant") if inner else body(t)
        y = checkpoint(middle, x, use_reentrant=kind == "reentrant") if inner else middle(x)
        y.square().sum().backward()
        return [y.detach(), x.grad, *(p.grad for p in body.parameters())]

    seen = []
    for inner in (False, True):
        torch.manual_seed(5)
        seen.append(both(torch.randn(6, 12, dtype=F64, requires_grad=True), inner))
    for a, b in zip(*seen):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["reentrant", "not reentrant"])
def test_recomputation_without_the_generator_is_refused(mpc, kind):
    """preserve_rng_state=False: nothing says whose masks a repeated pass is to take."""
    with pytest.raises(mpc.MpcError, match="recomput"):
        run(mpc, kind, calls=1, preserve_rng_state=False)


def test_a_call_too_far_back_is_refused(mpc, monkeypatch):
    from paper_2401_07788_gb300 import layers

    monkeypatch.setattr(layers._Seeded, "remembered", 4)
    drop = mpc.Dropout(0.5, seed=1)
    x = torch.ones(2, 8, dtype=F64, requires_grad=True)
    y = checkpoint(lambda t: drop(t).square(), x, use_reentrant=False)
    for _ in range(3):
        drop(x)
    (g,) = torch.autograd.grad(y.sum(), x, retain_graph=True)
    assert torch.equal(g, 2 * y.detach() / x.detach())
    for _ in range(4):
        drop(x)
    y = checkpoint(lambda t: drop(t).square(), x, use_reentrant=False)
    for _ in range(4):
        drop(x)
    with pytest.raises(mpc.MpcError, match="recomput"):
        torch.autograd.grad(y.sum(), x)


def test_seeds_follow_the_number_of_the_call(mpc):
    """New calls count on whatever is drawn between them, recomputed ones do not count; a generator that is put back
    by hand repeats its masks, as torch's own layers do."""
    drop = mpc.Dropout(0.5, seed=7)
    cpu = torch.device("cpu")
    state = torch.get_rng_state()
    assert [drop._draw(cpu)[1] - (7 << 32) for _ in range(3)] == [1, 2, 3]
    torch.set_rng_state(state)
    assert [drop._draw(cpu)[1] - (7 << 32) for _ in range(4)] == [1, 2, 3, 4]
    assert drop.calls == 4


def test_copies_and_pickles(mpc):
    """They keep seed and count, and not what only a pass in flight needs; a module saved before there was such a
    record loads."""
    import copy
    import pickle

    a = mpc.Dropout(0.5, seed=7)
    cpu = torch.device("cpu")
    a._draw(cpu)
    for b in (copy.deepcopy(a), pickle.loads(pickle.dumps(a))):
        assert b.seed == 7 and b.calls == 1 and not b._known and a._known
        assert b._draw(cpu)[1] == (7 << 32) + 2
    state = dict(a.__getstate__())
    del state["_known"]
    old = mpc.Dropout.__new__(mpc.Dropout)
    old.__setstate__(state)
    assert old._draw(cpu)[1] == (7 << 32) + 2
