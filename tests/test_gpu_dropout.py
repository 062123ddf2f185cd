"""Dropout from the counter-based generator, against splitmix64 on the host."""

import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


def plain(x, r, p, seed):
    """One fp32 rounding of the product, one of the sum, one to the type: bit for bit."""
    keep = forms.kept(seed, x.numel(), p).view(x.shape).float().cuda()
    y = torch.where(keep > 0, x.float() * keep, torch.zeros((), device="cuda"))
    return (y if r is None else r.float() + y).to(x.dtype)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("shape", [(1,), (3,), (4,), (5,), (8,), (31,), (16, 1024), (7, 333), (3, 5, 7), (1000, 1003), (257, 4096)])
def test_sizes(mpc, shape, residual, kind):
    gen = torch.Generator().manual_seed(len(shape))
    x = torch.randn(shape, generator=gen).to(forms.KINDS[kind]).cuda()
    r = torch.randn(shape, generator=gen).to(x.dtype).cuda() if residual else None
    for p, seed in ((0.1, 0), (0.5, 2 ** 64 - 1), (0.123, 12345 << 32)):
        assert torch.equal(mpc.mpc_dropout(x, p, seed, residual=r), plain(x, r, p, seed))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("off", [1, 2, 3, 4, 8])
def test_any_alignment(mpc, off, kind):
    base = torch.randn(3, 5000).to(forms.KINDS[kind]).cuda()
    x, r = base[0, off:4001 + off], base[1, 1:4002]
    y = torch.full((4100,), 7.0, dtype=x.dtype, device="cuda")
    mpc.mpc_dropout(x, 0.3, 9, residual=r, y=y[off:4001 + off])
    assert torch.equal(y[off:4001 + off], plain(x, r, 0.3, 9))
    assert (y[:off] == 7).all() and (y[4001 + off:] == 7).all()


def test_in_place_and_gradient(mpc):
    x = torch.randn(100, 77, device="cuda")
    r = torch.randn(100, 77, device="cuda")
    want = plain(x, r, 0.2, 5)
    a, c = x.clone(), r.clone()
    assert mpc.mpc_dropout(a, 0.2, 5, residual=r, y=a) is a and torch.equal(a, want)
    assert mpc.mpc_dropout(x, 0.2, 5, residual=c, y=c) is c and torch.equal(c, want)
    x.requires_grad_(True)
    r.requires_grad_(True)
    dy = torch.randn(100, 77, device="cuda")
    gx, gr = torch.autograd.grad(mpc.dropout(x, 0.2, 5, r), (x, r), dy)
    assert torch.equal(gx, plain(dy, None, 0.2, 5)) and torch.equal(gr, dy)


def test_ends_of_p(mpc):
    x = torch.randn(1000, device="cuda")
    x[5], x[6] = float("nan"), float("inf")
    assert torch.equal(mpc.mpc_dropout(x, 0.0, 1).nan_to_num(7.0), x.nan_to_num(7.0))
    assert torch.equal(mpc.mpc_dropout(x, 1.0, 1), torch.zeros_like(x))
    y = mpc.mpc_dropout(x, 0.5, 1)
    mask = forms.kept(1, 1000, 0.5).cuda() > 0
    assert torch.equal(y[5].isnan(), mask[5]) and torch.equal(y[6].isinf(), mask[6])


def test_share_and_mean(mpc):
    """2^24 entries: the kept share is p's within 5 standard deviations, for neighbouring seeds alike, and the masks of
    two seeds agree as often as independent ones would."""
    n, p = 1 << 24, 0.3
    x = torch.ones(n, device="cuda")
    masks = [mpc.mpc_dropout(x, p, seed) > 0 for seed in (7, 8)]
    q = 1.0 - p
    for m in masks:
        assert abs(m.double().mean().item() - q) <= 5 * (p * q / n) ** 0.5
    same = (masks[0] == masks[1]).double().mean().item()
    want = q * q + p * p
    assert abs(same - want) <= 5 * (want * (1 - want) / n) ** 0.5


def test_step_counter_and_capture(mpc):
    x = torch.randn(4097, device="cuda")
    step = torch.tensor([3], dtype=torch.int64, device="cuda")
    assert torch.equal(mpc.mpc_dropout(x, 0.4, 100, step=step), mpc.mpc_dropout(x, 0.4, 103))
    graph = torch.cuda.CUDAGraph()
    mpc.mpc_dropout(x, 0.4, 100, step=step)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = mpc.mpc_dropout(x, 0.4, 100, step=step)
        step.add_(1)
    for k in range(3):
        graph.replay()
        assert torch.equal(y, mpc.mpc_dropout(x, 0.4, 103 + k))
    step.fill_(-2)
    assert torch.equal(mpc.mpc_dropout(x, 0.4, 1, step=step), mpc.mpc_dropout(x, 0.4, -1))


def test_many_entries(mpc):
    """Entries from 2^32 on have draws of their own number (bf16, 8 GiB each way)."""
    n = (1 << 32) + 1027
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = mpc.mpc_dropout(x, 0.5, 3, y=x)
    tail = y[-2048:].float().cpu()
    import numpy as np

    with np.errstate(over="ignore"):
        i = np.arange(n - 2048, n, dtype=np.uint64)
        z = np.uint64(3) + (i // np.uint64(4) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z ^= z >> np.uint64(31)
    want = ((z >> (np.uint64(16) * (i % np.uint64(4)))) & np.uint64(0xFFFF)) >= 32768
    assert torch.equal(tail > 0, torch.from_numpy(want))


def test_nothing(mpc):
    assert mpc.mpc_dropout(torch.empty(0, 5, device="cuda"), 0.5).shape == (0, 5)
