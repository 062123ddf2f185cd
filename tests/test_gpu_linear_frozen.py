"""The linear layer's gradient without x, where that of w is not formed: the same results, and without an activation x is
given back as soon as the forward call is done."""

import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("need", [(True, False, False), (True, False, True), (False, False, True), (False, False, False)])
@pytest.mark.parametrize("M,K,N,off", [(3, 40, 64, 0), (150, 96, 130, 0), (70, 65, 77, 1)])
def test_without_x(mpc, M, K, N, off, need, kind):
    gen = torch.Generator().manual_seed(M)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(forms.KINDS[kind]).cuda()  # noqa: E731
    x, w, dy = rnd(M, K + off)[:, off:], rnd(N, K + off)[:, off:], rnd(M, N + off)[:, off:]
    for act in (None, "gelu"):
        _, z = mpc.mpc_linear_forward(x, w, act=act, keep=act is not None)
        want = mpc.mpc_linear_backward(dy, x, w, z, act=act, p=0.2, seed=3, need=need)
        got = mpc.mpc_linear_backward(dy, None, w, z, act=act, p=0.2, seed=3, need=need)
        for a, c, n in zip(got, want, need):
            assert a is c is None if not n else torch.equal(a, c)
    assert mpc.mpc_get_status() == 0


def test_refusals(mpc):
    dy, w = torch.zeros(4, 8, device="cuda"), torch.zeros(8, 16, device="cuda")
    with pytest.raises(mpc.MpcError):
        mpc.mpc_linear_backward(dy, None, w)  # dw is wanted
    for bad_dy, bad_w in ((dy, w.bfloat16()), (dy, w.cpu()), (dy, w[:5]), (dy[0], w), (dy, w[:, :0])):
        with pytest.raises(mpc.MpcError):
            mpc.mpc_linear_backward(bad_dy, None, bad_w, need=(True, False, False))


def test_memory_of_x(mpc):
    w = torch.randn(256, 2048, device="cuda")
    leaf = torch.randn(4096, 2048, device="cuda", requires_grad=True)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = mpc.linear(leaf * 2.0, w)
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated() - before
    assert held <= y.numel() * 4 + (1 << 16)
    (g,) = torch.autograd.grad(y.sum(), leaf)
    assert g.shape == leaf.shape
