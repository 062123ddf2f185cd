"""Gradient calls of the linear layer in a workspace of exactly the size that their query gives: the same results as
with room to spare, and nothing is written behind it."""

import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("off", [0, 1, 8])
@pytest.mark.parametrize("need", [(True, True, True), (True, False, False), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("M,K,N", [(3, 64, 128), (300, 520, 384), (1030, 136, 2056), (70, 77, 91)])
def test_enough_and_no_more(mpc, M, K, N, need, off, kind):
    gen = torch.Generator().manual_seed(M + off)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(forms.KINDS[kind]).cuda()  # noqa: E731
    x, w, dy = rnd(M, K + off)[:, off:], rnd(N, K + off)[:, off:], rnd(M, N + off)[:, off:]
    on = lambda t: 0 if t.data_ptr() % 16 else t.stride(0)  # noqa: E731
    for act, p in ((None, 0.0), (None, 0.25), ("gelu", 0.0)):
        plain = act is None and p == 0.0
        _, z = mpc.mpc_linear_forward(x, w, act=act, p=p, seed=5, keep=act is not None)
        size = mpc.mpc_linear_workspace_bytes(M, K, N, x.dtype, backward=True, ldx=on(x), ldw=on(w), lddy=on(dy), plain=plain)
        more = mpc.mpc_linear_workspace_bytes(M, K, N, x.dtype, backward=True, ldx=on(x), ldw=on(w), lddy=on(dy))
        assert size <= more
        seen = []
        for n in (more, size):
            ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
            seen.append(mpc.mpc_linear_backward(dy, x, w, z, act=act, p=p, seed=5, need=need, ws=ws[:n]))
            assert (ws[n:] == 77).all(), "written behind the workspace"
        for a, c, wanted in zip(*seen, need):
            assert a is c is None if not wanted else torch.equal(a, c)
        if plain:  # the formula, over what a sum of that many terms may be off by
            dys, xs, ws_ = dy.double(), x.double(), w.double()
            u = forms.half(x.dtype)
            for got, a, b, count in zip(seen[1], (dys, dys.t(), None), (ws_, xs, None), (N, M, M)):
                if got is None:
                    continue
                want = dys.sum(0) if a is None else a @ b
                terms = dys.abs().sum(0) if a is None else a.abs() @ b.abs()
                e = (count + 16) * forms.F32 * terms
                forms.close(got, want, e + u * (want.abs() + e))
    assert mpc.mpc_get_status() == 0


def test_memory_of_a_plain_gradient(mpc):
    """bf16 without activation and dropout: beside the gradients, room for db's sums and the tiles in parts."""
    M, K, N = 8192, 512, 8192
    x, w, dy = (torch.randn(*s, device="cuda").bfloat16() for s in ((M, K), (N, K), (M, N)))
    mpc.mpc_linear_backward(dy, x, w)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    mpc.mpc_linear_backward(dy, x, w)
    torch.cuda.synchronize()
    peak = torch.cuda.max_memory_allocated() - before
    assert peak - 2 * (M * K + N * K + N) < M * N * 2 // 2
