"""A call on a stream of the caller's choice beside work that is still queued on the current one, on memory that has
been given back to the allocator: neither gets at the other's."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


def calls(mpc):
    gen = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    x, w, dy, weight = rnd(300, 512), rnd(640, 512), rnd(300, 640), rnd(512)
    y, h, rstd = mpc.mpc_rms_norm_forward(x, weight)
    targets = torch.randint(0, 640, (300,), generator=gen).cuda()
    return [
        lambda s: (mpc.mpc_dropout(x, 0.5, 3, stream=s),),
        lambda s: mpc.mpc_rms_norm_forward(x, weight, residual=y, stream=s),
        lambda s: mpc.mpc_rms_norm_quant(x, weight, residual=y, stream=s),
        lambda s: mpc.mpc_rms_norm_backward(y, h, weight, rstd, stream=s),
        lambda s: mpc.mpc_linear_forward(x, w, act="gelu", keep=True, stream=s),
        lambda s: mpc.mpc_linear_backward(dy, x, w, stream=s),
        lambda s: mpc.mpc_linear_ce_train(x, w, targets, stream=s),
        lambda s: mpc.mpc_quant_compress(x, 8, stream=s),
        lambda s: mpc.mpc_topk_compress(x, 50, stream=s),
    ]


@pytest.mark.parametrize("which", range(9))
def test_beside_queued_work(mpc, which):
    call = calls(mpc)[which]
    want = [t.clone() for t in call(None)]
    need = [t.numel() * t.element_size() for t in want]
    if which in (3, 4, 5):  # the workspaces too
        need.append({3: mpc.mpc_rms_norm_workspace_bytes(300, 512), 4: mpc.mpc_linear_workspace_bytes(300, 512, 640),
                     5: mpc.mpc_linear_workspace_bytes(300, 512, 640, backward=True)}[which])
    side = torch.cuda.Stream()
    for write in (False, True):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        held = [torch.full((n,), 3, dtype=torch.uint8, device="cuda") for n in need]
        read = [torch.zeros_like(t) for t in held]
        torch.cuda.synchronize()
        torch.cuda._sleep(50_000_000)
        for t, r in zip(held, read):
            if write:
                t.fill_(255)
            else:
                r.copy_(t)
        del held, t
        got = call(side)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        if not write:
            assert all(bool((r == 3).all()) for r in read)
    assert mpc.mpc_get_status() == 0


def test_outputs_given_back_while_they_are_read(mpc):
    """An output of a side stream that the current stream reads and gives back: a later call on the side stream waits for
    that read before it takes the memory again."""
    x = torch.randn(1000, 1000, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = mpc.mpc_dropout(x, 0.5, 1)
    y = mpc.mpc_dropout(x, 0.5, 1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(50_000_000)
    seen = torch.empty_like(x)
    seen.copy_(y)
    del y
    mpc.mpc_dropout(x, 0.5, 2, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(seen, want)


def test_captured_on_a_side_stream(mpc):
    """A graph whose side branch is such a call."""
    x, w = torch.randn(200, 256, device="cuda"), torch.randn(300, 256, device="cuda")
    want, _ = mpc.mpc_linear_forward(x, w, act="silu")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        y, _ = mpc.mpc_linear_forward(x, w, act="silu", stream=side)
        main.wait_stream(side)
        twice = y + y
    for _ in range(2):
        twice.zero_()
        graph.replay()
        assert torch.equal(twice, want + want)
