"""The stage's layers as modules: together in a block with a boundary behind it, their gradients through
autograd, their seeds, captured steps."""

import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


class Block(torch.nn.Module):
    """h -> h + down(gelu(up(norm(h + x))))  as a stage uses the layers: x comes out of the block before."""

    def __init__(self, mpc, width, hidden, p, dtype=None, step=None):
        super().__init__()
        self.norm = mpc.RMSNorm(width, device="cuda", dtype=dtype)
        self.up = mpc.Linear(width, hidden, act="gelu", device="cuda", dtype=dtype)
        self.down = mpc.Linear(hidden, width, p=p, seed=3, step=step, device="cuda", dtype=dtype)
        self.drop = mpc.Dropout(p, seed=4, step=step)

    def forward(self, x, h):
        y, h = self.norm(x, h)
        return self.drop(self.down(self.up(y)), residual=h)


def plain_block(block, x, h, call):
    """The same from the modules' weights in 64 bits, with the masks of training call number `call`."""
    h = x + h
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + block.norm.eps) * block.norm.weight.double()
    a = forms.act(y @ block.up.weight.double().t() + block.up.bias.double(), "gelu")
    a = a @ block.down.weight.double().t() + block.down.bias.double()
    if block.training and block.drop.p:
        for m in (block.down, block.drop):
            a = a * forms.kept((m.seed << 32) + call, a.numel(), m.p).view(a.shape).cuda()
    return h + a


def rel(a, b):
    return ((a.double() - b.double()).norm() / b.double().norm().clamp_min(1e-300)).item()


@pytest.mark.parametrize("dtype,most", [(torch.float32, 3e-6), (torch.bfloat16, 2e-2)])
@pytest.mark.parametrize("shape,hidden", [((3, 50, 64), 200), ((2, 7, 33), 65)])
def test_block_and_gradients(mpc, shape, hidden, dtype, most):
    """Forward and all gradients over two training calls.  fp32: three products in a row, each off by a few
    2^-24 sqrt(terms) of its result; bf16: five roundings of 2^-8 in a row at most, 2e-2."""
    torch.manual_seed(0)
    block = Block(mpc, shape[-1], hidden, 0.25, dtype)
    for call in (1, 2):
        x, h, dy = (torch.randn(shape, device="cuda").to(dtype) for _ in range(3))
        x.requires_grad_(True)
        h.requires_grad_(True)
        out = block(x, h)
        leaves = [x, h, *block.parameters()]
        grads = torch.autograd.grad(out, leaves, dy)
        xd, hd = x.detach().double().requires_grad_(True), h.detach().double().requires_grad_(True)
        want = plain_block(block, xd, hd, call)
        wants = torch.autograd.grad(want, [xd, hd, *block.parameters()], dy.double())
        assert rel(out, want) < most
        for g, w in zip(grads, wants):
            assert g.shape == w.shape and rel(g, w) < 2 * most
    block.eval()
    with torch.no_grad():
        assert rel(block(x, h), plain_block(block, x.double(), h.double(), 0)) < most
    assert mpc.mpc_get_status() == 0


def test_stages_with_boundaries(mpc):
    """Two stages with a compressed boundary between them: the layers' gradient is what the boundary sends back."""
    torch.manual_seed(1)

    class Stage(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.block = Block(mpc, 64, 128, 0.0)

        def forward(self, x):
            return self.block(x, torch.zeros_like(x))

    first, second = Stage(), Stage()
    body = mpc.with_boundaries([first, second], lambda i: mpc.CompressionBoundary(mpc.Quant(8), mpc.Quant(8), rows="last"))
    x = torch.randn(4, 16, 64, device="cuda")
    dy = torch.randn(4, 16, 64, device="cuda")
    out = body(x)
    out.backward(dy)
    a = first(x)
    rows = a.detach().reshape(-1, 64)
    sent = mpc.mpc_quant_decompress(*mpc.mpc_quant_compress(rows, 8), 64, 8).view_as(a).requires_grad_(True)
    want = second(sent)
    assert torch.equal(out, want)
    (back,) = torch.autograd.grad(want, sent, dy)
    rows = back.reshape(-1, 64).contiguous()
    back = mpc.mpc_quant_decompress(*mpc.mpc_quant_compress(rows, 8), 64, 8).view_as(a)
    grads = torch.autograd.grad(a, list(first.parameters()), back)
    for p, g in zip(first.parameters(), grads):
        assert torch.equal(p.grad, g)


def test_norm_that_sends_8_bits(mpc):
    torch.manual_seed(2)
    x = torch.randn(5, 9, 96, device="cuda", requires_grad=True)
    norm = mpc.RMSNorm(96, bits=8, device="cuda")
    y = norm(x)
    codes, scale, minv, _, rstd = mpc.mpc_rms_norm_quant(x.detach().view(-1, 96), norm.weight.detach(), norm.eps)
    assert torch.equal(y.view(-1, 96), mpc.mpc_quant_decompress(codes, scale, minv, 96, 8))
    dy = torch.randn_like(y)
    gx, gw = torch.autograd.grad(y, (x, norm.weight), dy)
    wx, ww = mpc.mpc_rms_norm_backward(dy.view(-1, 96), x.detach().view(-1, 96), norm.weight.detach(), rstd)
    assert torch.equal(gx.view(-1, 96), wx) and torch.equal(gw, ww)


def test_only_one_output_of_the_norm_is_used(mpc):
    x, r = (torch.randn(6, 40, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.ones(40, device="cuda", requires_grad=True)
    y, h = mpc.rms_norm(x, w, residual=r)
    gx, gr, gw = torch.autograd.grad(h, (x, r, w), torch.ones_like(h), retain_graph=True, allow_unused=True)
    assert (gx == 1).all() and (gr == 1).all() and gw is None
    gx, gr, gw = torch.autograd.grad(y, (x, r, w), torch.ones_like(y))
    assert torch.equal(gx, gr) and gw is not None
    y, h = mpc.rms_norm(x.detach(), w, residual=r.detach())
    (gw2,) = torch.autograd.grad(y, w, torch.ones_like(y))
    assert torch.equal(gw, gw2)


@pytest.mark.parametrize("p", [0.0, 0.5])
def test_one_tensor_twice_and_broadcast(mpc, p):
    """The same leaf as input and residual, an expanded input, an expanded gradient."""
    x = torch.randn(12, 32, device="cuda", requires_grad=True)
    w = torch.randn(32, 32, device="cuda", requires_grad=True)
    mask = forms.kept(9, 12 * 32, p).view(12, 32).cuda() if p else 1.0
    out = mpc.linear(x, w, residual=x, p=p, seed=9)
    gx, gw = torch.autograd.grad(out.sum(), (x, w))
    want = x.double() @ w.double().t() * mask + x.double()
    wx, ww = torch.autograd.grad(want.sum(), (x, w))
    assert rel(gx, wx) < 1e-5 and rel(gw, ww) < 1e-5
    row = torch.randn(1, 32, device="cuda", requires_grad=True)
    out = mpc.linear(row.expand(12, 32), w)
    (g,) = torch.autograd.grad(out, row, torch.ones(1, 1, device="cuda").expand(12, 32))
    (want,) = torch.autograd.grad(row.double().expand(12, 32) @ w.double().t(), row, torch.ones(12, 32, device="cuda").double())
    assert rel(g, want) < 1e-5
    y = mpc.dropout(row.expand(12, 32), 0.5, 3, residual=x)
    (g,) = torch.autograd.grad(y.sum(), row)
    assert rel(g[0], forms.kept(3, 12 * 32, 0.5).view(12, 32).cuda().sum(0)) < 1e-6


def test_frozen_parts_form_no_gradient(mpc):
    x = torch.randn(8, 16, device="cuda")
    w = torch.randn(24, 16, device="cuda", requires_grad=True)
    (gw,) = torch.autograd.grad(mpc.linear(x, w, act="silu").sum(), w)
    x2 = x.clone().requires_grad_(True)
    (gx,) = torch.autograd.grad(mpc.linear(x2, w.detach(), act="silu").sum(), x2)
    both = torch.autograd.grad(mpc.linear(x2, w, act="silu").sum(), (x2, w))
    assert torch.equal(gx, both[0]) and torch.equal(gw, both[1])


def test_second_derivatives_raise(mpc):
    x = torch.randn(8, 16, device="cuda", requires_grad=True)
    w = torch.randn(16, 16, device="cuda", requires_grad=True)
    n = torch.ones(16, device="cuda", requires_grad=True)
    for out in (mpc.linear(x, w, act="gelu"), mpc.dropout(x, 0.5, 1), mpc.rms_norm(x, n)):
        (g,) = torch.autograd.grad((out * out).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="not differentiable"):
            torch.autograd.grad(g.sum(), x)


def test_a_changed_counter_is_noticed(mpc):
    """A device counter advanced between the passes would give the backward pass another mask: autograd refuses."""
    x = torch.randn(8, 16, device="cuda", requires_grad=True)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    y = mpc.dropout(x, 0.5, 1, step=step)
    step.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_capture_needs_a_counter(mpc):
    drop = mpc.Dropout(0.5, seed=1)
    x = torch.randn(64, device="cuda")
    drop(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(mpc.MpcError, match="device counter"):
        with torch.cuda.graph(graph):
            drop(x)


def test_captured_training_step(mpc):
    """Forward and backward of a block in one graph: every replay takes the counter's next masks, as an eager step
    with the same counter does."""
    torch.manual_seed(3)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    block = Block(mpc, 96, 160, 0.3, step=step)
    x, h, dy = (torch.randn(20, 96, device="cuda") for _ in range(3))
    params = list(block.parameters())

    def pass_():
        out = block(x, h)
        return (out, *torch.autograd.grad(out, params, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pass_()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = pass_()
        step.add_(1)
    seen = []
    for k in range(3):
        graph.replay()
        replayed = [t.clone() for t in held]
        step.fill_(k)
        eager = pass_()
        step.fill_(k + 1)
        for a, b in zip(replayed, eager):
            assert torch.equal(a, b)
        seen.append(replayed[0])
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_copies_of_a_module(mpc):
    """A state dict holds the weights; copies and pickles keep seed and count."""
    import copy
    import io

    a = mpc.Linear(16, 8, act="silu", p=0.5, device="cuda")
    x = torch.randn(4, 16, device="cuda")
    a(x)
    b = copy.deepcopy(a)
    buf = io.BytesIO()
    torch.save(a, buf)
    buf.seek(0)
    c = torch.load(buf, weights_only=False)
    want = a(x)
    assert torch.equal(b(x), want) and torch.equal(c(x), want)
    assert set(a.state_dict()) == {"weight", "bias"}


def test_the_example_runs_on_the_layers(mpc):
    """A few steps of the training example with dropout: finite losses, and every layer gets a gradient."""
    import importlib.util
    import os

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("train_stages", os.path.join(root, "examples", "train_stages.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(steps=3, vocab=200, width=64, stages=2, blocks=1, batch=4, length=32, dropout=0.1, log=None)
    assert bool(losses.isfinite().all())
    stage = example.Stage(64, 2, dropout=0.1).cuda()
    x = torch.randn(2, 16, 64, device="cuda", requires_grad=True)
    stage(x).sum().backward()
    for p in (x, *stage.parameters()):
        assert p.grad is not None and bool(p.grad.isfinite().all()) and p.grad.abs().sum() > 0
