"""The module and the optimizer as a training loop uses them: upstream factors, frozen operands, a second
backward pass, memory, targets that are out of range, states that are replaced between steps."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    torch.cuda.set_device(0)
    return m


def held(which="current"):
    """Bytes that tensors asked for (what the allocator gives for them depends on the blocks it has)."""
    return torch.cuda.memory_stats()["requested_bytes.all." + which]


def inputs(T, D, V, dtype=torch.float32, ignored=0.2):
    gen = torch.Generator(device="cuda").manual_seed(T + 7 * D + 13 * V)
    dev = {"device": "cuda", "generator": gen}
    w, h = torch.randn(V, D, **dev) / D ** 0.5, torch.randn(T, D, **dev)
    y = torch.randint(0, V, (T,), **dev)
    y[torch.randperm(T, **dev)[: int(ignored * T)]] = -100
    return h.to(dtype), w.to(dtype), y


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("of", ["h", "w", "factor"])
def test_a_second_derivative_is_refused(mpc, reduction, of):
    """Asking for it raises instead of adding nothing; gradients that are recorded but not differentiated are
    the same as ever."""
    h, w, y = inputs(50, 24, 90)
    factor = torch.full((), 0.7, device="cuda")
    {"h": h, "w": w, "factor": factor}[of].requires_grad_(True)
    x = w if of == "w" else h.requires_grad_(True)
    loss = mpc.linear_cross_entropy(h, w, y, reduction=reduction).sum() * factor
    grad, = torch.autograd.grad(loss, x, create_graph=True)
    plain, = torch.autograd.grad(mpc.linear_cross_entropy(h, w, y, reduction=reduction).sum() * factor.detach(), x)
    assert torch.equal(grad, plain)
    with pytest.raises(RuntimeError, match="not differentiable"):
        grad.square().sum().backward()


@pytest.mark.parametrize("T", [12, 500])
@pytest.mark.parametrize("factor", [1.0, 1.0 / 3.0, 0.1, -7.0])
def test_an_upstream_factor_is_not_rounded(mpc, T, factor):
    """The gradient of a bf16 mean is that of the call times the fp32 factor, rounded once."""
    h, w, y = inputs(T, 64, 300, torch.bfloat16)
    _, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    h.requires_grad_(True)
    w.requires_grad_(True)
    (mpc.linear_cross_entropy(h, w, y) * factor).backward()
    for got, plain in ((h.grad, dh), (w.grad, dw)):
        assert got.dtype == torch.bfloat16
        assert torch.equal(got, (plain.float() * factor).bfloat16())


def test_mean_and_sum_agree_in_bf16(mpc):
    """The mean's gradient with a factor against the sum's with the factor over the count, in 64 bits: a factor
    that were rounded to bf16 would be off by up to 2^-9 in all entries alike, a mean of rounding errors of
    2^-8 each over n entries stays below 2^-8 * 6 / sqrt(n)."""
    h, w, y = inputs(600, 64, 300, torch.bfloat16)
    grads = []
    for reduction, factor in (("mean", 1.0 / 3.0), ("sum", 1.0 / 3.0 / int((y != -100).sum()))):
        a, b = h.clone().requires_grad_(True), w.clone().requires_grad_(True)
        (mpc.linear_cross_entropy(a, b, y, reduction=reduction) * factor).backward()
        grads.append((a.grad.double(), b.grad.double()))
    for x, z in zip(*grads):
        ratio = float((x * z).sum() / (z * z).sum())
        assert abs(ratio - 1.0) < 2.0 ** -8 * 6 / x.numel() ** 0.5


def test_one_gradient_of_the_weight(mpc):
    """The backward pass hands out the gradients that the forward call made: no second dw."""
    h, w, y = inputs(300, 256, 50000)
    h.requires_grad_(True)
    w.requires_grad_(True)
    loss = mpc.linear_cross_entropy(h, w, y)
    before = held()
    torch.cuda.reset_peak_memory_stats()
    loss.backward()
    assert held("peak") - before < w.numel() * 4 // 2
    assert held() - before < w.numel() * 4 // 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_graph_that_is_kept(mpc, dtype):
    """Two backward passes through one graph, with factors of their own, whatever became of the first one's
    gradients."""
    h, w, y = inputs(300, 40, 500, dtype)
    _, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    h.requires_grad_(True)
    w.requires_grad_(True)
    loss = mpc.linear_cross_entropy(h, w, y)
    for factor in (0.3, 1.0 / 7.0, 1.0):
        got = torch.autograd.grad(loss, (h, w), torch.full((), factor, device="cuda"), retain_graph=True)
        for x, plain in zip(got, (dh, dw)):
            assert torch.equal(x, (plain.float() * torch.full((), factor, device="cuda")).to(dtype))
            x.fill_(float("nan"))


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_frozen_operands(mpc, reduction):
    """Only what requires a gradient gets one, the same as if both did; a frozen weight's is not kept."""
    h, w, y = inputs(300, 64, 20000)
    a, b = h.clone().requires_grad_(True), w.clone().requires_grad_(True)
    mpc.linear_cross_entropy(a, b, y, reduction=reduction).sum().backward()
    x = h.clone().requires_grad_(True)
    torch.cuda.synchronize()
    before = held()
    loss = mpc.linear_cross_entropy(x, w, y, reduction=reduction).sum()
    assert held() - before < w.numel() * 4 // 2
    loss.backward()
    assert torch.equal(x.grad, a.grad) and w.grad is None
    v = w.clone().requires_grad_(True)
    mpc.linear_cross_entropy(h, v, y, reduction=reduction).sum().backward()
    assert torch.equal(v.grad, b.grad) and h.grad is None


def test_mean_of_targets_out_of_range(mpc):
    """A target outside the vocabulary does not count: not in the loss, nor in the number that it is divided
    by, with and without gradients."""
    V = 90
    h, w, y = inputs(50, 24, V)
    y[:4] = torch.tensor([V, -1, 1 << 40, -(1 << 40)], device="cuda")
    counts = (y >= 0) & (y < V)
    loss = mpc.mpc_linear_ce_forward(h, w, y)[0]
    want = float(loss.double().sum() / counts.sum())
    masked = torch.where(counts, y, torch.full_like(y, -100))
    _, dh, dw = mpc.mpc_linear_ce_train(h, w, masked)
    with torch.no_grad():
        plain = mpc.linear_cross_entropy(h, w, y)
    h.requires_grad_(True)
    w.requires_grad_(True)
    loss = mpc.linear_cross_entropy(h, w, y)
    loss.backward()
    assert mpc.mpc_get_status() == 6
    assert torch.equal(h.grad, dh) and torch.equal(w.grad, dw)
    # a sum of 36 losses in fp32 and a quotient
    assert abs(float(plain) - want) <= 2.0 ** -20 * want and abs(float(loss.detach()) - want) <= 2.0 ** -20 * want


def test_mean_where_the_ignored_index_is_in_the_vocabulary(mpc):
    h, w, y = inputs(50, 24, 90, ignored=0.0)
    y[::3] = 5
    want = torch.nn.functional.cross_entropy(h.double() @ w.double().t(), y, ignore_index=5)
    assert abs(float(mpc.linear_cross_entropy(h, w, y, ignore_index=5)) - float(want)) < 1e-5 * float(want)


def optimizer(mpc, made, bits, **options):
    ps = [torch.nn.Parameter(x.clone()) for x in made]
    return ps, mpc.AdamW(ps, lr=1e-2, betas=(0.9, 0.95), state_bits=bits, **options)


def advance(ps, opt, grads):
    for p, g in zip(ps, grads):
        p.grad = g.clone()
    opt.step()


def same_states(a, pa, b, pb):
    for p, q in zip(pa, pb):
        assert torch.equal(p, q)
        assert a.state[p].keys() == b.state[q].keys()
        for k, x in a.state[p].items():
            assert torch.equal(x, b.state[q][k]) if isinstance(x, torch.Tensor) else x == b.state[q][k], k


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("change", ["cleared", "replaced", "exchanged"])
def test_states_that_are_replaced_between_steps(mpc, bits, change):
    """A step uses the states that the optimizer holds then, wherever they came from since the last one."""
    torch.manual_seed(1)
    made = [torch.randn(300, device="cuda"), torch.randn(40, 30, device="cuda")]
    grads = [torch.randn_like(x) for x in made]
    ps, opt = optimizer(mpc, made, bits)
    advance(ps, opt, grads)
    advance(ps, opt, grads)
    qs, other = optimizer(mpc, [p.detach() for p in ps], bits)
    if change == "cleared":
        opt.state.clear()
    else:
        names = [k for k, x in opt.state[ps[0]].items() if isinstance(x, torch.Tensor)]
        for p, q in zip(ps, qs):
            other.state[q] = {k: x.clone() if k in names else x for k, x in opt.state[p].items()}
        if change == "replaced":  # one tensor of each, by zeros
            for name in names:
                opt.state[ps[1]][name] = torch.zeros_like(opt.state[ps[1]][name])
                other.state[qs[1]][name].zero_()
        else:  # the same tensors' memory, by new ones
            for p in ps:
                for name in names:
                    opt.state[p][name].data = opt.state[p][name].clone()
    for _ in range(2):
        advance(ps, opt, grads)
        advance(qs, other, grads)
    same_states(opt, ps, other, qs)


def test_copies_that_are_replaced_between_steps(mpc):
    torch.manual_seed(2)
    made = [torch.randn(300, device="cuda")]
    grads = [torch.randn_like(x) for x in made]
    ps, opt = optimizer(mpc, made, 32)
    advance(ps, opt, grads)
    for _ in range(2):  # a copy where there was none, then another one
        opt.copies[ps[0]] = torch.zeros(300, dtype=torch.bfloat16, device="cuda")
        old = opt.copies[ps[0]]
        advance(ps, opt, grads)
        assert torch.equal(old, ps[0].detach().bfloat16())
    del opt.copies[ps[0]]
    advance(ps, opt, grads)
    assert not torch.equal(old, ps[0].detach().bfloat16())
    ps[0].data = ps[0].detach()[:200].clone()
    for k in ("exp_avg", "exp_avg_sq"):
        opt.state[ps[0]][k] = opt.state[ps[0]][k][:200].clone()
    before = ps[0].detach().clone()
    advance(ps, opt, [grads[0][:200]])
    assert not bool((ps[0].detach() == before).any())


def test_rates_that_change_between_steps(mpc):
    """lr and weight decay of the groups as they are at each step, numbers or a tensor changed in place."""
    torch.manual_seed(4)
    made, grads = [torch.randn(300, device="cuda")], [torch.randn(300, device="cuda")]
    ps, opt = optimizer(mpc, made, 32)
    qs, other = optimizer(mpc, made, 32)
    rate = torch.full((), 1e-2)
    opt.param_groups[0]["lr"] = rate
    for lr, decay in ((1e-2, 0.0), (3e-3, 0.1), (0.0, 0.1), (1e-2, 0.5)):
        rate.fill_(lr)
        other.param_groups[0]["lr"] = float(rate)
        opt.param_groups[0]["weight_decay"] = other.param_groups[0]["weight_decay"] = decay
        before = ps[0].detach().clone()
        advance(ps, opt, grads)
        advance(qs, other, grads)
        assert torch.equal(ps[0], qs[0]) and torch.equal(ps[0].detach(), before) == (lr == 0.0)


@pytest.mark.parametrize("max_norm", [0.0, 1.0])
def test_gradients_are_let_go(mpc, max_norm):
    """After step() and zero_grad() nothing holds the gradients."""
    ps, opt = optimizer(mpc, [torch.randn(4 << 20, device="cuda"), torch.randn(1000, 500, device="cuda").t().contiguous()],
                        8, max_norm=max_norm)
    bytes_of = sum(p.numel() * 4 for p in ps)
    for layout in range(2):
        for p in ps:
            p.grad = torch.randn(p.shape, device="cuda")
        if layout == 1:  # one that the step copies
            ps[1].grad = torch.randn(1000, 500, device="cuda").t()
        before = held()
        opt.step()
        opt.zero_grad()
        assert held() <= before - bytes_of + (1 << 16) + sum(
            x.numel() * x.element_size() for p in ps for x in opt.state[p].values() if isinstance(x, torch.Tensor)) * (layout == 0)


def test_lists_of_changing_parameters(mpc):
    """Any subset of the parameters may have gradients: results as with a step for each alone, and memory
    that does not grow with the number of subsets seen."""
    torch.manual_seed(3)
    made = [torch.randn(50 + i, device="cuda") for i in range(6)]
    ps, opt = optimizer(mpc, made, 32, max_norm=1e9)
    singles = [optimizer(mpc, [x], 32, max_norm=1e9) for x in made]
    sizes = []
    for turn in range(2):
        for subset in range(1, 64):
            grads = [torch.randn_like(x) if subset >> i & 1 else None for i, x in enumerate(made)]
            for p, g in zip(ps, grads):
                p.grad = None if g is None else g.clone()
            opt.step()
            for (one, each), g in zip(singles, grads):
                if g is not None:
                    one[0].grad = g.clone()
                    each.step()
                    each.zero_grad()
            opt.zero_grad()
            del grads
            sizes.append(held())
    for p, (one, _) in zip(ps, singles):
        assert torch.equal(p, one[0])
    assert sizes[-1] - sizes[5] < 20 * 32768  # a plan's workspace is 32 KB


def test_a_plan_without_gradients_is_refused(mpc):
    p, g = torch.zeros(30, device="cuda"), torch.ones(30, device="cuda")
    plan = mpc.AdamWPlan([p], [g])
    plan.drop_grads()
    for call in (lambda: mpc.mpc_adamw_step(plan, 1e-3, 0.9, 0.99, 1e-8, 1), lambda: mpc.mpc_grad_norm(plan)):
        with pytest.raises(mpc.MpcError):
            call()
    plan.set_grads([g])
    mpc.mpc_adamw_step(plan, 1e-3, 0.9, 0.99, 1e-8, 1)
    assert bool((p < 0).all())


@pytest.mark.parametrize("reduction", ["mean", "sum"])
def test_pieces_of_the_vocabulary(mpc, reduction):
    """`piece` bounds what a training step holds: without it the exponentials of all logits, three bf16 planes
    in fp32; with it those of a piece."""
    T, D, V = 2048, 64, 50257
    results = []
    for piece in (0, 2048):
        h, w, y = inputs(T, D, V)
        head = mpc.LinearCrossEntropy(D, V, reduction=reduction, device="cuda", piece=piece)
        with torch.no_grad():
            head.weight.copy_(w)
        h.requires_grad_(True)
        torch.cuda.synchronize()
        before = held()
        torch.cuda.reset_peak_memory_stats()
        head(h, y).backward()
        peak = held("peak") - before
        results.append((h.grad.double(), head.weight.grad.double(), peak))
        del head
    (dh, dw, large), (eh, ew, small) = results
    if reduction == "mean":
        assert large > T * V * 6
    # the planes of h and w, dw, the tiles' sums, the coefficients of a piece, and the sums of up to 32
    # parts of dh and 16 of a piece's dw
    assert small < 6 * (T + V) * D + 4 * V * D + 8 * T * (V // 128 + 1) + 6 * T * 2048 + 4 * 32 * T * D + 4 * 16 * 2048 * D + (4 << 20)
    for a, b in ((dh, eh), (dw, ew)):
        assert float((a - b).norm()) < 2e-5 * float(a.norm())
