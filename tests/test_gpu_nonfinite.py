"""NaN and infinity in w, in tokens that count and in gradients: they show in the results that the
formulas give them to, whichever form a call takes, and nowhere else."""

import pytest
import torch

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    torch.cuda.set_device(0)
    return m


def inputs(T, D, V, dtype, ignored=0.2):
    gen = torch.Generator(device="cuda").manual_seed(T + 7 * D + 13 * V)
    dev = {"device": "cuda", "generator": gen}
    w, h = torch.randn(V, D, **dev) / D ** 0.5, torch.randn(T, D, **dev)
    y = torch.randint(0, V, (T,), **dev)
    y[torch.randperm(T, **dev)[: int(ignored * T)]] = -100
    return h.to(dtype), w.to(dtype), y


TYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


@TYPES
@pytest.mark.parametrize("T", [40, 100, 600])
@pytest.mark.parametrize("V,first,last", [(129, 128, 129), (4225, 4224, 4225), (600, 128, 256), (600, 512, 600),
                                          (5000, 0, 1), (5000, 4096, 5000)])
def test_nan_in_w_reaches_every_loss(mpc, dtype, T, V, first, last):
    """Rows of w that are NaN, alone in the last columns of a tile, all of a half tile's, and among others:
    every token that counts has a NaN logit, so its loss and lse are NaN.  Tokens that do not count stay 0."""
    h, w, y = inputs(T, 72, V, dtype)
    w[first:last] = NAN
    counts = y != -100
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    train = mpc.mpc_linear_ce_train(h, w, y)[0]
    for x in (loss, lse, train):
        assert bool(x[counts].isnan().all()) and not x[~counts].any()


@TYPES
@pytest.mark.parametrize("T", [40, 600])
def test_nan_in_one_token(mpc, dtype, T):
    """A token that counts and holds NaN: its own loss and row of dh, and (by its coefficients) dw; the
    other tokens' losses and rows are as without it."""
    h, w, y = inputs(T, 72, 900, dtype, ignored=0.0)
    clean_loss, clean_lse = mpc.mpc_linear_ce_forward(h, w, y)
    clean = mpc.mpc_linear_ce_train(h, w, y)
    h[17, 5] = NAN
    others = torch.arange(T, device="cuda") != 17
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    tloss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    assert bool(loss[17].isnan()) and bool(lse[17].isnan()) and bool(tloss[17].isnan()) and bool(dh[17].isnan().all())
    assert bool(dw.isnan().all())
    assert torch.equal(loss[others], clean_loss[others]) and torch.equal(lse[others], clean_lse[others])
    assert torch.equal(tloss[others], clean[0][others]) and torch.equal(dh[others], clean[1][others])


@TYPES
@pytest.mark.parametrize("T", [1, 2, 4, 8, 16, 32])
@pytest.mark.parametrize("V,row", [(50257, 0), (50257, 25000), (50257, 50256), (40, 3), (129, 128)])
def test_nan_in_w_reaches_every_loss_of_a_few_tokens(mpc, dtype, T, V, row):
    """The same for a few tokens, where a thread goes on to other rows of w after the NaN."""
    h, w, y = inputs(T, 40, V, dtype, ignored=0.0)
    w[row] = NAN
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    train = mpc.mpc_linear_ce_train(h, w, y)[0]
    for x in (loss, lse, train):
        assert bool(x.isnan().all())


@TYPES
@pytest.mark.parametrize("T", [1, 16, 100, 600])
def test_target_at_an_infinite_logit(mpc, dtype, T):
    """A target's logit of +inf: lse is +inf and the loss, inf - inf, NaN, in the forward call as in training.
    Of -inf: lse is that of the others and the loss +inf.  (An fp32 infinity of many tokens is NaN in the
    planes of the matrix products: not finite either.)"""
    h, w, y = inputs(T, 40, 700, dtype, ignored=0.0)
    h[:, 0] = 1.0
    y[:] = torch.arange(T, device="cuda") % 600
    w[:, 0] = 0.0
    others = w.clone()
    at = int(y[T // 2])
    mine = y == at
    for value in (INF, -INF):
        w[at, 0] = value
        loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
        train = mpc.mpc_linear_ce_train(h, w, y)[0]
        logits = h.double() @ others.double().t()
        logits[:, at] = value
        want = torch.logsumexp(logits, 1)
        if dtype == torch.float32 and T > 32:
            assert not bool(loss[mine].isfinite().any() | train[mine].isfinite().any() | lse[mine].isfinite().any())
        elif value == INF:
            assert bool(loss[mine].isnan().all()) and bool(train[mine].isnan().all())
            assert bool((lse[mine] == INF).all())
            assert not bool(loss.isfinite().any() | train.isfinite().any() | lse.isfinite().any())
        else:
            assert bool((loss[mine] == INF).all()) and bool((train[mine] == INF).all())
            # products of 40 terms in fp32 and an exponentials' sum: as for finite logits, 2^-18 of 1 + |lse|
            assert bool(((lse.double() - want).abs() <= 2.0 ** -18 * (1 + want.abs())).all())


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,first,last", [(300, 5, 6), (2048, 256, 512), (5000, 4999, 5000), (255, 0, 255)])
@pytest.mark.parametrize("bad", [NAN, INF], ids=["nan", "inf"])
def test_a_bad_gradient_shows_in_8_bit_states(mpc, gtype, n, first, last, bad):
    """A gradient that is not finite, without a norm that would leave the step out: as with fp32 states, m and
    v of its entries are not finite afterwards, nor after a further step with good gradients; a code has no
    value for that, so it is its block of 256 that shows it.  Other blocks are as without it."""
    def steps(value):
        g = torch.full((n,), 1e-3, device="cuda", dtype=gtype)
        g[first:last] = value
        p = torch.zeros(n, device="cuda")
        plan = mpc.AdamWPlan([p], [g], state_bits=8)
        seen = []
        for k in (1, 2):
            mpc.mpc_adamw_step(plan, 1e-3, 0.9, 0.95, 1e-8, k)
            m, v = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            mpc.mpc_adamw_decode(plan, [m], [v])
            seen.append((m, v))
            g.fill_(1e-3)
        return p, seen

    (p, seen), (clean_p, clean) = steps(bad), steps(1e-3)
    hit = torch.zeros(n, dtype=torch.bool, device="cuda")
    hit[first // 256 * 256:-(-last // 256) * 256] = True
    for (m, v), (clean_m, clean_v) in zip(seen, clean):
        for x, c in ((m, clean_m), (v, clean_v)):
            assert not bool(x[first:last].isfinite().any())
            assert torch.equal(x[~hit], c[~hit])
    assert not bool(p[first:last].isfinite().any()) and torch.equal(p[~hit], clean_p[~hit])
