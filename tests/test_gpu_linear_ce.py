"""Linear cross entropy on the GPU against the formulas in 64 bits.

Tolerances, from the arithmetic (u = 2^-24 is fp32's rounding unit).  A product summed over K terms
in fp32, in steps of 16 that may truncate, is off by at most S(K) = (K/16 + 6 sqrt(K)) 2u times the
sum of its terms' magnitudes (a truncation a step, plus a random walk with a factor of 6).  A logit
is so off by delta = S(D) max_tv sum_d |h||w|, the loss by twice that and by the rounding of the
exponentials' sum and logarithm (2^-18 of 1 + |lse|).  A coefficient is off by exp(2 delta + 2^-18) - 1
of its probability part, and by r of itself where it is rounded for the matrix product (r = 2^-8 in
bf16, which leaves room for two roundings; 2^-20 in fp32); dh and dw add S(K) over their own sums and
the rounding of the result (2^-8 in bf16, 2^-22 in fp32, of its magnitude).
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U2 = 2.0 ** -23


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    torch.cuda.set_device(0)
    return m


def S(K):
    return (K / 16 + 6 * math.sqrt(K)) * U2


def inputs(T, D, V, dtype, seed=0, scale=1.0, ignored=0.2):
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + T + 7 * D + 13 * V)
    dev = {"device": "cuda", "generator": gen}
    w = torch.randn(V, D, **dev) / math.sqrt(D)
    y = torch.randint(0, V, (T,), **dev)
    h = torch.randn(T, D, **dev) * scale + 4.0 * w[y]
    n = int(ignored * T)
    gone = torch.randperm(T, **dev)[:n]
    y[gone] = -100
    h[gone] = float("nan")
    return h.to(dtype), w.to(dtype), y


def oracle(h, w, y, gloss=None, ignore=-100):
    """loss, lse, dh, dw and their tolerances, in 64 bits."""
    bf = h.dtype == torch.bfloat16
    T, D = h.shape
    V = w.shape[0]
    rows = (y != ignore).nonzero()[:, 0]
    hd, wd, yd = h[rows].double(), w.double(), y[rows]
    n = len(rows)
    l = hd @ wd.t()
    top = l.max(1, keepdim=True).values if n else l[:, :1]
    e = (l - top).exp()
    lse = (top[:, 0] + e.sum(1).log())
    loss = lse - l[torch.arange(n, device=l.device), yd]
    delta = S(D) * float((hd.abs() @ wd.abs().t()).max()) if n else 0.0
    g = torch.full((n,), 1.0 / max(n, 1), dtype=torch.float64, device=h.device) if gloss is None else gloss[rows].double()
    p = (l - lse[:, None]).exp()
    c = p.clone()
    c[torch.arange(n, device=l.device), yd] -= 1.0
    c *= g[:, None]
    r, out = (2.0 ** -8, 2.0 ** -8) if bf else (2.0 ** -20, 2.0 ** -22)
    ec = g.abs()[:, None] * p * math.expm1(2 * delta + 2.0 ** -18) + c.abs() * r
    dh, dw = c @ wd, c.t() @ hd
    edh = ec @ wd.abs() + S(V) * (c.abs() @ wd.abs()) + out * dh.abs() + 1e-30
    edw = ec.t() @ hd.abs() + S(max(n, 1)) * (c.abs().t() @ hd.abs()) + out * dw.abs() + 1e-30

    def whole(x):
        o = torch.zeros((T,) + x.shape[1:], dtype=torch.float64, device=h.device)
        o[rows] = x
        return o

    eloss = 2 * delta + 2.0 ** -18 * (1 + lse.abs())
    return {"loss": (whole(loss), whole(eloss)), "lse": (whole(lse), whole(eloss)),
            "dh": (whole(dh), whole(edh)), "dw": (dw, edw)}


def near(got, want, what):
    x, tol = want
    d = (got.double() - x).abs()
    bad = ~(d <= tol)
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d off, first at %s: got %r want %r tolerance %r" % (
            what, int(bad.sum()), bad.numel(), i, float(got[i]), float(x[i]), float(tol[i])))


SHAPES = [(1, 1, 1), (1, 8, 2), (1, 768, 5000), (2, 17, 5), (7, 64, 64), (64, 64, 300), (65, 63, 257), (127, 200, 129),
          (128, 128, 256), (129, 203, 5003), (200, 72, 1000), (257, 768, 3001), (513, 320, 777), (1000, 40, 513)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D,V", SHAPES)
def test_against_64_bits(mpc, T, D, V, dtype):
    h, w, y = inputs(T, D, V, dtype)
    if T > 1 and int((y != -100).sum()) == 0:
        y[0] = 0
    want = oracle(h, w, y)
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    near(loss, want["loss"], "loss")
    near(lse, want["lse"], "lse")
    dh, dw = mpc.mpc_linear_ce_backward(h, w, y, lse)
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")
    loss2, dh2, dw2 = mpc.mpc_linear_ce_train(h, w, y)
    near(loss2, want["loss"], "loss (train)")
    near(dh2, want["dh"], "dh (train)")
    near(dw2, want["dw"], "dw (train)")
    assert mpc.mpc_get_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("piece", [1, 64, 100, 256, 700, 5000])
def test_weights_and_pieces(mpc, dtype, piece):
    if piece == 1:
        T, D, V = 40, 24, 11
    else:
        T, D, V = 300, 96, 1500
    h, w, y = inputs(T, D, V, dtype, seed=3)
    gloss = torch.randn(T, device="cuda")
    want = oracle(h, w, y, gloss)
    _, lse = mpc.mpc_linear_ce_forward(h, w, y)
    for dh, dw in (mpc.mpc_linear_ce_backward(h, w, y, lse, gloss, piece=piece),
                   mpc.mpc_linear_ce_train(h, w, y, gloss, piece=piece)[1:]):
        near(dh, want["dh"], "dh")
        near(dw, want["dw"], "dw")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_no_token_counts(mpc, dtype):
    h, w, y = inputs(70, 40, 300, dtype, ignored=1.0)
    assert int((y != -100).sum()) == 0
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    assert not loss.any() and not lse.any()
    for dh, dw in (mpc.mpc_linear_ce_backward(h, w, y, lse), mpc.mpc_linear_ce_train(h, w, y)[1:]):
        assert not dh.any() and not dw.any()


def test_no_tokens(mpc):
    w = torch.randn(30, 16, device="cuda")
    h = torch.empty(0, 16, device="cuda")
    y = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    assert loss.shape == (0,) and dh.shape == (0, 16) and not dw.any()
    assert mpc.mpc_linear_ce_forward(h, w, y)[0].shape == (0,)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(8, 0), (1, 0), (0, 1), (5, 3)])
def test_strides_and_guards(mpc, dtype, pad, offset):
    """Rows further apart than their length, bases off 16 bytes; what lies between is left alone."""
    T, D, V = 150, 72, 400
    h, w, y = inputs(T, D, V, dtype, seed=5)
    want = oracle(h, w, y)

    def strided(x, fill):
        big = torch.full((x.shape[0] * (D + pad) + offset,), fill, dtype=dtype, device="cuda")
        v = big[offset:].view(x.shape[0], D + pad)[:, :D]
        v.copy_(x)
        return big, v

    (_, hs), (_, wt) = strided(h, float("nan")), strided(w, float("nan"))
    bdh, dh = strided(torch.zeros_like(h), 7.0)
    bdw, dw = strided(torch.zeros_like(w), 7.0)
    loss, dh, dw = mpc.mpc_linear_ce_train(hs, wt, y, dh=dh, dw=dw)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")
    for big, x in ((bdh, dh), (bdw, dw)):
        keep = torch.ones_like(big, dtype=torch.bool)
        keep[offset:].view(-1, D + pad)[:, :D] = False
        assert bool((big[keep] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shift", [-3000.0, 3000.0])
def test_logits_far_from_zero(mpc, dtype, shift):
    """exp of the logits over- or underflows; their differences do not."""
    T, D, V = 130, 64, 700
    h, w, y = inputs(T, D, V, dtype, seed=6)
    h[:, 0], w[:, 0] = shift / 64, 64.0
    h[y == -100] = float("nan")
    want = oracle(h, w, y)
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")


def test_confident_and_hopeless_tokens(mpc):
    """Targets far above and far below every other logit, beyond the range of exp in fp32."""
    T, D, V = 140, 32, 600
    h, w, y = inputs(T, D, V, torch.float32, seed=8, ignored=0.0)
    w = w / w.norm(dim=1, keepdim=True)
    h = w[y] * torch.where(torch.arange(T, device="cuda") % 2 == 0, 400.0, -400.0)[:, None]
    want = oracle(h, w, y)
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")


def test_targets_out_of_range(mpc):
    h, w, y = inputs(50, 32, 100, torch.float32, ignored=0.0)
    y[3], y[7], y[9] = 100, -1, 1 << 40
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    assert mpc.mpc_get_status() == 6
    assert mpc.mpc_get_status() == 0
    masked = y.clone()
    masked[[3, 7, 9]] = -100
    want = oracle(h, w, masked)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")


def test_ignore_index_inside_the_vocabulary(mpc):
    h, w, y = inputs(90, 48, 64, torch.float32, ignored=0.0)
    y[::3] = 5
    want = oracle(h, w, y, ignore=5)
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y, ignore_index=5)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_results_repeat_on_any_stream(mpc, dtype):
    h, w, y = inputs(600, 136, 2500, dtype, seed=9)
    first = mpc.mpc_linear_ce_train(h, w, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = mpc.mpc_linear_ce_train(h, w, y)
    third = mpc.mpc_linear_ce_train(h, w, y, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_captured_in_a_graph(mpc):
    h, w, y = inputs(200, 64, 900, torch.bfloat16, seed=10)
    eager = mpc.mpc_linear_ce_train(h, w, y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = mpc.mpc_linear_ce_train(h, w, y)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager, out):
        assert torch.equal(a, b)


def test_gradient_against_differences(mpc):
    """<gradient, direction> against the central difference of the library's own loss.  The loss is
    off by e (above), the difference by e/step, and its truncation is step^2/6 of the third
    derivative along the direction, at most the cube of the spread of the logits' change."""
    T, D, V = 9, 20, 50
    h, w, y = inputs(T, D, V, torch.float32, seed=11)
    keep = y != -100
    h = torch.where(keep[:, None], h, torch.zeros_like(h))
    gloss = torch.rand(T, device="cuda") + 0.5
    _, dh, dw = mpc.mpc_linear_ce_train(h, w, y, gloss)
    eloss = oracle(h, w, y)["loss"][1]
    step = 2.0 ** -6
    for a in range(4):
        gen = torch.Generator(device="cuda").manual_seed(a)
        uh = torch.randn(T, D, device="cuda", generator=gen) * (a != 1) / math.sqrt(D)
        uw = torch.randn(V, D, device="cuda", generator=gen) * (a != 2) / math.sqrt(D)
        up, down = (mpc.mpc_linear_ce_forward(h + s * uh, w + s * uw, y)[0].double() for s in (step, -step))
        diff = float(((up - down) * gloss.double()).sum() / (2 * step))
        dot = float((dh.double() * uh.double()).sum() + (dw.double() * uw.double()).sum())
        change = (uh.double() @ w.double().t() + h.double() @ uw.double().t())[keep]
        bend = 2 * (uh.double() @ uw.double().t())[keep]
        spread = change.max(1).values - change.min(1).values
        curve = bend.max(1).values - bend.min(1).values
        third = ((spread ** 3 + 3 * spread * curve) * gloss[keep].double()).sum()
        tol = 2 * float((eloss * gloss.double()).sum()) / step + step ** 2 / 6 * float(third) + 1e-5 * abs(dot)
        assert abs(diff - dot) <= tol, (a, diff, dot, tol)


def test_autograd(mpc):
    """The module's three reductions against torch's in 64 bits."""
    T, D, V = 120, 56, 333
    for reduction in ("mean", "sum", "none"):
        head = mpc.LinearCrossEntropy(D, V, reduction=reduction, device="cuda")
        h, _, y = inputs(T, D, V, torch.float32, seed=12)
        h = torch.where((y != -100)[:, None], h, torch.zeros_like(h)).view(4, 30, D).requires_grad_(True)
        y = y.view(4, 30)
        out = head(h, y)
        factor = torch.rand(out.shape, device="cuda") + 0.5
        (out * factor).sum().backward()
        hd = h.detach().double().requires_grad_(True)
        wd = head.weight.detach().double().requires_grad_(True)
        ref = torch.nn.functional.cross_entropy((hd @ wd.t()).view(-1, V), y.view(-1), reduction=reduction)
        ref = ref.view(out.shape)
        (ref * factor.double()).sum().backward()
        assert out.dtype == torch.float32
        for got, want in ((out, ref), (h.grad, hd.grad), (head.weight.grad, wd.grad)):
            err = float((got.detach().double() - want.detach()).norm() / want.detach().norm())
            assert err < 2e-5, (reduction, err)
        with torch.no_grad():
            assert float((head(h, y).double() - ref).norm() / ref.norm()) < 2e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "hopeless", "one row", "same target", "weights"])
def test_exponentials_kept(mpc, dtype, kind):
    """Training that forms the logits once (more tokens than a row tile): ordinary tokens, losses far
    beyond exp's range in some row tiles, one such token alone, runs of one target that span several
    sums, given weights.  In bf16 a term of dw takes two roundings of up to 2^-8 (the exponential's,
    the scaled hidden state's): the tolerance for c gets one more of them."""
    T, D, V = 700, 72, 900
    h, w, y = inputs(T, D, V, dtype, seed=20, ignored=0.1)
    gloss = None
    if kind in ("hopeless", "one row"):
        w = (w.float() / w.float().norm(dim=1, keepdim=True)).to(dtype)
        lot = torch.arange(T, device="cuda") == 650 if kind == "one row" else \
            (torch.arange(T, device="cuda") % 3 == 0) & (torch.arange(T, device="cuda") < 500)
        y[650] = 17
        sign = torch.where(torch.arange(T, device="cuda") % 2 == 0, -400.0, 400.0)[:, None]
        h = torch.where((lot & (y >= 0))[:, None], (w.float()[y.clamp_min(0)] * sign).to(dtype), h)
    elif kind == "same target":
        y[y >= 0] = torch.where(y[y >= 0] % 4 == 0, y[y >= 0], 5)
    elif kind == "weights":
        gloss = torch.randn(T, device="cuda")
    want = oracle(h, w, y, gloss)
    if dtype == torch.bfloat16:
        rows = (y != -100).nonzero()[:, 0]
        hd, wd = h[rows].double(), w.double()
        c = torch.softmax(hd @ wd.t(), 1)
        c[torch.arange(len(rows), device="cuda"), y[rows]] -= 1.0
        c *= (torch.full((len(rows),), 1.0 / len(rows), device="cuda") if gloss is None else gloss[rows]).double()[:, None]
        want["dw"] = (want["dw"][0], want["dw"][1] + 2.0 ** -8 * (c.abs().t() @ hd.abs()))
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y, gloss)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")
    again = mpc.mpc_linear_ce_train(h, w, y, gloss)
    for a, b in zip((loss, dh, dw), again):
        assert torch.equal(a, b)
    assert mpc.mpc_get_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 3, 5, 8, 9, 16, 17])
@pytest.mark.parametrize("D,V", [(64, 1), (8, 40), (7, 9), (768, 3001), (1001, 777), (1032, 2500), (4100, 130)])
def test_few_tokens(mpc, dtype, T, D, V):
    """The form for a few tokens and its first neighbour: widths of whole and of broken 16-byte groups,
    vocabularies shorter than a warp's rows, some tokens ignored, given weights, rows further apart."""
    h, w, y = inputs(T, D, V, dtype, seed=30, ignored=0.3)
    gloss = torch.randn(T, device="cuda")
    want = oracle(h, w, y, gloss)
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    near(loss, want["loss"], "loss")
    near(lse, want["lse"], "lse")
    dh, dw = mpc.mpc_linear_ce_backward(h, w, y, lse, gloss)
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")
    big = torch.full((V, D + 8), float("nan"), dtype=dtype, device="cuda")
    big[:, :D] = w
    dbig = torch.full((V, D + 3), 7.0, dtype=dtype, device="cuda")
    loss, dh, dw = mpc.mpc_linear_ce_train(h, big[:, :D], y, gloss, dw=dbig[:, :D])
    near(loss, want["loss"], "loss (train)")
    near(dh, want["dh"], "dh (train)")
    near(dw, want["dw"], "dw (train)")
    assert bool((dbig[:, D:] == 7.0).all())
    assert mpc.mpc_get_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [8, 9, 16, 20, 31, 32, 33])
@pytest.mark.parametrize("D,V,off", [(768, 22000, 0), (771, 22000, 0), (768, 22000, 1), (7000, 2500, 0)])
def test_few_tokens_of_a_large_head(mpc, dtype, T, D, V, off):
    """Where the two forms meet over a head of more than 2^24 entries: rows on and off 16 bytes, a base
    off 16 bytes, rows whose h takes several passes; each direction by itself and together."""
    h, w, y = inputs(T, D, V, dtype, seed=31, ignored=0.2)
    flat = torch.zeros(V * D + 8, dtype=dtype, device="cuda")
    flat[off:off + V * D] = w.reshape(-1)
    placed = flat[off:off + V * D].view(V, D)
    gloss = torch.randn(T, device="cuda")
    want = oracle(h, w, y, gloss)
    loss, lse = mpc.mpc_linear_ce_forward(h, placed, y)
    near(loss, want["loss"], "loss")
    near(lse, want["lse"], "lse")
    dh, dw = mpc.mpc_linear_ce_backward(h, placed, y, lse, gloss)
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")
    loss, dh, dw = mpc.mpc_linear_ce_train(h, placed, y, gloss)
    near(loss, want["loss"], "loss (train)")
    near(dh, want["dh"], "dh (train)")
    near(dw, want["dw"], "dw (train)")
    assert mpc.mpc_get_status() == 0


def test_autograd_of_layouts(mpc):
    """Hidden states that are broadcast, transposed or cut out of something wider; a transposed weight."""
    D, V = 40, 90
    gen = torch.Generator(device="cuda").manual_seed(3)
    y = torch.randint(0, V, (60,), device="cuda", generator=gen)
    one = torch.randn(1, D, device="cuda", generator=gen)
    flat = torch.randn(D, 60, device="cuda", generator=gen)
    wide = torch.randn(60, D + 9, device="cuda", generator=gen)
    wt = torch.randn(D, V, device="cuda", generator=gen)
    for base, view in ((one, lambda t: t.expand(60, D)), (flat, lambda t: t.t()), (wide, lambda t: t[:, 5:5 + D])):
        a, b = base.clone().requires_grad_(True), base.double().requires_grad_(True)
        u, v = wt.clone().requires_grad_(True), wt.double().requires_grad_(True)
        loss = mpc.linear_cross_entropy(view(a), u.t(), y)
        ref = torch.nn.functional.cross_entropy(view(b) @ v, y)
        loss.backward()
        ref.backward()
        assert abs(float(loss.detach()) - float(ref.detach())) < 2e-5 * abs(float(ref.detach()))
        for got, want in ((a.grad, b.grad), (u.grad, v.grad)):
            assert got.shape == want.shape
            assert float((got.double() - want).norm()) < 2e-5 * float(want.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [100, 600])
def test_a_wait_that_gives_up_is_reported(mpc, dtype, T):
    """With the limit of device-side waits at 0 every first wait gives up: the products' kernels return,
    the status says so, and the next call is as before."""
    h, w, y = inputs(T, 96, 1000, dtype, seed=40)
    before = mpc.mpc_linear_ce_train(h, w, y)
    assert mpc.mpc_get_status() == 0
    mpc.mpc_set_knob(mpc.MPC_KNOB_SPIN_LIMIT, 0)
    try:
        mpc.mpc_linear_ce_train(h, w, y)
        assert mpc.mpc_get_status() == 5
    finally:
        mpc.mpc_set_knob(mpc.MPC_KNOB_SPIN_LIMIT, 1 << 20)
    assert mpc.mpc_get_status() == 0
    for a, b in zip(before, mpc.mpc_linear_ce_train(h, w, y)):
        assert torch.equal(a, b)


def test_plain_stream_order_gives_the_same(mpc):
    """Launches with and without programmatic dependent launch."""
    h, w, y = inputs(700, 136, 1300, torch.bfloat16, seed=41)
    with_pdl = [x.clone() for x in mpc.mpc_linear_ce_train(h, w, y)]
    mpc.mpc_set_knob(mpc.MPC_KNOB_PDL, 0)
    try:
        without = mpc.mpc_linear_ce_train(h, w, y)
    finally:
        mpc.mpc_set_knob(mpc.MPC_KNOB_PDL, 1)
    for a, b in zip(with_pdl, without):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_no_token_of_many_counts(mpc, dtype):
    h, w, y = inputs(600, 40, 300, dtype, ignored=1.0)
    for dh, dw in (mpc.mpc_linear_ce_backward(h, w, y, torch.zeros(600, device="cuda")),
                   mpc.mpc_linear_ce_train(h, w, y)[1:]):
        assert not dh.any() and not dw.any()
    loss, lse = mpc.mpc_linear_ce_forward(h, w, y)
    assert not loss.any() and not lse.any()
    assert mpc.mpc_get_status() == 0


def test_one_token_of_many_counts(mpc):
    h, w, y = inputs(600, 40, 300, torch.float32, seed=50, ignored=1.0)
    y[431] = 7
    h[431] = w[7] * 2
    want = oracle(h, w, y)
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_more_tokens_than_are_ordered(mpc, dtype):
    """Beyond 16384 tokens a training call forms the logits twice."""
    h, w, y = inputs(16500, 24, 200, dtype, seed=51)
    want = oracle(h, w, y)
    loss, dh, dw = mpc.mpc_linear_ce_train(h, w, y)
    near(loss, want["loss"], "loss")
    near(dh, want["dh"], "dh")
    near(dw, want["dw"], "dw")
