"""The linear layer with bias, activation, dropout and residual, and its gradient, against the plain form in
64 bits."""

import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


def make(seed, M, K, N, kind, bias=True, residual=True):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(kind).cuda()  # noqa: E731
    x, w = rnd(M, K), (torch.randn(N, K, generator=gen) / K ** 0.5).to(kind).cuda()
    return x, w, rnd(N) if bias else None, rnd(M, N) if residual else None, rnd(M, N)


def check(mpc, x, w, b, r, dy, act, p, seed, **calls):
    M, K = x.shape
    N = w.shape[0]
    kind = x.dtype
    mask = forms.kept(seed, M * N, p).view(M, N).cuda() if p else None
    y, z = mpc.mpc_linear_forward(x, w, b, r, act=act, p=p, seed=seed, keep=act is not None, **calls)
    want, zw = forms.linear(x, w, b, r, act, mask)
    forms.close(y, want, forms.linear_bound(x, w, b, r, act, mask, want, kind), "y")
    z_off = (K + 16) * forms.F32 * (x.double().abs() @ w.double().abs().t() + (0.0 if b is None else b.double().abs()))
    if act is not None:
        forms.close(z, zw, z_off + forms.half(kind) * (zw.abs() + z_off), "z")
    dx, dw, db = mpc.mpc_linear_backward(dy, x, w, z, act=act, p=p, seed=seed)
    wants = forms.linear_grads(dy, x, w, zw, act, mask)
    bounds = forms.linear_grad_bounds(dy, x, w, zw, wants[3], *wants[:3], act, mask, kind, z_off)
    for name, got, want, bound in zip(("dx", "dw", "db"), (dx, dw, db), wants, bounds):
        forms.close(got, want, bound, name)
    assert mpc.mpc_get_status() == 0
    return y, z, dx, dw, db


SIZES = [(1, 1, 1), (1, 64, 64), (1, 1024, 4096), (2, 8, 16), (3, 17, 33), (7, 129, 65), (16, 256, 100), (24, 512, 768),
         (31, 65, 1000), (33, 1000, 64), (64, 64, 64), (100, 72, 200), (129, 203, 307), (255, 257, 129), (256, 256, 256),
         (257, 384, 520), (300, 1031, 77), (513, 264, 1025)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_sizes(mpc, M, K, N, kind):
    check(mpc, *make(M + 7 * K + N, M, K, N, forms.KINDS[kind]), act="gelu_tanh", p=0.1, seed=5)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("K,N", [(8, 5), (24, 16), (40, 33), (264, 31), (1000, 12001), (2056, 100), (74, 90), (75, 91)])
@pytest.mark.parametrize("M", [1, 4, 7, 8, 9, 16, 20, 32, 33, 64, 65])
def test_few_rows(mpc, M, K, N, kind):
    x, w, b, r, _ = make(M + K, M, K, N, forms.KINDS[kind])
    for act, p, bias, residual in (("silu", 0.0, b, None), (None, 0.3, None, r)):
        mask = forms.kept(2, M * N, p).view(M, N).cuda() if p else None
        y, z = mpc.mpc_linear_forward(x, w, bias, residual, act=act, p=p, seed=2, keep=True)
        want, zw = forms.linear(x, w, bias, residual, act, mask)
        forms.close(y, want, forms.linear_bound(x, w, bias, residual, act, mask, want, x.dtype), "y")
        forms.close(z, zw, forms.linear_bound(x, w, bias, None, None, None, zw, x.dtype), "z")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act,residual", [(None, True), ("gelu", True), ("silu", False)])
@pytest.mark.parametrize("M,K,N", [(4128, 520, 2056), (3001, 331, 3203), (1030, 2100, 4104), (130, 4500, 96)])
def test_many_tiles(mpc, M, K, N, act, residual, kind):
    """More tiles than the SMs take at once, whole and ragged, and long sums."""
    check(mpc, *make(M, M, K, N, forms.KINDS[kind], True, residual), act=act, p=0.1, seed=5)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(9000, 2064, 2576), (2576, 9000, 2064), (70, 9001, 130)])
def test_sums_of_several_chunks(mpc, M, K, N, kind):
    """More K blocks than one accumulator of the matrix units sums, in whole tiles and in tiles cut along K."""
    check(mpc, *make(M, M, K, N, forms.KINDS[kind]), act="gelu_tanh", p=0.1, seed=7)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("act", [None, "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("bias,residual,p", [(False, False, 0.0), (True, False, 0.0), (False, True, 0.5), (True, True, 0.25)])
@pytest.mark.parametrize("M,K,N", [(5, 40, 72), (150, 136, 200), (131, 99, 143)])
def test_epilogues(mpc, M, K, N, act, bias, residual, p, kind):
    check(mpc, *make(11, M, K, N, forms.KINDS[kind], bias, residual), act=act, p=p, seed=2 ** 63 + 9)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(4, 16, 24), (140, 128, 136)])
def test_relu_of_whole_numbers(mpc, M, K, N, kind):
    """Whole numbers: every z is exact, so its sign and all sums are too."""
    gen = torch.Generator().manual_seed(3)
    x, w, dy = (torch.randint(-3, 4, s, generator=gen).to(forms.KINDS[kind]).cuda() for s in ((M, K), (N, K), (M, N)))
    y, z = mpc.mpc_linear_forward(x, w, act="relu", keep=True)
    dx, dw, db = mpc.mpc_linear_backward(dy, x, w, z, act="relu")
    zw = x.double() @ w.double().t()
    g = dy.double() * (zw > 0)
    for got, want in ((z, zw), (y, zw.clamp_min(0)), (dx, g @ w.double()), (dw, g.t() @ x.double()), (db, g.sum(0))):
        assert torch.equal(got, want.to(got.dtype))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("off", [0, 1, 4, 8])
@pytest.mark.parametrize("M,K,N", [(6, 64, 80), (140, 72, 160)])
def test_strides_and_alignment(mpc, M, K, N, off, kind):
    """Rows apart and bases off 16 bytes, for inputs and outputs; what lies between rows stays."""
    x, w, b, r, dy = make(4, M, K, N, forms.KINDS[kind])

    def apart(t, fill=None):
        wide = torch.full((t.shape[0] + 1, t.shape[1] + 2 * off + 3), 7.0, dtype=t.dtype, device="cuda")
        view = wide[:-1, off:off + t.shape[1]]
        if fill is not None:
            view.copy_(fill)
        return wide, view

    ins = [apart(t, t)[1] for t in (x, w, r, dy)]
    outs = [apart(t) for t in (r, r, x, w)]
    (yw, y), (zw, z), (dxw, dx), (dww, dw) = outs
    bias = torch.cat([b[:1], b])[1:] if off else b
    mpc.mpc_linear_forward(ins[0], ins[1], bias, ins[2], act="silu", p=0.1, seed=8, y=y, z=z)
    mpc.mpc_linear_backward(ins[3], ins[0], ins[1], z, act="silu", p=0.1, seed=8, dx=dx, dw=dw)
    y0, z0, dx0, dw0, _ = check(mpc, x, w, b, r, dy, "silu", 0.1, 8)
    mask = forms.kept(8, M * N, 0.1).view(M, N).cuda()
    want, _ = forms.linear(x, w, b, r, "silu", mask)
    forms.close(y, want, forms.linear_bound(x, w, b, r, "silu", mask, want, x.dtype), "y")
    for (wide, view), like in zip(outs, (y0, z0, dx0, dw0)):
        assert (view.float() - like.float()).abs().max() <= 0.05 * like.float().abs().max()
        wide[:-1, off:off + view.shape[1]] = 7.0
        assert (wide == 7.0).all(), "written outside its rows"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("need", [(True, False, False), (False, True, False), (False, False, True), (True, False, True)])
def test_parts_of_the_gradient(mpc, need, kind):
    x, w, b, _, dy = make(6, 70, 96, 130, forms.KINDS[kind])
    _, z = mpc.mpc_linear_forward(x, w, b, act="gelu", keep=True)
    whole = mpc.mpc_linear_backward(dy, x, w, z, act="gelu")
    part = mpc.mpc_linear_backward(dy, x, w, z, act="gelu", need=need)
    for n, a, c in zip(need, part, whole):
        assert a is None if not n else torch.equal(a, c)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(3, 64, 128), (200, 320, 384)])
def test_repeats(mpc, M, K, N, kind):
    args = make(9, M, K, N, forms.KINDS[kind])
    first = check(mpc, *args, act="gelu", p=0.1, seed=1)
    for _ in range(3):
        for a, c in zip(first, check(mpc, *args, act="gelu", p=0.1, seed=1)):
            assert a is c is None or torch.equal(a, c)


def test_no_rows(mpc):
    x, w = torch.empty(0, 16, device="cuda"), torch.randn(8, 16, device="cuda")
    y, _ = mpc.mpc_linear_forward(x, w)
    assert y.shape == (0, 8)
    dx, dw, db = mpc.mpc_linear_backward(y, x, w)
    assert dx.shape == (0, 16) and not dw.any() and not db.any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M", [3, 150])
def test_residual_in_place(mpc, M, kind):
    x, w, b, r, _ = make(13, M, 96, 128, forms.KINDS[kind])
    want, _ = mpc.mpc_linear_forward(x, w, b, r, act="silu", p=0.2, seed=4)
    got, _ = mpc.mpc_linear_forward(x, w, b, r, act="silu", p=0.2, seed=4, y=r)
    assert got is r and torch.equal(got, want)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M", [2, 300])
def test_nan_stays_in_its_row(mpc, M, kind):
    """A NaN of one row of x reaches that row of y and no other, and none where dropout drops it."""
    x, w, b, r, _ = make(14, M, 80, 144, forms.KINDS[kind])
    x[1, 3] = float("nan")
    y, _ = mpc.mpc_linear_forward(x, w, b, r, act="gelu", p=0.5, seed=6)
    mask = forms.kept(6, M * 144, 0.5).view(M, 144).cuda()
    nan = y.isnan()
    assert torch.equal(nan[1], mask[1] > 0)
    assert not nan[torch.arange(M) != 1].any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_nan_in_dropped_places_of_the_gradient(mpc, kind):
    """NaN of z and dy where dropout drops reaches nothing; elsewhere it reaches its row of dx and its column of db."""
    M, K, N = 40, 64, 72
    x, w, _, _, dy = make(19, M, K, N, forms.KINDS[kind])
    _, z = mpc.mpc_linear_forward(x, w, act="silu", p=0.5, seed=6, keep=True)
    clean = mpc.mpc_linear_backward(dy, x, w, z, act="silu", p=0.5, seed=6)
    gone = forms.kept(6, M * N, 0.5).view(M, N).cuda() == 0
    z[gone], dy[gone] = float("nan"), float("nan")
    for a, c in zip(clean, mpc.mpc_linear_backward(dy, x, w, z, act="silu", p=0.5, seed=6)):
        assert torch.equal(a, c)
    row, col = (~gone).nonzero()[0].tolist()
    z[row, col] = float("nan")
    dx, _, db = mpc.mpc_linear_backward(dy, x, w, z, act="silu", p=0.5, seed=6)
    assert dx[row].isnan().all() and db[col].isnan()
    assert not dx[torch.arange(M) != row].isnan().any() and not db[torch.arange(N) != col].isnan().any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("limit", [1, 2, 20])
def test_waits_of_one_and_a_few_tries(mpc, kind, limit):
    """Whichever wait gives up first, the kernels return with nothing in flight: the status says so, and the calls
    after that are as before."""
    x, w, b, r, dy = make(20, 600, 1160, 1400, forms.KINDS[kind])

    def calls():
        y, z = mpc.mpc_linear_forward(x, w, b, r, act="gelu", p=0.1, seed=2, keep=True)
        return (y, *mpc.mpc_linear_backward(dy, x, w, z, act="gelu", p=0.1, seed=2))

    before = calls()
    assert mpc.mpc_get_status() == 0
    mpc.mpc_set_knob(mpc.MPC_KNOB_SPIN_LIMIT, limit)
    try:
        calls()
        assert mpc.mpc_get_status() in (0, 5)
    finally:
        mpc.mpc_set_knob(mpc.MPC_KNOB_SPIN_LIMIT, 1 << 20)
    assert mpc.mpc_get_status() == 0
    for a, c in zip(before, calls()):
        assert torch.equal(a, c)
    assert mpc.mpc_get_status() == 0


def test_two_streams_at_once(mpc):
    """Calls on two streams, each with a workspace of its own, give what they give one after the other."""
    sets = [make(30 + i, 700, 900, 1100, torch.float32) for i in range(2)]
    want = [mpc.mpc_linear_backward(s[4], s[0], s[1]) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [mpc.mpc_linear_backward(s[4], s[0], s[1], stream=st) for s, st in zip(sets, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, c) for a, c in zip(g, w))


def test_pdl_knob_changes_nothing(mpc):
    args = make(22, 520, 600, 700, torch.bfloat16)
    first = check(mpc, *args, act="silu", p=0.1, seed=1)
    mpc.mpc_set_knob(mpc.MPC_KNOB_PDL, 0)
    try:
        for a, c in zip(first, check(mpc, *args, act="silu", p=0.1, seed=1)):
            assert torch.equal(a, c)
    finally:
        mpc.mpc_set_knob(mpc.MPC_KNOB_PDL, 1)


def test_everything_dropped(mpc):
    x, w, b, r, dy = make(15, 40, 64, 48, torch.float32)
    y, _ = mpc.mpc_linear_forward(x, w, b, r, p=1.0, seed=3)
    assert torch.equal(y, r)
    dx, dw, db = mpc.mpc_linear_backward(dy, x, w, p=1.0, seed=3)
    assert not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M", [4, 270])
def test_captured_with_a_device_step(mpc, M, kind):
    """Replays of a captured call take the mask of the counter's value then, and inputs written between."""
    x, w, b, r, dy = make(16, M, 128, 192, forms.KINDS[kind])
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def call():
        y, z = mpc.mpc_linear_forward(x, w, b, r, act="gelu", p=0.3, seed=77, step=step, keep=True)
        return (y, *mpc.mpc_linear_backward(dy, x, w, z, act="gelu", p=0.3, seed=77, step=step))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for value in (0, 5):
        step.fill_(value)
        x.mul_(-1.0)
        graph.replay()
        y, z = mpc.mpc_linear_forward(x, w, b, r, act="gelu", p=0.3, seed=77 + value, keep=True)
        wants = (y, *mpc.mpc_linear_backward(dy, x, w, z, act="gelu", p=0.3, seed=77 + value))
        for a, c in zip(held, wants):
            assert torch.equal(a, c)


def test_another_stream(mpc):
    """The call runs on the stream it is given, after that stream's earlier work."""
    x, w, b, r, _ = make(17, 300, 512, 512, torch.bfloat16)
    want, _ = mpc.mpc_linear_forward(x, w, b, r)
    side = torch.cuda.Stream()
    late = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late.copy_(x)
    y, _ = mpc.mpc_linear_forward(late, w, b, r, stream=side)
    side.synchronize()
    assert torch.equal(y, want)


def test_differences(mpc):
    """The gradients against central differences of the plain form along random directions (fp32; a step of 1e-4 in
    64 bits leaves 1e-7 of curvature and 1e-10 of rounding)."""
    x, w, b, r, dy = make(18, 37, 45, 53, torch.float32)
    seed, p = 21, 0.2
    mask = forms.kept(seed, 37 * 53, p).view(37, 53).cuda()
    _, z = mpc.mpc_linear_forward(x, w, b, r, act="gelu", p=p, seed=seed, keep=True)
    grads = mpc.mpc_linear_backward(dy, x, w, z, act="gelu", p=p, seed=seed)
    gen = torch.Generator("cuda").manual_seed(1)
    for i, grad in enumerate(grads):
        base = [x.double(), w.double(), b.double()]
        v = torch.randn(base[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        loss = []
        for sign in (1.0, -1.0):
            moved = list(base)
            moved[i] = base[i] + sign * 1e-4 * v
            loss.append((forms.linear(*moved, r, "gelu", mask)[0] * dy.double()).sum())
        want = (loss[0] - loss[1]) / 2e-4
        got = (grad.double() * v).sum()
        scale = (grad.double().abs() * v.abs()).sum()
        assert (got - want).abs() <= 1e-5 * scale
