"""The root-mean-square norm with the residual's addition, its 8-bit form and its gradient, against the plain
form in 64 bits."""

import pytest
import torch

import layer_forms as forms
from layer_forms import F32

pytestmark = pytest.mark.gpu
EPS = 1e-5
# fp32 steps of a row's sum: 16 entries a thread and 10 levels; rows over 16384 have 1 in 1024 entries a thread
STEPS = lambda D: 48 + D // 1024  # noqa: E731


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


def make(seed, M, D, kind, residual=True):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = rnd(M, D) * torch.exp(rnd(M, 1))
    x[:, D // 3] *= 20.0
    w = 1.0 + 0.3 * rnd(D)
    return [t.to(kind).cuda() for t in (x, w)] + [rnd(M, D).to(kind).cuda() if residual else None, rnd(M, D).to(kind).cuda(),
                                                  rnd(M, D).to(kind).cuda() if residual else None]


def plain(x, w, r, eps=EPS):
    h = x.double() if r is None else x.double() + r.double()
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h * rstd * w.double(), h, rstd


def check(mpc, x, w, r, dy, dh):
    kind, D = x.dtype, x.shape[1]
    u, steps = forms.half(kind), STEPS(x.shape[1])
    y, h, rstd = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r)
    yw, hw, sw = plain(x, w, r)
    forms.close(rstd.view(-1, 1), sw, sw * steps * F32, "rstd")
    forms.close(y, yw, yw.abs() * (2 * steps * F32 + u), "y")
    if r is None:
        assert h is x
    else:
        forms.close(h, hw, hw.abs() * (u + 2 * F32), "h")
    dx, dw = mpc.mpc_rms_norm_backward(dy, h, w, rstd, dh=dh)
    n, g = hw * sw, dy.double() * w.double()
    c = (g * n).mean(1, keepdim=True)
    base = sw * (g - n * c)
    want = base if dh is None else base + dh.double()
    off = u if r is not None and kind == torch.bfloat16 else 0.0  # of n, where h was rounded
    rough = (g * n).abs().mean(1, keepdim=True)
    e = sw * (g.abs() * 8 * F32 + n.abs() * rough * (2 * off + off * off + 3 * steps * F32)) + 4 * F32 * (base.abs() + want.abs())
    forms.close(dx, want, e + u * (want.abs() + e), "dx")
    terms = (dy.double() * n).abs().sum(0)
    want = (dy.double() * n).sum(0)
    e = terms * (off + (x.shape[0] + steps) * F32)
    forms.close(dw, want, e + u * (want.abs() + e), "dw")
    assert mpc.mpc_get_status() == 0
    return y, h, rstd, dx, dw


SIZES = [(1, 1), (1, 8), (1, 4096), (2, 7), (3, 129), (5, 128), (9, 500), (33, 512), (70, 768), (130, 1000), (257, 1024),
         (64, 1601), (40, 2048), (700, 64), (31, 3001), (20, 4096), (9, 5120), (7, 8192), (5, 9999), (6, 16384), (3, 16385),
         (4, 20000), (400, 17000)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,D", SIZES)
def test_sizes(mpc, M, D, residual, kind):
    check(mpc, *make(M + D, M, D, forms.KINDS[kind], residual))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,D", SIZES)
def test_codes(mpc, M, D, residual, kind):
    """The codes of the quantiser for h w, bit for bit (its rounding decides), scale and minimum times rstd."""
    x, w, r, _, _ = make(M * 3 + D, M, D, forms.KINDS[kind], residual)
    u = (x.float() if r is None else x.float() + r.float()) * w.float()
    want, scale0, min0 = mpc.mpc_quant_compress(u.contiguous(), 8)
    codes, scale, minv, h, rstd = mpc.mpc_rms_norm_quant(x, w, EPS, residual=r)
    assert torch.equal(codes, want)
    assert torch.equal(scale, scale0 * rstd) and torch.equal(minv, min0 * rstd)
    _, h1, rstd1 = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r)
    assert torch.equal(h, h1) and torch.equal(rstd, rstd1)
    # what is read back: within half a step of the norm
    y = mpc.mpc_quant_decompress(codes, scale, minv, D, 8)
    yw = plain(x, w, r)[0]
    span = yw.amax(1, keepdim=True) - yw.amin(1, keepdim=True)
    forms.close(y, yw, 0.5 * span / 255.0 + (span + yw.abs()) * (3 * STEPS(D) * F32), "read back")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_of_one_value(mpc, kind):
    """No range: codes 0 and scale 0, as the quantiser's; a row of zeros has rstd = eps^-1/2."""
    x = torch.zeros(5, 96, dtype=forms.KINDS[kind], device="cuda")
    x[1] = 3.0
    x[2, 7] = 1.0
    w = torch.ones(96, dtype=x.dtype, device="cuda")
    codes, scale, minv, _, rstd = mpc.mpc_rms_norm_quant(x, w, EPS)
    assert not codes[[0, 1, 3, 4]].any() and not scale[[0, 1, 3, 4]].any()
    assert torch.allclose(minv[1].double(), torch.tensor(3.0 / (9.0 + EPS) ** 0.5, dtype=torch.float64, device="cuda"), rtol=4e-7)
    assert torch.allclose(rstd[0].double(), torch.tensor(EPS ** -0.5, dtype=torch.float64, device="cuda"), rtol=4e-7)
    y, _, _ = mpc.mpc_rms_norm_forward(x, w, EPS)
    assert not y[0].any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("off", [1, 4, 8])
@pytest.mark.parametrize("D", [96, 1000, 17000])
def test_strides_and_alignment(mpc, D, off, kind):
    M = 6
    x, w, r, dy, dh = make(5, M, D, forms.KINDS[kind])

    def apart(t, fill=False):
        wide = torch.full((t.shape[0] + 1, t.shape[1] + off + 5), 7.0, dtype=t.dtype, device="cuda")
        view = wide[:-1, off:off + t.shape[1]]
        if fill:
            view.copy_(t)
        return wide, view

    want = check(mpc, x, w, r, dy, dh)
    xs, rs, dys, dhs = (apart(t, True)[1] for t in (x, r, dy, dh))
    (yw, y), (hw, h), (dw, dx) = (apart(x) for _ in range(3))
    _, _, rstd = mpc.mpc_rms_norm_forward(xs, w, EPS, residual=rs, y=y, h=h)
    _, dweight = mpc.mpc_rms_norm_backward(dys, h, w, rstd, dh=dhs, dx=dx)
    for got, ref, wide in ((y, want[0], yw), (h, want[1], hw), (dx, want[3], dw)):
        assert (got.float() - ref.float()).abs().max() <= 2 * forms.half(x.dtype) * ref.float().abs().max()
        wide[:-1, off:off + D] = 7.0
        assert (wide == 7.0).all(), "written outside its rows"
    codes, *_ = mpc.mpc_rms_norm_quant(xs, w, EPS, residual=rs)
    assert torch.equal(codes, mpc.mpc_rms_norm_quant(x, w, EPS, residual=r)[0])


@pytest.mark.parametrize("D", [96, 5000, 17000])
def test_in_place(mpc, D):
    x, w, r, dy, dh = make(6, 9, D, torch.bfloat16)
    y0, h0, rstd0 = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r)
    dx0, dw0 = mpc.mpc_rms_norm_backward(dy, h0, w, rstd0, dh=dh)
    y, h, _ = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r, y=x, h=r)
    assert torch.equal(y, y0) and torch.equal(h, h0) and y is x and h is r
    dx, dw = mpc.mpc_rms_norm_backward(dy, h0, w, rstd0, dh=dh, dx=dh)
    assert dx is dh and torch.equal(dx, dx0) and torch.equal(dw, dw0)


def test_nan_and_infinity_stay_in_their_rows(mpc):
    x, w, r, dy, dh = make(7, 40, 300, torch.float32)
    clean, _, _ = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r)
    x[3, 5], x[17, 0] = float("nan"), float("inf")
    y, _, rstd = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r)
    others = [i for i in range(40) if i not in (3, 17)]
    assert torch.equal(y[others], clean[others])
    assert y[3].isnan().all() and rstd[3].isnan() and rstd[17] == 0 and y[17, 0].isnan()
    *_, rstd = mpc.mpc_rms_norm_quant(x, w, EPS, residual=r)
    assert rstd[3].isnan()


def test_no_rows(mpc):
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    y, h, rstd = mpc.mpc_rms_norm_forward(x, w)
    dx, dw = mpc.mpc_rms_norm_backward(y, h, w, rstd)
    assert dx.shape == (0, 64) and not dw.any()
    assert mpc.mpc_rms_norm_quant(x, w)[0].shape == (0, 16)


@pytest.mark.parametrize("M,D", [(1000, 768), (65, 17000)])
def test_repeats_and_capture(mpc, M, D):
    x, w, r, dy, dh = make(8, M, D, torch.bfloat16)
    first = check(mpc, x, w, r, dy, dh)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y, h, rstd = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r)
        dx, dw = mpc.mpc_rms_norm_backward(dy, h, w, rstd, dh=dh)
    for _ in range(2):
        for t in (y, h, dx, dw):
            t.zero_()
        graph.replay()
        for a, c in zip(first, (y, h, rstd, dx, dw)):
            assert torch.equal(a, c)


def test_differences(mpc):
    """dx and dw against central differences of the plain form (a step of 1e-4 leaves 1e-7)."""
    x, w, r, dy, dh = make(9, 23, 210, torch.float32)
    _, h, rstd = mpc.mpc_rms_norm_forward(x, w, EPS, residual=r)
    grads = mpc.mpc_rms_norm_backward(dy, h, w, rstd, dh=dh)
    gen = torch.Generator("cuda").manual_seed(1)
    for i, grad in enumerate(grads):
        base = [x.double(), w.double()]
        v = torch.randn(base[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        loss = []
        for sign in (1.0, -1.0):
            moved = list(base)
            moved[i] = base[i] + sign * 1e-4 * v
            yw, hw, _ = plain(*moved, r)
            loss.append((yw * dy.double()).sum() + (hw * dh.double()).sum())
        want = (loss[0] - loss[1]) / 2e-4
        got = (grad.double() * v).sum()
        assert (got - want).abs() <= 1e-5 * (grad.double().abs() * v.abs()).sum()
