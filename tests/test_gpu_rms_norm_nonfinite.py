"""NaN in what the 8-bit norm sends (in the weight, in the input, from zero times infinity): the row's scale and
minimum are NaN, as the quantiser's are, so that the receiver reads NaN and no finite value."""

import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


def make(M, D, kind, apart):
    gen = torch.Generator().manual_seed(M + D)
    base = torch.randn(M, D + apart, generator=gen).to(kind).cuda()
    return base[:, apart:], (1.0 + 0.3 * torch.randn(D, generator=gen)).to(kind).cuda()


def send(mpc, x, w, residual=None):
    codes, scale, minv, _, rstd = mpc.mpc_rms_norm_quant(x, w, 1e-6, residual=residual)
    u = (x.float() if residual is None else x.float() + residual.float()) * w.float()
    want, scale0, min0 = mpc.mpc_quant_compress(u.contiguous(), 8)
    for got, ref in ((scale, scale0 * rstd), (minv, min0 * rstd)):
        assert torch.equal(got.isnan(), u.isnan().any(1) | ref.isnan())
        fine = ~got.isnan()
        assert torch.equal(got[fine], ref[fine])
    clean = ~u.isnan().any(1)
    assert torch.equal(codes[clean], want[clean])
    return mpc.mpc_quant_decompress(codes, scale, minv, x.shape[1], 8), clean


# rows of a few threads, a warp, several warps and a CTA, rows read entry by entry (apart, odd widths), long rows
FORMS = [(5, 16, 0), (5, 96, 0), (9, 300, 1), (6, 768, 0), (7, 1601, 0), (4, 4096, 0), (4, 4096, 3), (3, 9000, 0), (2, 16384, 0),
         (3, 17000, 0), (3, 20001, 0)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,apart", FORMS)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("where", ["first", "last", "all"])
def test_nan_in_the_weight(mpc, M, D, apart, sign, where, kind):
    x, w = make(M, D, forms.KINDS[kind], apart)
    at = {"first": slice(0, 1), "last": slice(D - 1, D), "all": slice(0, D)}[where]
    w[at] = torch.tensor(NAN).copysign(torch.tensor(sign)).to(w.dtype)
    y, _ = send(mpc, x, w)
    assert y.isnan().all()
    plain, _, _ = mpc.mpc_rms_norm_forward(x, w, 1e-6)
    assert plain[:, at].isnan().all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,apart", FORMS)
def test_zero_times_infinity(mpc, M, D, apart, kind):
    """Rows whose entry is zero where the weight is infinite are NaN; in the others the product is infinite, and the row
    has the quantiser's scale for that, 0."""
    x, w = make(M, D, forms.KINDS[kind], apart)
    w[D // 2] = INF
    x[: M // 2, D // 2] = 0.0
    y, clean = send(mpc, x, w)
    assert torch.equal(clean, torch.arange(M, device="cuda") >= M // 2)
    assert y[~clean].isnan().all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,D,apart", FORMS)
def test_nan_in_one_row(mpc, M, D, apart, residual, kind):
    """It reaches that row and no other; infinities of opposite sign that a residual adds to x are NaN too."""
    x, w = make(M, D, forms.KINDS[kind], apart)
    r = torch.zeros_like(x) if residual else None
    before, _ = send(mpc, x, w, r)
    if residual:
        x[1, D // 3], r[1, D // 3] = INF, -INF
    else:
        x[1, D // 3] = NAN
    y, clean = send(mpc, x, w, r)
    others = torch.arange(M, device="cuda") != 1
    assert torch.equal(clean, others)
    assert y[1].isnan().all() and torch.equal(y[others], before[others])
