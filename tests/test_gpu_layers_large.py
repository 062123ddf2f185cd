"""The stage's layers on tensors of more than 2^31 entries: rows from both ends, and sums over all rows."""

import pytest
import torch

import layer_forms as forms
from layer_forms import F32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    yield m
    torch.cuda.empty_cache()


def rnd(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


def ends(M):
    return torch.cat([torch.arange(40), torch.arange(M // 2, M // 2 + 40), torch.arange(M - 40, M)]).cuda()


def test_linear(mpc):
    M, K, N, p, seed = (1 << 21) + 37, 16, 1032, 0.25, 7
    x, w, b, dy = rnd(M, K), rnd(N, K, seed=1) / 4, rnd(N, seed=2), rnd(M, N, seed=3)
    y, z = mpc.mpc_linear_forward(x, w, b, dy, act="silu", p=p, seed=seed, keep=True)
    dx, _, _ = mpc.mpc_linear_backward(dy, x, w, z, act="silu", p=p, seed=seed)
    assert mpc.mpc_get_status() == 0
    at = ends(M)
    # the masks of those rows: N is a multiple of four, so a row starts a draw
    draws = torch.stack([forms.kept((seed + int(i) * (N // 4) * 0x9E3779B97F4A7C15) % 2 ** 64, N, p) for i in at]).cuda()
    xs, dys = x[at], dy[at]
    want, zw = forms.linear(xs, w, b, dys, "silu", draws)
    forms.close(y[at], want, forms.linear_bound(xs, w, b, dys, "silu", draws, want, x.dtype), "y")
    forms.close(z[at], zw, forms.linear_bound(xs, w, b, None, None, None, zw, x.dtype), "z")
    grads = forms.linear_grads(dys, xs, w, zw, "silu", draws)
    z_off = (K + 16) * F32 * (xs.double().abs() @ w.double().abs().t() + b.double().abs())
    bound = forms.linear_grad_bounds(dys, xs, w, zw, grads[3], *grads[:3], "silu", draws, x.dtype, z_off)[0]
    forms.close(dx[at], grads[0], bound, "dx")
    # sums over all rows from the z that was kept, without dropout
    _, dw, db = mpc.mpc_linear_backward(dy, x, w, z, act="silu", need=(False, True, True))
    want_w, want_b, terms_w, terms_b, off_w, off_b = (0.0,) * 6
    for i in range(0, M, 1 << 17):
        rows = slice(i, min(M, i + (1 << 17)))
        zs, d, xd = z[rows].double(), dy[rows].double(), x[rows].double()
        s = torch.sigmoid(zs)
        g = d * s * (1.0 + zs * (1.0 - s))
        slope = d.abs() * (16 * F32 * (1.0 + zs.abs()) + 1e-6)  # what a term is off by
        off = g.abs() + slope
        want_w, terms_w = want_w + g.t() @ xd, terms_w + off.t() @ xd.abs()
        want_b, terms_b = want_b + g.sum(0), terms_b + off.sum(0)
        off_w, off_b = off_w + slope.t() @ xd.abs(), off_b + slope.sum(0)
    u = forms.half(torch.bfloat16)
    # dz is rounded for dw; a chain of fp32 sums is as long as the matrix units' chunks of 8192 rows and their number
    chain = (8192 // 16 + M // 8192 + 16) * 2 * F32
    e = off_w + terms_w * (u + chain)
    forms.close(dw, want_w, e + u * (want_w.abs() + e), "dw")
    # db: 16 rows a thread, 8 threads, then 16384 parts by 8 threads
    e = off_b + terms_b * (16 + 8 + M // 128 // 8 + 8 + 16) * F32
    forms.close(db, want_b, e + u * (want_b.abs() + e), "db")


@pytest.mark.parametrize("D", [4104, 4099])
def test_norm(mpc, D):
    M, eps = (1 << 19) + 11, 1e-5
    x, r, w = rnd(M, D), rnd(M, D, seed=1), 1.0 + rnd(D, seed=2) / 4
    y, h, rstd = mpc.mpc_rms_norm_forward(x, w, eps, residual=r)
    at = ends(M)
    total = x[at].double() + r[at].double()
    s = 1.0 / torch.sqrt((total * total).mean(1, keepdim=True) + eps)
    u, steps = forms.half(torch.bfloat16), 48
    want = total * s * w.double()
    forms.close(y[at], want, want.abs() * (2 * steps * F32 + u), "y")
    forms.close(h[at], total, total.abs() * (u + 2 * F32), "h")
    codes, scale, minv, *_ = mpc.mpc_rms_norm_quant(x, w, eps, residual=r)
    few = mpc.mpc_rms_norm_quant(x[at], w, eps, residual=r[at])
    for a, c in zip((codes, scale, minv), few):
        assert torch.equal(a[at], c)
    del codes, y
    dx, _ = mpc.mpc_rms_norm_backward(r, h, w, rstd, dh=x, need_weight=False)
    few, _ = mpc.mpc_rms_norm_backward(r[at], h[at], w, rstd[at], dh=x[at], need_weight=False)
    assert torch.equal(dx[at], few)
    assert mpc.mpc_get_status() == 0
