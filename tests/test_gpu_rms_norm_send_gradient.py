"""The gradient of the 8-bit norm of bf16 rows: its output is fp32, so its gradient arrives in fp32, and is not
rounded before the norm's gradient is formed from it."""

import pytest
import torch

import layer_forms as forms
from layer_forms import F32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,D", [(1, 64), (40, 96), (300, 777), (6, 17000)])
def test_one_rounding_at_the_end(mpc, M, D, residual):
    """dx within half a step of the formula for the h that is kept, and dweight within half a step and the sums' own
    fp32 steps, as for an fp32 norm."""
    gen = torch.Generator().manual_seed(M + D)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x, r = (rnd(M, D).bfloat16().cuda().requires_grad_(True) for _ in range(2))
    w = (1.0 + 0.3 * rnd(D)).bfloat16().cuda().requires_grad_(True)
    dy, dh = rnd(M, D).cuda(), rnd(M, D).bfloat16().cuda()
    eps = 1e-5
    if residual:
        y, h = mpc.rms_norm(x, w, eps, residual=r, bits=8)
        dx, dr, dw = torch.autograd.grad((y, h), (x, r, w), (dy, dh))
        assert torch.equal(dx, dr)
        total = x.detach().double() + r.detach().double()
        h = h.detach().double()
    else:
        y = mpc.rms_norm(x, w, eps, bits=8)
        dx, dw = torch.autograd.grad(y, (x, w), dy)
        h = total = x.detach().double()
    assert y.dtype == torch.float32 and dx.dtype == dw.dtype == torch.bfloat16
    rstd = 1.0 / torch.sqrt((total * total).mean(1, keepdim=True) + eps)
    n, g = h * rstd, dy.double() * w.detach().double()
    base = rstd * (g - n * (g * n).mean(1, keepdim=True))
    want = base + dh.double() if residual else base
    steps, u = 48 + D // 1024, forms.half(torch.bfloat16)
    rough = (g * n).abs().mean(1, keepdim=True)
    e = rstd * (g.abs() * (8 + steps) * F32 + n.abs() * rough * 3 * steps * F32) + 4 * F32 * (base.abs() + want.abs())
    forms.close(dx, want, e + u * (want.abs() + e), "dx")
    want = (dy.double() * n).sum(0)
    e = (dy.double() * n).abs().sum(0) * (M + 2 * steps) * F32
    forms.close(dw, want, e + u * (want.abs() + e), "dw")
    assert mpc.mpc_get_status() == 0
