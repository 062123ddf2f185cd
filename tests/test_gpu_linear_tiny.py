"""fp32 operands near the smallest numbers: the three bf16 terms of an entry keep its bits down to 2^-133, the smallest
bf16 number, so an entry is off by 2^-134 at most (a few rows are read in fp32 as they are)."""

import pytest
import torch

import layer_forms as forms
from layer_forms import F32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


@pytest.mark.parametrize("power", [0, -100, -109, -112, -117, -120, -125, -127, -132])
@pytest.mark.parametrize("M,K,N", [(5, 40, 72), (70, 72, 80), (300, 96, 130)])
@pytest.mark.parametrize("which", ["x", "w"])
def test_small_operands(mpc, M, K, N, power, which):
    gen = torch.Generator().manual_seed(M + K)
    rnd = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    x, w, dy = rnd(M, K), rnd(N, K), rnd(M, N)
    # one operand so small, the other so large that products are of ordinary size
    small, large = (x, w) if which == "x" else (w, x)
    up = min(-power, 120)
    small.mul_(2.0 ** (power / 2)).mul_(2.0 ** (power - power / 2))
    large.mul_(2.0 ** up)
    y, _ = mpc.mpc_linear_forward(x, w)
    dx, dw, _ = mpc.mpc_linear_backward(dy, x, w, need=(which == "w", which == "x", False))
    off = 2.0 ** -134 if M > 8 else 0.0

    def product(got, a, b, off_a, off_b, count, what):
        """a [m, k] times b [n, k], whose entries are off by off_a and off_b."""
        a, b = a.double(), b.double()
        want = a @ b.t()
        e = (count + 16) * F32 * (a.abs() @ b.abs().t())
        e = e + off_a * b.abs().sum(1)[None, :] + off_b * a.abs().sum(1)[:, None]
        forms.close(got, want, e + F32 * want.abs() + 2.0 ** -149, what)

    product(y, x, w, off, off, K, "y")
    # the gradient's products go through the terms whatever the rows
    if which == "w":
        product(dx, dy, w.t(), 2.0 ** -134, 2.0 ** -134, N, "dx")
    else:
        product(dw, dy.t(), x.t(), 2.0 ** -134, 2.0 ** -134, M, "dw")
    assert mpc.mpc_get_status() == 0
