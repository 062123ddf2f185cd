"""The norm's gradient of a few long rows, in a workspace of the size that the query gives and no more."""

import pytest
import torch

import layer_forms as forms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mpc():
    import paper_2401_07788_gb300 as m

    return m


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("need_weight", [True, False])
@pytest.mark.parametrize("M,D", [(1, 8193), (1, 16385), (2, 30001), (5, 16384), (303, 8200), (304, 16400), (310, 17000), (1, 1 << 24)])
def test_workspace_is_enough(mpc, M, D, need_weight, kind):
    gen = torch.Generator("cuda").manual_seed(M + D)
    x, dy = (torch.randn(M, D, device="cuda", generator=gen).to(forms.KINDS[kind]) for _ in range(2))
    w = (1.0 + 0.3 * torch.randn(D, device="cuda", generator=gen)).to(x.dtype)
    _, h, rstd = mpc.mpc_rms_norm_forward(x, w, 1e-5)
    need = mpc.mpc_rms_norm_workspace_bytes(M, D)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    dx, dw = mpc.mpc_rms_norm_backward(dy, h, w, rstd, need_weight=need_weight, ws=ws[:need])
    assert (ws[need:] == 77).all(), "written behind the workspace"
    n, g = h.double() * rstd.double().view(-1, 1), dy.double() * w.double()
    want = rstd.double().view(-1, 1) * (g - n * (g * n).mean(1, keepdim=True))
    # sums of up to D / 1024 entries a thread and 10 levels in fp32
    steps, u = 48 + D // 1024, forms.half(x.dtype)
    rough = (g * n).abs().mean(1, keepdim=True)
    e = rstd.double().view(-1, 1) * (g.abs() * 8 * forms.F32 + n.abs() * rough * 3 * steps * forms.F32) + 4 * forms.F32 * want.abs()
    forms.close(dx, want, e + u * (want.abs() + e), "dx")
    if need_weight:
        want = (dy.double() * n).sum(0)
        e = (dy.double() * n).abs().sum(0) * (M + steps) * forms.F32
        forms.close(dw, want, e + u * (want.abs() + e), "dw")
    else:
        assert dw is None
    assert mpc.mpc_get_status() == 0
