"""Argument checks of the stage's layers: the C entry points refuse bad calls before any launch, the binding and
the modules refuse what they cannot pass (no GPU)."""

import pytest
import torch

P = 0x10000  # an address that no call reaches


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    m.lib()
    return m


@pytest.mark.parametrize("change,code", [
    (dict(x=None), 1), (dict(y=None), 1), (dict(x=P + 2), 1), (dict(r=P + 1), 1), (dict(kind=2), 1), (dict(kind=-1), 1),
    (dict(n=-1), 1), (dict(n=(1 << 40) + 1), 1), (dict(p=-0.1), 1), (dict(p=1.1), 1), (dict(p=float("nan")), 1),
    (dict(step=P + 4), 1), (dict(n=0, x=None, y=None), 0),
])
def test_dropout_refuses(mpc, change, code):
    a = dict(x=P, r=None, n=8, kind=0, p=0.5, seed=1, step=None, y=P) | change
    assert mpc.lib().mpc_dropout(a["x"], a["r"], a["n"], a["kind"], a["p"], a["seed"], a["step"], a["y"], None) == code
    assert (mpc.mpc_last_error() != "") == (code != 0)


NORM = [
    (dict(x=None), 1), (dict(w=None), 1), (dict(x=P + 2), 1), (dict(w=P + 1, kind=1), 1), (dict(ldx=63), 1),
    (dict(rows=-1), 1), (dict(rows=1 << 31), 1), (dict(D=0), 1), (dict(D=(1 << 24) + 1), 1), (dict(kind=3), 1),
    (dict(eps=-1e-6), 1), (dict(eps=float("nan")), 1), (dict(ldx=1 << 62), 1), (dict(r=P, ldr=10), 1), (dict(r=P + 2), 1),
    (dict(h=P, ldh=63), 1), (dict(h=P + 2), 1), (dict(rstd=P + 2), 1),
]


@pytest.mark.parametrize("change,code", NORM + [(dict(y=None), 1), (dict(ldy=63), 1), (dict(rows=0, x=None, y=None), 0)])
def test_norm_refuses(mpc, change, code):
    a = dict(x=P, ldx=64, r=None, ldr=64, w=P, rows=4, D=64, kind=0, eps=1e-6, y=P, ldy=64, h=None, ldh=64, rstd=None) | change
    assert mpc.lib().mpc_rms_norm_forward(*a.values(), None) == code


@pytest.mark.parametrize("change,code", NORM + [(dict(codes=None), 1), (dict(codes=P + 8), 1), (dict(scale=None), 1),
                                                (dict(minv=P + 2), 1), (dict(rows=0, x=None, codes=None), 0)])
def test_norm_quant_refuses(mpc, change, code):
    a = dict(x=P, ldx=64, r=None, ldr=64, w=P, rows=4, D=64, kind=0, eps=1e-6, codes=P, scale=P, minv=P, h=None, ldh=64,
             rstd=None) | change
    assert mpc.lib().mpc_rms_norm_quant(*a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(dy=None), 1), (dict(h=None), 1), (dict(w=None), 1), (dict(rstd=None), 1), (dict(dx=None), 1), (dict(lddy=63), 1),
    (dict(ldh=0), 1), (dict(dh=P, lddh=8), 1), (dict(lddx=63), 1), (dict(dw=P + 2), 1), (dict(ws=None), 3), (dict(size=100), 3),
    (dict(ws=P + 8), 1), (dict(kind=2), 1), (dict(D=0), 1), (dict(rows=-5), 1), (dict(rows=0, dw=None, ws=None), 0),
])
def test_norm_backward_refuses(mpc, change, code):
    a = dict(dy=P, lddy=64, h=P, ldh=64, w=P, rstd=P, dh=None, lddh=64, rows=4, D=64, kind=0, dx=P, lddx=64, dw=P, ws=P,
             size=1 << 30) | change
    assert mpc.lib().mpc_rms_norm_backward(*a.values(), None) == code


SIZES = [(dict(rows=-1), 1), (dict(rows=(1 << 30) + 1), 1), (dict(K=0), 1), (dict(N=0), 1), (dict(K=(1 << 24) + 1), 1),
         (dict(N=(1 << 24) + 1), 1), (dict(kind=2), 1), (dict(act=5), 1), (dict(act=-1), 1), (dict(p=-1.0), 1), (dict(p=2.0), 1),
         (dict(p=float("nan")), 1), (dict(step=P + 4), 1), (dict(ldx=63), 1), (dict(ldw=63), 1)]


@pytest.mark.parametrize("change,code", SIZES + [
    (dict(x=None), 1), (dict(w=None), 1), (dict(y=None), 1), (dict(x=P + 2), 1), (dict(b=P + 1), 1), (dict(r=P, ldr=31), 1),
    (dict(ldy=31), 1), (dict(z=P, ldz=31), 1), (dict(z=P + 2), 1), (dict(rows=0, x=None, y=None, ws=None), 0),
])
def test_linear_forward_refuses(mpc, change, code):
    a = dict(x=P, ldx=64, w=P, ldw=64, b=None, r=None, ldr=32, rows=200, K=64, N=32, kind=0, act=0, p=0.0, seed=0, step=None, y=P,
             ldy=32, z=None, ldz=32, ws=P, size=1 << 40) | change
    assert mpc.lib().mpc_linear_forward(*a.values(), None) == code


@pytest.mark.parametrize("change,code", SIZES + [
    (dict(dy=None), 1), (dict(x=None), 1), (dict(w=None), 1), (dict(lddy=31), 1), (dict(act=2, z=None), 1), (dict(act=2, ldz=31), 1),
    (dict(dx=P + 2), 1), (dict(lddx=63), 1), (dict(lddw=63), 1), (dict(db=P + 2), 1), (dict(ws=None), 3), (dict(size=10), 3),
    (dict(ws=P + 128), 1), (dict(rows=0, dx=None, dw=None, db=None, ws=None), 0), (dict(dx=None, dw=None, db=None, ws=None), 0),
])
def test_linear_backward_refuses(mpc, change, code):
    a = dict(dy=P, lddy=32, x=P, ldx=64, w=P, ldw=64, z=P, ldz=32, rows=200, K=64, N=32, kind=0, act=0, p=0.0, seed=0, step=None,
             dx=P, lddx=64, dw=P, lddw=64, db=P, ws=P, size=1 << 40) | change
    assert mpc.lib().mpc_linear_backward(*a.values(), None) == code


def test_workspace_queries(mpc):
    assert mpc.mpc_rms_norm_workspace_bytes(0, 64) == 0 and mpc.mpc_rms_norm_workspace_bytes(-1, 64) == 0
    assert mpc.mpc_rms_norm_workspace_bytes(4, 64) >= 4 * 64
    assert mpc.mpc_linear_workspace_bytes(0, 64, 64) == 0 and mpc.mpc_linear_workspace_bytes(5, 0, 64) == 0
    assert mpc.mpc_linear_workspace_bytes(300, 64, 32, torch.bfloat16, backward=True) > 0


def test_binding_refuses(mpc):
    x, w = torch.zeros(4, 8), torch.zeros(3, 8)
    for call in (lambda: mpc.mpc_dropout(x, 0.5), lambda: mpc.mpc_linear_forward(x, w), lambda: mpc.mpc_rms_norm_forward(x, w[0]),
                 lambda: mpc.mpc_rms_norm_quant(x, w[0]), lambda: mpc.mpc_linear_backward(x, x, w),
                 lambda: mpc.mpc_rms_norm_backward(x, x, w[0], x[0]), lambda: mpc.linear(x, w), lambda: mpc.dropout(x, 0.5),
                 lambda: mpc.rms_norm(x, w[0])):
        with pytest.raises(mpc.MpcError, match="CUDA tensor"):
            call()


def test_functions_and_modules_refuse(mpc):
    x, w = torch.zeros(4, 8), torch.zeros(3, 8)
    with pytest.raises(mpc.MpcError, match="residual must have the shape"):
        mpc.linear(x, w, residual=x)
    with pytest.raises(mpc.MpcError, match="residual must have the shape"):
        mpc.dropout(x, 0.5, residual=w)
    with pytest.raises(mpc.MpcError, match="residual must have the shape"):
        mpc.rms_norm(x, w[0], residual=w)
    with pytest.raises(mpc.MpcError, match="bits"):
        mpc.rms_norm(x, w[0], bits=4)
    for make in (lambda: mpc.Linear(8, 8, act="tanh"), lambda: mpc.Linear(8, 8, p=1.5), lambda: mpc.Dropout(-0.1),
                 lambda: mpc.RMSNorm(8, bits=7)):
        with pytest.raises(ValueError):
            make()


def test_module_seeds(mpc):
    """Modules draw their seeds from torch's generator; a call's seed is its module's and its number."""
    torch.manual_seed(5)
    a, b = mpc.Dropout(0.5), mpc.Dropout(0.5)
    torch.manual_seed(5)
    c = mpc.Dropout(0.5)
    assert a.seed == c.seed != b.seed
    cpu = torch.device("cpu")
    assert a._draw(cpu) == (0.5, (a.seed << 32) + 1, None) and a._draw(cpu) == (0.5, (a.seed << 32) + 2, None)
    a.eval()
    assert a._draw(cpu) == (0.0, 0, None)
