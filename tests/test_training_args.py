"""Argument checks of the linear cross entropy, the AdamW step and the gradient norm: the C entry
points refuse bad calls before any launch, the binding refuses tensors it cannot pass (no GPU)."""

import ctypes

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


def forward(mpc, h=P, ldh=64, w=P, ldw=64, y=P, T=8, D=64, V=100, kind=0, loss=P, lse=P, ws=P, size=1 << 40):
    return mpc.lib().mpc_linear_ce_forward(h, ldh, w, ldw, y, T, D, V, kind, -100, loss, lse, ws, size, None)


@pytest.mark.parametrize("change,code", [
    (dict(h=None), 1), (dict(w=None), 1), (dict(y=None), 1), (dict(loss=None), 1), (dict(lse=None), 1),
    (dict(h=P + 2), 1), (dict(w=P + 1, kind=1), 1), (dict(y=P + 4), 1), (dict(loss=P + 2), 1),
    (dict(ldh=63), 1), (dict(ldw=0), 1), (dict(ldw=-64), 1), (dict(T=-1), 1), (dict(T=1 << 31), 1), (dict(D=0), 1),
    (dict(D=1 << 25), 1), (dict(V=0), 1), (dict(V=1 << 31), 1), (dict(kind=2), 1), (dict(ldh=1 << 62), 1),
    (dict(ws=None), 3), (dict(size=100), 3), (dict(ws=P + 128), 1),
])
def test_linear_ce_forward_refuses(mpc, change, code):
    assert forward(mpc, **change) == code
    assert mpc.mpc_last_error() != ""


def backward(mpc, train=False, h=P, w=P, y=P, lse=P, g=None, T=8, D=64, V=100, kind=0, piece=0, dh=P, lddh=64, dw=P,
             lddw=64, ws=P, size=1 << 40):
    f = mpc.lib()
    if train:
        return f.mpc_linear_ce_train(h, 64, w, 64, y, g, T, D, V, kind, -100, piece, lse, dh, lddh, dw, lddw, ws, size, None)
    return f.mpc_linear_ce_backward(h, 64, w, 64, y, lse, g, T, D, V, kind, -100, piece, dh, lddh, dw, lddw, ws, size, None)


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("change,code", [
    (dict(dh=None), 1), (dict(dw=None), 1), (dict(lse=None), 1), (dict(g=P + 1), 1), (dict(lddh=10), 1), (dict(lddw=63), 1),
    (dict(piece=-1), 1), (dict(dw=P + 2), 1), (dict(size=10), 3), (dict(T=0, dw=None), 1),
])
def test_linear_ce_backward_refuses(mpc, train, change, code):
    assert backward(mpc, train, **change) == code


def test_no_tokens_is_a_no_op(mpc):
    assert forward(mpc, T=0, h=None, y=None, loss=None, lse=None, ws=None, size=0) == 0


def test_linear_ce_workspace(mpc):
    size = mpc.mpc_linear_ce_workspace_bytes
    assert size(0, 64, 100) == 0
    a, b = size(128, 64, 5000, torch.float32, False), size(128, 64, 5000, torch.float32, True)
    assert 0 < a < b and a % 256 == 0 and b % 256 == 0
    # the coefficients of a piece bound what training takes, not those of the vocabulary
    small, large = (size(8192, 768, 131072, torch.bfloat16, True, p) for p in (1024, 0))
    assert small < large < 3 << 30


def entry(mpc, **change):
    from paper_2401_07788_gb300.training import _Tensor

    t = dict(param=P, grad=P, exp_avg=P, exp_avg_sq=P, scale_m=P, scale_v=P, copy=None, n=10, lr_scale=1.0, weight_decay=0.0)
    t.update(change)
    return (_Tensor * 1)(_Tensor(**t))


def step(mpc, table, count=1, pt=0, gt=0, bits=32, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, step=1, norm=None):
    return mpc.lib().mpc_adamw_step(table, count, pt, gt, bits, lr, b1, b2, eps, step, norm, 1.0, None)


@pytest.mark.parametrize("change,args", [
    (dict(param=None), {}), (dict(grad=None), {}), (dict(exp_avg=None), {}), (dict(exp_avg_sq=P + 1), {}),
    (dict(param=P + 2), {}), (dict(param=P + 1), dict(pt=1)), (dict(grad=P + 1), dict(gt=1)), (dict(copy=P + 1), {}),
    (dict(n=-1), {}), (dict(n=(1 << 40) + 1), {}), (dict(scale_m=None), dict(bits=8)), (dict(scale_v=P + 2), dict(bits=8)),
    ({}, dict(bits=16)), ({}, dict(pt=3)), ({}, dict(gt=-1)), ({}, dict(b1=1.0)), ({}, dict(b2=-0.1)),
    ({}, dict(b1=float("nan"))), ({}, dict(eps=-1.0)), ({}, dict(step=0)), ({}, dict(count=-1)), ({}, dict(norm=P + 1)),
])
def test_adamw_refuses(mpc, change, args):
    assert step(mpc, entry(mpc, **change), **args) == 1


def test_adamw_refuses_a_missing_list(mpc):
    assert step(mpc, None) == 1
    assert step(mpc, None, count=0) == 0
    assert step(mpc, entry(mpc, n=0, param=None)) == 0
    assert ctypes.sizeof(entry(mpc)) == 80


def test_decode_and_norm_refuse(mpc):
    f = mpc.lib()
    one = (ctypes.c_void_p * 1)(P)
    none = (ctypes.c_void_p * 1)(None)
    assert f.mpc_adamw_decode(entry(mpc), 1, None, one, None) == 1
    assert f.mpc_adamw_decode(entry(mpc), 1, one, none, None) == 1
    assert f.mpc_adamw_decode(entry(mpc, scale_v=None), 1, one, one, None) == 1
    need = mpc.mpc_grad_norm_workspace_bytes(1)
    assert need > 0
    assert f.mpc_grad_norm(entry(mpc), 1, 0, None, P, need, None) == 1
    assert f.mpc_grad_norm(entry(mpc), 1, 2, P, P, need, None) == 1
    assert f.mpc_grad_norm(entry(mpc), 1, 0, P, P, need - 1, None) == 3
    assert f.mpc_grad_norm(entry(mpc), 1, 0, P, None, need, None) == 3
    assert f.mpc_grad_norm(entry(mpc, grad=P + 2), 1, 0, P, P, need, None) == 1


def test_binding_refuses_cpu_tensors_and_bad_options(mpc):
    x, y = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(mpc.MpcError):
        mpc.mpc_linear_ce_forward(x, torch.zeros(5, 8), y)
    with pytest.raises(mpc.MpcError):
        mpc.AdamWPlan([torch.zeros(4)], [torch.zeros(4)])
    with pytest.raises(mpc.MpcError):
        mpc.AdamWPlan([], [])
    p = torch.nn.Parameter(torch.zeros(4))
    for bad in (dict(state_bits=4), dict(betas=(1.0, 0.9)), dict(eps=-1.0), dict(lr=-1.0)):
        with pytest.raises(ValueError):
            mpc.AdamW([p], **bad)
    with pytest.raises(ValueError):
        mpc.linear_cross_entropy(x, torch.zeros(5, 8), y, reduction="max")
