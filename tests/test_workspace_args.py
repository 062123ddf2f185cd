"""A workspace of the caller's that is not dense memory of the tensors' device is refused before any launch: its address
and size are all that the library sees.  No GPU: tensors that say they are on one, and a library that records its
launches."""

import pytest
import torch

HERE = torch.device("cuda", 1)


class On1(torch.Tensor):
    is_cuda = True
    device = HERE


class On0(torch.Tensor):
    is_cuda = True
    device = torch.device("cuda", 0)


def there(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(On1)


BAD = {
    "on the host": lambda: torch.zeros(4096, dtype=torch.uint8),
    "on another GPU": lambda: torch.zeros(4096, dtype=torch.uint8).as_subclass(On0),
    "with gaps": lambda: there(8192, dtype=torch.uint8)[::2],
    "expanded": lambda: there(1, dtype=torch.uint8).expand(4096),
    "an address": lambda: 0x10000,
}


@pytest.fixture
def box(monkeypatch):
    import paper_2401_07788_gb300 as mpc

    launched = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith(("_bytes", "_words")):
                    return 64
                launched.append(name)
                return 0
            return call

    monkeypatch.setattr(mpc, "lib", lambda: Library())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1001, raising=False)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *shape, device=None, **options: empty(*shape, **options).as_subclass(On1))
    return mpc, launched


def calls(mpc):
    x, w, r = there(4, 16), there(8, 16), there(4, 8)
    targets, lse, rstd = there(4, dtype=torch.int64), there(4), there(4)
    ids, buf = there(2, dtype=torch.int64), there(3, 2, 16)
    plan = mpc.AdamWPlan([there(6)], [there(6)], [there(6)], [there(6)])
    return [
        lambda ws: mpc.mpc_topk_compress(x, 2, ws=ws),
        lambda ws: mpc.mpc_ef_topk_compress(x, there(4, 16), 2, ws=ws),
        lambda ws: mpc.mpc_efmix_topk_compress(x, there(4, 16), 2, ws=ws),
        lambda ws: mpc.mpc_ef21_topk_compress(x, there(4, 16), 2, ws=ws),
        lambda ws: mpc.mpc_aqsgd_compress(there(2, 2, 16), buf, ids, 2, ws=ws),
        lambda ws: mpc.mpc_quant_compress(x, 8, ws=ws),
        lambda ws: mpc.mpc_aqsgd_quant_compress(there(2, 2, 16), buf, ids, 8, ws=ws),
        lambda ws: mpc.mpc_linear_ce_forward(x, w, targets, ws=ws),
        lambda ws: mpc.mpc_linear_ce_backward(x, w, targets, lse, ws=ws),
        lambda ws: mpc.mpc_linear_ce_train(x, w, targets, ws=ws),
        lambda ws: mpc.mpc_grad_norm(plan, ws=ws),
        lambda ws: mpc.mpc_rms_norm_backward(x, x, there(16), rstd, ws=ws),
        lambda ws: mpc.mpc_linear_forward(x, w, ws=ws),
        lambda ws: mpc.mpc_linear_backward(r, x, w, ws=ws),
    ]


@pytest.mark.parametrize("kind", list(BAD))
@pytest.mark.parametrize("which", range(14))
def test_bad_workspaces(box, which, kind):
    mpc, launched = box
    call = calls(mpc)[which]
    call(there(4096, dtype=torch.uint8))
    call(there(64, 16))  # any type of the device's memory
    assert len(launched) == 2
    with pytest.raises(mpc.MpcError, match="ws must be"):
        call(BAD[kind]())
    assert len(launched) == 2
