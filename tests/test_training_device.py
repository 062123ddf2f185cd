"""The loss and optimiser calls launch on the device where their tensors are, whichever is current (no GPU:
tensors that say they are on one, and a library that records its calls)."""

import pytest
import torch

HERE = torch.device("cuda", 1)


class On1(torch.Tensor):
    is_cuda = True
    device = HERE


def there(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(On1)


class FakeStream:
    def __init__(self, device, handle):
        self.device, self.cuda_stream = torch.device("cuda", device), handle


@pytest.fixture
def box(monkeypatch):
    """The package with the device that a launch finds current, and the launches: (name, device, stream)."""
    import paper_2401_07788_gb300 as mpc

    calls = []

    class Device:
        current = 0

        def __init__(self, device):
            self.index = device.index

        def __enter__(self):
            self.before, Device.current = Device.current, self.index

        def __exit__(self, *_):
            Device.current = self.before

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_bytes"):
                    return 64
                calls.append((name, Device.current, args[-1]))
                return 0
            return call

    monkeypatch.setattr(mpc, "lib", lambda: Library())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: Device.current)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)
    monkeypatch.setattr(On1, "record_stream", lambda self, stream: None)
    return mpc, Device, calls


def every_call(mpc, stream):
    h, w, y = there(6, 8), there(10, 8), there(6, dtype=torch.int64)
    loss, lse, dh, dw, ws = there(6), there(6), there(6, 8), there(10, 8), there(64, dtype=torch.uint8)
    mpc.mpc_linear_ce_forward(h, w, y, loss=loss, lse=lse, ws=ws, stream=stream)
    mpc.mpc_linear_ce_backward(h, w, y, lse, dh=dh, dw=dw, ws=ws, stream=stream)
    mpc.mpc_linear_ce_train(h, w, y, loss=loss, dh=dh, dw=dw, ws=ws, stream=stream)
    plan = mpc.AdamWPlan([there(6)], [there(6)], [there(6, dtype=torch.int8)], [there(6, dtype=torch.uint8)],
                         [there(1)], [there(1)])
    mpc.mpc_adamw_step(plan, 1e-3, 0.9, 0.99, 1e-8, 1, grad_norm=there(1), stream=stream)
    mpc.mpc_adamw_decode(plan, [there(6)], [there(6)], stream=stream)
    mpc.mpc_grad_norm(plan, norm=there(1), ws=ws, stream=stream)


NAMES = ["mpc_linear_ce_forward", "mpc_linear_ce_backward", "mpc_linear_ce_train", "mpc_adamw_step",
         "mpc_adamw_decode", "mpc_grad_norm"]


@pytest.mark.parametrize("current", [0, 1])
def test_launches_follow_the_tensors(box, current):
    mpc, device, calls = box
    device.current = current
    every_call(mpc, None)
    assert calls == [(name, 1, 1001) for name in NAMES]
    assert device.current == current


def test_a_given_stream(box):
    mpc, device, calls = box
    every_call(mpc, FakeStream(1, 77))
    assert calls == [(name, 1, 77) for name in NAMES]
    del calls[:]
    with pytest.raises(mpc.MpcError, match="the stream is on cuda:0"):
        every_call(mpc, FakeStream(0, 78))
    assert calls == []
