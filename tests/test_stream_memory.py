"""A call on a stream of the caller's choice takes its outputs and its workspace from that stream's memory (what the
allocator hands out for the current stream may still be read or written by work that is queued there), and
the outputs are the current stream's too.  No GPU: tensors that say they are on one, an allocator and a library that
record their calls."""

import contextlib

import pytest
import torch

HERE = torch.device("cuda", 1)


class On1(torch.Tensor):
    is_cuda = True
    device = HERE


def there(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(On1)


class FakeStream:
    def __init__(self, name, handle):
        self.name, self.device, self.cuda_stream = name, HERE, handle

    def __repr__(self):
        return self.name


SIDE, MAIN = FakeStream("side", 77), FakeStream("main", 1001)


@pytest.fixture
def box(monkeypatch):
    """The package, what was allocated as (tensor, the stream then), and what was recorded as (tensor, stream)."""
    import paper_2401_07788_gb300 as mpc

    empty, made, recorded, current = torch.empty, [], [], [MAIN]

    class Library:
        def __getattr__(self, name):
            return lambda *args: 64 if name.endswith(("_bytes", "_words")) else 0

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def allocate(*shape, device=None, **options):
        t = empty(*shape, **options).as_subclass(On1)
        made.append((t, current[-1]))
        return t

    monkeypatch.setattr(mpc, "lib", lambda: Library())
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(torch, "empty_like", lambda t: allocate(t.shape, dtype=t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1001, raising=False)
    monkeypatch.setattr(On1, "record_stream", lambda self, stream: recorded.append((self, stream)))
    return mpc, made, recorded


def calls(mpc):
    """Every call of the binding that allocates: a function of the stream that returns its outputs."""
    x, w, bias, r = there(4, 16), there(8, 16), there(8), there(4, 8)
    vals, idx = there(4, 2), there(4, 2, dtype=torch.int32)
    codes, scale = there(4, 16, dtype=torch.int32), there(4)
    targets, lse, rstd = there(4, dtype=torch.int64), there(4), there(4)
    ids, buf = there(2, dtype=torch.int64), there(3, 2, 16)
    plan = mpc.AdamWPlan([there(6)], [there(6)], [there(6)], [there(6)])
    return {
        "topk": lambda s: mpc.mpc_topk_compress(x, 2, stream=s),
        "ef": lambda s: mpc.mpc_ef_topk_compress(x, there(4, 16), 2, stream=s),
        "efmix": lambda s: mpc.mpc_efmix_topk_compress(x, there(4, 16), 2, stream=s),
        "ef21": lambda s: mpc.mpc_ef21_topk_compress(x, there(4, 16), 2, stream=s),
        "topk_decompress": lambda s: (mpc.mpc_topk_decompress(vals, idx, 16, stream=s),),
        "gather": lambda s: (mpc.mpc_topk_gather(x, idx, stream=s),),
        "aqsgd": lambda s: mpc.mpc_aqsgd_compress(there(2, 2, 16), buf, ids, 2, stream=s),
        "quant": lambda s: mpc.mpc_quant_compress(x, 8, stream=s),
        "dequant": lambda s: (mpc.mpc_quant_decompress(codes, scale, scale, 16, 8, stream=s),),
        "aqsgd_quant": lambda s: mpc.mpc_aqsgd_quant_compress(there(2, 2, 16), buf, ids, 8, stream=s),
        "ce_forward": lambda s: mpc.mpc_linear_ce_forward(x, w, targets, stream=s),
        "ce_backward": lambda s: mpc.mpc_linear_ce_backward(x, w, targets, lse, stream=s),
        "ce_train": lambda s: mpc.mpc_linear_ce_train(x, w, targets, stream=s),
        "grad_norm": lambda s: (mpc.mpc_grad_norm(plan, stream=s),),
        "dropout": lambda s: (mpc.mpc_dropout(x, 0.5, stream=s),),
        "norm": lambda s: mpc.mpc_rms_norm_forward(x, there(16), residual=there(4, 16), stream=s),
        "norm_quant": lambda s: mpc.mpc_rms_norm_quant(x, there(16), residual=there(4, 16), stream=s),
        "norm_backward": lambda s: mpc.mpc_rms_norm_backward(x, x, there(16), rstd, stream=s),
        "linear": lambda s: mpc.mpc_linear_forward(x, w, bias, r, keep=True, stream=s),
        "linear_backward": lambda s: mpc.mpc_linear_backward(r, x, w, stream=s),
    }


NAMES = ["topk", "ef", "efmix", "ef21", "topk_decompress", "gather", "aqsgd", "quant", "dequant", "aqsgd_quant", "ce_forward",
         "ce_backward", "ce_train", "grad_norm", "dropout", "norm", "norm_quant", "norm_backward", "linear",
         "linear_backward"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_the_stream_that_writes_it(box, name):
    mpc, made, recorded = box
    call = calls(mpc)[name]
    del made[:]
    out = call(SIDE)
    assert made and all(stream is SIDE for _, stream in made)
    for t in out:
        assert any(t is a for a, _ in made), "an output was allocated elsewhere"
        assert any(t is a and stream is MAIN for a, stream in recorded)


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_the_current_stream(box, name):
    mpc, made, recorded = box
    call = calls(mpc)[name]
    del made[:]
    call(None)
    assert made and all(stream is MAIN for _, stream in made) and not recorded
