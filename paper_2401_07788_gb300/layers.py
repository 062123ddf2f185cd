"""The layers of a stage, between its boundaries: the linear layer with bias, activation, dropout and
residual in its epilogue, dropout by itself, and the root-mean-square norm with the residual's
addition.  A block of a stage that normalises before its layers:

    y, h = rms_norm(x, norm.weight, residual=h)          # h: the residual stream
    x = linear(linear(y, up.weight, act="gelu"), down.weight, p=0.1, seed=s)

* ``linear`` / ``Linear``, ``dropout`` / ``Dropout``, ``rms_norm`` / ``RMSNorm``: functions with their
  gradients, and modules on them.  Each makes the ``mpc_*`` calls of its name; these check their arguments.
* ``RMSNorm(..., bits=8)`` is also the end of a stage whose boundary lies behind the norm: its output is sent
  as an 8-bit payload and read back, in fp32.  It is no ``CompressionBoundary``: it sends 8 bits in ``eval()`` as in
  training, and its gradient goes back as it is (``CompressionBoundary(None, Quant(8))`` behind it compresses that).

Dropout: masks are made from a seed where they are used and never stored.  A module's seed is
``(seed << 32) + calls``, with ``calls`` the number of its training calls.  Each of these also draws a number
from torch's CPU generator (4 us).  Recomputation (``torch.utils.checkpoint``) puts that generator back for the
pass that it repeats, so a number that a module drew before marks a repeated call, which takes the earlier
one's mask; so does any other program that puts the generator back.  A call inside a backward pass whose number
is not known (recomputation that leaves the generator alone, or more than ``remembered`` calls later) is
refused.

A captured graph repeats the host's numbers at every replay, so a module refuses to be captured unless it is
given a device counter (``step=tensor``, int64, one entry) that the program advances between steps, after the
backward pass.  All calls between two advances take one mask: with several micro-batches a step, advance it
after each one's backward pass.

When masks repeat: a copy of a module (``copy.deepcopy``, a pickle) has its seed and count, so it drops the same places
at its next call; layers cloned from one another want seeds of their own (``layer.seed = ...``).  A copy's device counter
is a copy too, which the program has to advance.  ``calls`` is in no state dict: a run that resumes with a given seed
sets it (``layer.calls = ...``), or its first masks are those of the first run.

None of the gradients here can be differentiated again, and there are no forward-mode derivatives: asking for
either raises.
"""

from __future__ import annotations

import collections

import torch

from . import (MpcError, _differentiated, mpc_dropout, mpc_linear_backward, mpc_linear_forward,
               mpc_quant_decompress, mpc_rms_norm_backward, mpc_rms_norm_forward, mpc_rms_norm_quant)

__all__ = ["Dropout", "Linear", "RMSNorm", "dropout", "linear", "rms_norm"]


class _Final(torch.autograd.Function):
    """A gradient as it is, which raises where it is to be differentiated itself."""

    @staticmethod
    def forward(ctx, grad, *sources):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients of a stage's layers are not differentiable")


def _final(grads, *sources):
    """What a backward pass hands out; where autograd records it, hung on the tensors it comes from by a node
    that refuses (as constants the gradients would add nothing to a second derivative)."""
    if not torch.is_grad_enabled():
        return tuple(grads)
    sources = [s for s in sources if s is not None]
    return tuple(None if g is None else _Final.apply(g, *sources) for g in grads)


def _rows(t):
    """t as a matrix of its last dimension's rows; a copy where they are not contiguous or share memory."""
    t = t.reshape(-1, t.shape[-1])
    fine = (t.stride(1) == 1 or t.shape[1] == 1) and (t.stride(0) >= t.shape[1] or t.shape[0] <= 1)
    return t if fine else t.contiguous()


def _whole(t):
    return None if t is None else t.contiguous()


class _LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, residual, act, p, seed, step):
        y, z = mpc_linear_forward(x, w, bias, residual, act=act, p=p, seed=seed, step=step, keep=act is not None)
        # x: for dw; x and bias also to hang the gradients on them where they depend on them by z
        ctx.save_for_backward(x if ctx.needs_input_grad[1] or act is not None else None, w, z, step,
                              None if act is None else bias)
        ctx.call = act, p, seed
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w, z, step, bias = ctx.saved_tensors
        act, p, seed = ctx.call
        need = ctx.needs_input_grad
        grads = None, None, None
        if any(need[:3]):
            grads = mpc_linear_backward(_rows(dy.detach()), x, w, z, act=act, p=p, seed=seed, step=step, need=need[:3])
        return (*_final(grads, x, w, bias, dy), dy if need[3] else None, None, None, None, None)


def linear(x, w, bias=None, residual=None, act: str | None = None, p: float = 0.0, seed: int = 0, step=None):
    """residual + drop(act(x @ w.T + bias)), x [..., K], w [N, K], residual [..., N].  act: None, "relu", "gelu",
    "gelu_tanh" or "silu"; ``p``, ``seed`` and ``step`` as for ``dropout``.  With an activation the gradient keeps
    the values before it, in the type of x."""
    shape = (*x.shape[:-1], w.shape[0])
    if residual is not None:
        if residual.shape != shape:
            raise MpcError(1, "residual must have the shape %s" % (tuple(shape),))
        residual = _rows(residual)
    rows, w, bias = _rows(x), _rows(w), _whole(bias)
    if _differentiated(rows, w, bias, residual):
        y = _LinearFn.apply(rows, w, bias, residual, act, p, seed, step)
    else:
        y, _ = mpc_linear_forward(rows, w, bias, residual, act=act, p=p, seed=seed, step=step)
    return y.view(shape)


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, step):
        ctx.save_for_backward(step)
        ctx.call = p, seed
        return mpc_dropout(x, p, seed, residual=residual, step=step)

    @staticmethod
    def backward(ctx, dy):
        p, seed = ctx.call
        (step,) = ctx.saved_tensors
        dx = None
        if ctx.needs_input_grad[0]:
            dx = mpc_dropout(dy.detach().contiguous(), p, seed, step=step)
        return (*_final((dx,), dy), dy if ctx.needs_input_grad[1] else None, None, None, None)


def dropout(x, p: float, seed: int = 0, residual=None, step=None):
    """residual + drop(x): entries are dropped with probability p, the others scaled by 1 / (1 - p).  The mask
    follows from ``seed`` (plus ``step``, an int64 device tensor of one entry) and the entry's number."""
    x, residual = x.contiguous(), _whole(residual)
    if residual is not None and residual.shape != x.shape:
        raise MpcError(1, "residual must have the shape %s" % (tuple(x.shape),))
    if _differentiated(x, residual):
        return _DropoutFn.apply(x, residual, p, seed, step)
    return mpc_dropout(x, p, seed, residual=residual, step=step)


class _RmsNormFn(torch.autograd.Function):
    """(y, h): h = x + residual, whose other uses' gradient arrives as dh."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps, bits):
        ctx.set_materialize_grads(False)
        if bits is None:
            y, h, rstd = mpc_rms_norm_forward(x, weight, eps, residual=residual)
        else:
            codes, scale, minv, h, rstd = mpc_rms_norm_quant(x, weight, eps, residual=residual)
            y = mpc_quant_decompress(codes, scale, minv, x.shape[1], 8)
        ctx.save_for_backward(h, weight, rstd)
        return (y,) if residual is None else (y, h)

    @staticmethod
    def backward(ctx, dy, dh=None):
        h, weight, rstd = ctx.saved_tensors
        need = ctx.needs_input_grad
        if dy is None:  # only h was used
            return dh, dh if need[1] else None, None, None, None
        more = None if dh is None else _rows(dh.detach())
        if dy.dtype != h.dtype:
            # what bf16 rows sent was read back in fp32: its gradient is used as it is, on fp32 copies of the bf16
            # operands, and the results are rounded once
            more = None if more is None else more.float()
            dx, dw = mpc_rms_norm_backward(_rows(dy.detach()), h.float(), weight.float(), rstd, dh=more, need_weight=need[2])
            dx, dw = dx.to(h.dtype), None if dw is None else dw.to(h.dtype)
        else:
            dx, dw = mpc_rms_norm_backward(_rows(dy.detach()), h, weight, rstd, dh=more, need_weight=need[2])
        dx, dw = _final((dx, dw), h, weight, dy, dh)
        return dx if need[0] else None, dx if need[1] else None, dw, None, None


def rms_norm(x, weight, eps: float = 1e-6, residual=None, bits: int | None = None):
    """Root-mean-square norm over the last dimension.  Without a residual: y.  With one: (y, h), the norm of
    h = x + residual and h itself, in the type of x.  ``bits`` 8: y is what a receiver reads back from the norm's
    8-bit payload, in fp32; its gradient goes through as if it had not been rounded."""
    if bits not in (None, 8):
        raise MpcError(2, "bits must be None or 8, got %r" % (bits,))
    shape = x.shape
    if residual is not None and residual.shape != shape:
        raise MpcError(1, "residual must have the shape %s" % (tuple(shape),))
    x = _rows(x)
    out = _RmsNormFn.apply(x, None if residual is None else _rows(residual), weight.contiguous(), eps, bits)
    return out[0].view(shape) if residual is None else (out[0].view(shape), out[1].view(shape))


# ---------------------------------------------------------------------------------------
# Modules
# ---------------------------------------------------------------------------------------

class _Seeded(torch.nn.Module):
    """The dropout seeds of a module: (seed << 32) + the number of its training calls, or the device counter.

    ``_known`` holds the seeds of the last calls by the numbers that they drew from torch's CPU generator
    (about 200 bytes each)."""

    remembered = 4096

    def _seeded(self, p, seed, step):
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must be in [0, 1]")
        self.p = float(p)
        self.seed = int(torch.randint(1 << 31, ()) if seed is None else seed)
        self.step, self.calls = step, 0
        self._known = collections.OrderedDict()

    def __getstate__(self):
        # what only passes in flight need is not copied
        return self.__dict__ | {"_known": collections.OrderedDict()}

    def __setstate__(self, state):
        super().__setstate__({"_known": collections.OrderedDict()} | state)

    def _draw(self, device):
        """(p, seed, step) of one call."""
        if not self.training or self.p == 0.0:
            return 0.0, 0, None
        if self.step is None:
            if device.type == "cuda" and torch.cuda.is_current_stream_capturing():
                raise MpcError(1, "a captured dropout needs a device counter: every replay would repeat its mask")
            drawn = int(torch.randint(1 << 62, (), device="cpu"))
            seed = self._known.get(drawn)
            if seed is None:
                if torch._C._current_graph_task_id() != -1:  # in a backward pass
                    raise MpcError(1, "a dropout that is recomputed needs torch's CPU generator as it was at the first "
                                      "call (preserve_rng_state), and no more than %d other calls since" % self.remembered)
                self.calls += 1
                seed = self._known[drawn] = (self.seed << 32) + self.calls
                if len(self._known) > self.remembered:
                    self._known.popitem(last=False)
            return self.p, seed, None
        return self.p, self.seed << 32, self.step


class Dropout(_Seeded):
    """residual + drop(x) in training, residual + x otherwise.  ``seed`` None: drawn from torch's generator."""

    def __init__(self, p: float = 0.5, seed: int | None = None, step: torch.Tensor | None = None):
        super().__init__()
        self._seeded(p, seed, step)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None) -> torch.Tensor:
        p, seed, step = self._draw(x.device)
        if p == 0.0:
            return x if residual is None else x + residual
        return dropout(x, p, seed, residual, step)


class Linear(_Seeded):
    """A weight [outputs, inputs], a bias, an activation and dropout; forward(x, residual) adds a residual.
    Initialised as torch.nn.Linear is."""

    def __init__(self, inputs: int, outputs: int, bias: bool = True, act: str | None = None, p: float = 0.0,
                 seed: int | None = None, step: torch.Tensor | None = None, device=None, dtype=None):
        super().__init__()
        if act not in (None, "relu", "gelu", "gelu_tanh", "silu"):
            raise ValueError("act must be None, 'relu', 'gelu', 'gelu_tanh' or 'silu'")
        self.act = act
        self.weight = torch.nn.Parameter(torch.empty(outputs, inputs, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.empty(outputs, device=device, dtype=dtype)) if bias else None
        bound = inputs ** -0.5
        for t in (self.weight, self.bias):
            if t is not None:
                torch.nn.init.uniform_(t, -bound, bound)
        self._seeded(p, seed, step)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None) -> torch.Tensor:
        return linear(x, self.weight, self.bias, residual, self.act, *self._draw(x.device))


class RMSNorm(torch.nn.Module):
    """A weight [width] of ones; forward(x) is the norm, forward(x, residual) the pair (norm, x + residual).  ``bits`` 8: the
    norm by way of its 8-bit payload, in fp32, in training and in ``eval()`` alike."""

    def __init__(self, width: int, eps: float = 1e-6, bits: int | None = None, device=None, dtype=None):
        super().__init__()
        if bits not in (None, 8):
            raise ValueError("bits must be None or 8")
        self.weight = torch.nn.Parameter(torch.ones(width, device=device, dtype=dtype))
        self.eps, self.bits = float(eps), bits

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        return rms_norm(x, self.weight, self.eps, residual, self.bits)
