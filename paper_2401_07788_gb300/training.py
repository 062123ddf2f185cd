"""The two ends of a stage's training step that lie outside its layers: the last stage's loss over
the vocabulary, and the optimiser step that every stage makes after its backward pass.

* ``linear_cross_entropy`` / ``LinearCrossEntropy``: softmax cross entropy of a linear head
  whose loss keeps no logits; the gradient of the hidden states is what the boundary before the last
  stage compresses.
* ``AdamWPlan``: the list of tensors that ``mpc_adamw_step``, ``mpc_grad_norm`` and
  ``mpc_adamw_decode`` take, laid out once.
* ``AdamW``: a ``torch.optim.Optimizer`` on these calls, with fp32 or 8-bit states, bf16 copies of
  fp32 weights and clipping by the global norm.
"""

from __future__ import annotations

import ctypes
import itertools
import operator

import numpy as np
import torch

from . import (MpcError, _data_ptr, _dtype, _numel, _vectors, mpc_adamw_step, mpc_grad_norm,
               mpc_linear_ce_backward, mpc_linear_ce_forward, mpc_linear_ce_train)

__all__ = ["AdamW", "AdamWPlan", "LinearCrossEntropy", "linear_cross_entropy"]

BLOCK = 256  # entries of a tensor that share a scale in the 8-bit states


# ---------------------------------------------------------------------------------------
# Linear cross entropy
# ---------------------------------------------------------------------------------------

class _Final(torch.autograd.Function):
    """A gradient as it is, which raises where it is to be differentiated itself."""

    @staticmethod
    def forward(ctx, grad, *sources):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients of linear_cross_entropy are not differentiable")


def _mean(loss, targets, ignore_index, vocab):
    """The mean over the tokens that count, as the kernels take it for the gradient: those whose target is
    in the vocabulary and is not ignore_index."""
    counts = (targets == targets.clamp(0, vocab - 1)) & (targets != ignore_index)
    return loss.sum() / counts.sum().clamp_min(1)


def _final(grads, *sources):
    """What a backward pass hands out.  Where autograd records it (create_graph), the gradients hang on
    the tensors they come from by a node that refuses: as constants they would add nothing to a
    second derivative.  (torch's once_differentiable does so only where the incoming gradient
    requires one.)"""
    return tuple(None if g is None else _Final.apply(g, *sources) for g in grads)


class _LinearCeFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, w, targets, ignore_index, piece):
        loss, lse = mpc_linear_ce_forward(h, w, targets, ignore_index)
        ctx.save_for_backward(h, w, targets, lse)
        ctx.ignore_index, ctx.piece = ignore_index, piece
        return loss

    @staticmethod
    def backward(ctx, gloss):
        h, w, targets, lse = ctx.saved_tensors
        grads = mpc_linear_ce_backward(h, w, targets, lse, gloss.detach().contiguous().float(),
                                       ctx.ignore_index, ctx.piece)
        grads = [g if need else None for g, need in zip(grads, ctx.needs_input_grad)]
        if torch.is_grad_enabled():
            grads = _final(grads, h, w, gloss)
        return (*grads, None, None, None)


class _LinearCeMeanFn(torch.autograd.Function):
    """The mean: its gradient is known up to one factor when the loss is formed, so both come from
    one call, and the backward pass applies the factor to what that call made and hands it out.
    A further pass through a graph that is kept makes it again."""

    @staticmethod
    def _made(ctx, h, w, targets):
        loss, *grads = mpc_linear_ce_train(h, w, targets, None, ctx.ignore_index, ctx.piece)
        return loss, [g if need else None for g, need in zip(grads, ctx.needs_input_grad)]

    @staticmethod
    def forward(ctx, h, w, targets, ignore_index, piece):
        ctx.ignore_index, ctx.piece = ignore_index, piece
        loss, ctx.grads = _LinearCeMeanFn._made(ctx, h, w, targets)
        ctx.save_for_backward(h, w, targets)
        return _mean(loss, targets, ignore_index, w.shape[0])

    @staticmethod
    def backward(ctx, upstream):
        grads, ctx.grads = ctx.grads, None
        if grads is None:
            _, grads = _LinearCeMeanFn._made(ctx, *ctx.saved_tensors)
        # as a matrix and not a scalar, which would be rounded to the gradients' type first
        g = upstream.detach().float().view(1, 1)
        grads = [None if x is None or not need else torch.mul(x, g, out=x)
                 for x, need in zip(grads, ctx.needs_input_grad)]
        if torch.is_grad_enabled():
            h, w, _ = ctx.saved_tensors
            grads = _final(grads, h, w, upstream)
        return (*grads, None, None, None)


def _rows_apart(t):
    """t itself, or a copy where its rows are not contiguous or share memory (broadcast)."""
    fine = (t.stride(1) == 1 or t.shape[1] == 1) and (t.stride(0) >= t.shape[1] or t.shape[0] == 1)
    return t if fine else t.contiguous()


def linear_cross_entropy(h, w, targets, ignore_index: int = -100, reduction: str = "mean", piece: int = 0):
    """Softmax cross entropy of the logits h @ w.T, h [..., D], w [V, D], targets [...] (int64).
    ``reduction``: "mean" over the tokens that count, "sum", or "none" (a loss for each token, 0
    where the target is ``ignore_index``).  A target outside [0, V) does not count either, and is reported
    by ``mpc_get_status``.  There is no second derivative: asking for one raises.

    The loss by itself keeps no logits.  The gradient of a mean does for the length of its call, as
    exponentials (2 bytes each in bf16, 6 in fp32, 4 GiB at most), and then forms them once.
    ``piece``: the vocabulary entries whose coefficients are held at a time instead, with the logits
    formed twice, a third more work; as the other reductions do, in pieces of 1 GiB at most.  (Up to
    16 tokens may keep 4 bytes a logit whatever ``piece`` is.)"""
    if reduction not in ("mean", "sum", "none"):
        raise ValueError("reduction must be mean, sum or none")
    rows, y = _rows_apart(h.reshape(-1, h.shape[-1])), targets.reshape(-1).contiguous()
    w = _rows_apart(w)
    grad = torch.is_grad_enabled() and (h.requires_grad or w.requires_grad)
    if reduction == "mean":
        if grad:
            return _LinearCeMeanFn.apply(rows, w, y, ignore_index, piece)
        loss = mpc_linear_ce_forward(rows.detach(), w.detach(), y, ignore_index)[0]
        return _mean(loss, y, ignore_index, w.shape[0])
    loss = _LinearCeFn.apply(rows, w, y, ignore_index, piece) if grad else \
        mpc_linear_ce_forward(rows.detach(), w.detach(), y, ignore_index)[0]
    return loss.sum() if reduction == "sum" else loss.reshape(targets.shape)


class LinearCrossEntropy(torch.nn.Module):
    """The head of a last stage: a weight [vocab, hidden] and the loss of its logits; arguments as for
    ``linear_cross_entropy``."""

    def __init__(self, hidden: int, vocab: int, ignore_index: int = -100, reduction: str = "mean",
                 device=None, dtype=None, piece: int = 0):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(vocab, hidden, device=device, dtype=dtype))
        torch.nn.init.normal_(self.weight, std=0.02)
        self.ignore_index = int(ignore_index)
        self.reduction = reduction
        self.piece = int(piece)

    def forward(self, h: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        return linear_cross_entropy(h, self.weight, targets, self.ignore_index, self.reduction, self.piece)


# ---------------------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------------------

class _Tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p),
                ("exp_avg_sq", ctypes.c_void_p), ("scale_m", ctypes.c_void_p),
                ("scale_v", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("lr_scale", ctypes.c_double), ("weight_decay", ctypes.c_double)]


_TABLE = np.dtype([(name, np.float64 if kind is ctypes.c_double else np.int64 if kind is ctypes.c_int64 else np.uint64)
                   for name, kind in _Tensor._fields_])


class AdamWPlan:
    """The tensors of an optimiser step: params (float32, or bfloat16 without a master copy),
    grads, and the states m and v, each a list with one contiguous CUDA tensor for each param.

    States are fp32, or 8-bit codes (m int8, v uint8) with ``m_scale`` and ``v_scale`` (fp32, one
    for each block of 256 entries).  ``m`` None allocates zero states of ``state_bits``.  ``copies``
    (bfloat16, entries may be None) receive the new params as well.  ``weight_decay`` and
    ``lr_scale`` are one number or one for each tensor.
    """

    def __init__(self, params, grads, m=None, v=None, m_scale=None, v_scale=None, copies=None,
                 weight_decay=0.0, lr_scale=1.0, state_bits: int = 32):
        params, grads = list(params), list(grads)
        n = len(params)
        if n == 0:
            raise MpcError(1, "a plan needs at least one tensor")
        if (m is None) != (v is None):
            raise MpcError(1, "m and v are given together")
        self.param_type = _dtype(params[0], "param")
        self.device = params[0].device
        self.norm_ws = None  # mpc_grad_norm's workspace, made by its first call
        self.count = n
        self.sizes = [p.numel() for p in params]
        blocks = [-(-k // BLOCK) for k in self.sizes]
        if m is None:
            if state_bits not in (32, 8):
                raise MpcError(1, "state_bits must be 32 or 8")
            kinds = (torch.float32, torch.float32) if state_bits == 32 else (torch.int8, torch.uint8)
            m, v = ([torch.zeros(k, dtype=t, device=self.device) for k in self.sizes] for t in kinds)
            if state_bits == 8:
                m_scale, v_scale = ([torch.zeros(b, device=self.device) for b in blocks]
                                    for _ in range(2))
        m, v = list(m), list(v)
        self.state_bits = 8 if m and m[0].dtype == torch.int8 else 32
        # the list that the calls take: ctypes owns it, numpy fills whole columns of it
        self.table = (_Tensor * n)()
        self._columns = np.frombuffer(self.table, dtype=_TABLE)
        low = self.state_bits == 8
        if low and (m_scale is None or v_scale is None):
            raise MpcError(1, "8-bit states need m_scale and v_scale")
        self._fill("param", params, params[0].dtype, self.sizes)
        self._fill("exp_avg", m, torch.int8 if low else torch.float32, self.sizes, "m")
        self._fill("exp_avg_sq", v, torch.uint8 if low else torch.float32, self.sizes, "v")
        if low:
            m_scale, v_scale = list(m_scale), list(v_scale)
            self._fill("scale_m", m_scale, torch.float32, blocks, "m_scale")
            self._fill("scale_v", v_scale, torch.float32, blocks, "v_scale")
        copies = [None] * n if copies is None else list(copies)
        if len(copies) != n:
            raise MpcError(1, "%d params but %d copies" % (n, len(copies)))
        there = [i for i, t in enumerate(copies) if t is not None]
        if there:
            self._columns["copy"][there] = _vectors([copies[i] for i in there], [self.sizes[i] for i in there],
                                                    torch.bfloat16, "copy", self.device)
        self._columns["n"] = self.sizes
        self.set_groups(lr_scale, weight_decay)
        self.params, self.m, self.v, self.copies = params, m, v, copies
        self.m_scale, self.v_scale = (m_scale, v_scale) if low else (None, None)
        if not grads:
            raise MpcError(1, "%d params but no grads" % n)
        self.grad_type = _dtype(grads[0], "grad")
        self.set_grads(grads)

    def _fill(self, column, tensors, dtype, sizes, name=None):
        self._columns[column] = _vectors(tensors, sizes, dtype, name or column, self.device)

    def set_grads(self, grads) -> None:
        """Other gradient tensors for the next calls, e.g. those of a new backward pass."""
        grads = list(grads)
        self._fill("grad", grads, torch.bfloat16 if self.grad_type else torch.float32, self.sizes)
        self.grads = grads

    def drop_grads(self) -> None:
        """Lets the gradient tensors go; calls are refused until set_grads gives others."""
        self._columns["grad"] = 0
        self.grads = None

    def set_groups(self, lr_scale, weight_decay) -> None:
        """The factor on lr and the weight decay from the next step on: one number or one for each
        tensor."""
        for name, x in (("lr_scale", lr_scale), ("weight_decay", weight_decay)):
            if not isinstance(x, (int, float)) and len(x) != self.count:
                raise MpcError(1, "%s is one number or one for each tensor" % name)
            self._columns[name] = x


class AdamW(torch.optim.Optimizer):
    """AdamW in one launch for all tensors of a type (and one more pass over the gradients when
    ``max_norm`` is set, which clips by the norm of all of them and leaves out a step whose norm is
    not finite; it still counts as a step for the bias corrections).

    ``state_bits``: 32, or 8 for states in blocks of 256 codes.  ``copies``: {param: bfloat16 tensor}
    that receives the param's new values, for a forward pass in bf16 from fp32 weights.
    Parameters without a gradient are left alone, as are their states.  Nothing holds a gradient
    after the step.
    """

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 1e-2, state_bits: int = 32, max_norm: float = 0.0, copies=None):
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        if not 0.0 <= betas[0] < 1.0 or not 0.0 <= betas[1] < 1.0 or eps < 0.0 or lr < 0.0:
            raise ValueError("lr, betas or eps out of range")
        super().__init__(params, {"lr": lr, "betas": betas, "eps": eps, "weight_decay": weight_decay})
        self.state_bits, self.max_norm = state_bits, max_norm
        self.copies = {} if copies is None else dict(copies)
        self._plans = {}
        self.last_norm = None  # device fp32 of one entry, when max_norm is set

    def __getstate__(self):
        return {**super().__getstate__(), "state_bits": self.state_bits, "max_norm": self.max_norm,
                "copies": self.copies}

    def __setstate__(self, state):
        super().__setstate__(state)
        self._plans, self.last_norm = {}, None

    def _state(self, p):
        s = self.state[p]
        if "exp_avg" not in s:
            n = p.numel()
            low = self.state_bits == 8
            s["step"] = 0
            s["exp_avg"] = torch.zeros(n, dtype=torch.int8 if low else torch.float32, device=p.device)
            s["exp_avg_sq"] = torch.zeros(n, dtype=torch.uint8 if low else torch.float32, device=p.device)
            if low:
                s["scale_m"] = torch.zeros(-(-n // BLOCK), device=p.device)
                s["scale_v"] = torch.zeros(-(-n // BLOCK), device=p.device)
        return s

    def load_state_dict(self, state_dict):
        """Restores the states in the types they were saved in (the codes of 8-bit states are not
        numbers to be cast to the parameter's type); those of the other ``state_bits`` are refused."""
        for s in state_dict["state"].values():
            if "exp_avg" in s and (s["exp_avg"].dtype == torch.int8) != (self.state_bits == 8):
                raise ValueError("the saved states are not of state_bits=%d" % self.state_bits)
        super().load_state_dict(state_dict)
        flat = [p for g in self.param_groups for p in g["params"]]
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        for p, i in zip(flat, saved):
            for k, x in state_dict["state"].get(i, {}).items():
                self.state[p][k] = x.to(p.device).clone() if isinstance(x, torch.Tensor) else x
        self._plans = {}

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        lists = {}
        for group in self.param_groups:
            betas, eps = tuple(group["betas"]), group["eps"]
            rate = float(group["lr"]), float(group["weight_decay"])
            for p in group["params"]:
                g = p.grad
                if g is None:
                    continue
                if g.is_sparse:
                    raise MpcError(1, "sparse gradients are not supported")
                s = self._state(p)
                s["step"] += 1
                key = (p.dtype, g.dtype, p.device, s["step"], betas, eps)
                lists.setdefault(key, []).append((p, g, s, rate))
        plans, used = [], {}
        for key, entries in lists.items():
            params, grads, states, rates = map(list, zip(*entries))
            ident = (*key[:3], *map(id, params))
            plan = self._plans.get(ident)
            grads = [g.contiguous() for g in grads]
            # a plan serves again while it is about the very tensors that the optimizer holds now
            names = ("exp_avg", "exp_avg_sq", "scale_m", "scale_v")[: 4 if self.state_bits == 8 else 2]
            m, v, *scales = ([s[name] for s in states] for name in names)
            copies = [self.copies.get(p) for p in params] if self.copies else None
            held = [*params, *m, *v, *itertools.chain(*scales)]
            places = [*map(_numel, params), *map(_data_ptr, held)]
            if copies is not None:
                held += copies
                places += [None if t is None else _data_ptr(t) for t in copies]
            if (plan is None or plan.places != places or len(plan.held) != len(held)
                    or not all(map(operator.is_, plan.held, held))):
                plan = AdamWPlan([p.detach() for p in params], grads, m, v, *(scales or (None, None)), copies)
                plan.held, plan.places, plan.rates = held, places, None
            else:
                plan.set_grads(grads)
            if plan.rates != rates:
                plan.set_groups(*zip(*rates))
                plan.rates = rates
            plans.append((key, plan))
            used[ident] = plan
        self._plans = used  # lists of other parameters' sets are let go
        norm = None
        if self.max_norm > 0.0 and plans:
            norms = []
            for key, plan in plans:
                with torch.cuda.device(key[2]):
                    norms.append(mpc_grad_norm(plan))
            if len(norms) > 1:  # lists of several types or steps: the norm of their norms
                norm = torch.linalg.vector_norm(torch.cat([x.to(norms[0].device) for x in norms])).view(1)
            else:
                norm = norms[0]
            self.last_norm = norm
        for (_, _, device, step, betas, eps), plan in plans:
            with torch.cuda.device(device):
                mpc_adamw_step(plan, 1.0, betas[0], betas[1], eps, step,
                               grad_norm=None if norm is None else norm.to(device), max_norm=self.max_norm)
            plan.drop_grads()  # zero_grad() is to free them
        return loss
