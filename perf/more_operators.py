"""Measured cases of the operators that a stage's layers are made of: the linear layer with bias, activation,
dropout and residual in its epilogue, dropout by itself, and the root-mean-square norm with the residual's
addition, whose output may leave in 8 bits."""

import math

import numpy as np
import torch

own = False  # False: plain torch operations; True: the calls a user makes of the package

EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token through an up projection: a serving call, where latency counts
        {"name": "linear_token", "op": "linear", "grad": False, "M": 1, "K": 1024, "N": 4096, "type": "bf16",
         "act": "gelu_tanh", "bias": True, "residual": False, "p": 0.0},
        # a batch of single tokens through a projection back into the residual stream
        {"name": "linear_decode_24", "op": "linear", "grad": False, "M": 24, "K": 4096, "N": 4096, "type": "bf16",
         "act": None, "bias": False, "residual": True, "p": 0.0},
        # a ragged prompt through a wide up projection
        {"name": "linear_prompt", "op": "linear", "grad": False, "M": 2000, "K": 4096, "N": 8192, "type": "bf16",
         "act": "silu", "bias": False, "residual": False, "p": 0.0},
        # odd sizes in the fp32 that the boundaries exchange
        {"name": "linear_odd_f32", "op": "linear", "grad": True, "M": 1000, "K": 777, "N": 2051, "type": "f32",
         "act": "gelu", "bias": True, "residual": False, "p": 0.0},
        # training, batch 8 of 1024 tokens: the down projection with bias, dropout and residual
        {"name": "linear_down_train", "op": "linear", "grad": True, "M": 8192, "K": 4096, "N": 1024, "type": "bf16",
         "act": None, "bias": True, "residual": True, "p": 0.1},
        # the largest: a wide up projection in training
        {"name": "linear_up_train", "op": "linear", "grad": True, "M": 16384, "K": 4096, "N": 16384, "type": "bf16",
         "act": "gelu_tanh", "bias": True, "residual": False, "p": 0.0},
        # a short sequence's dropout before the residual's addition: launch-bound
        {"name": "dropout_small", "op": "dropout", "grad": False, "M": 16, "N": 1024, "type": "bf16",
         "residual": True, "p": 0.1},
        # a training step's dropout, forward and backward, in fp32
        {"name": "dropout_train", "op": "dropout", "grad": True, "M": 16384, "N": 4096, "type": "f32",
         "residual": True, "p": 0.1},
        # the norm of a single token
        {"name": "norm_token", "op": "norm", "pass": "forward", "M": 1, "N": 4096, "type": "bf16", "residual": True},
        # a training step's norm with the residual's addition, and the gradient that comes along the residual stream
        {"name": "norm_train", "op": "norm", "pass": "train", "M": 16384, "N": 4096, "type": "bf16",
         "residual": True},
        # a boundary behind the norm, batch 8 of 1024 tokens of width 768: sent in 8 bits and read back
        {"name": "norm_send_768", "op": "norm", "pass": "send", "M": 8192, "N": 768, "type": "f32",
         "residual": True},
        # the same for a ragged batch of an odd width in bf16
        {"name": "norm_send_odd", "op": "norm", "pass": "send", "M": 3001, "N": 2051, "type": "bf16",
         "residual": False},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))

    def width(lo, hi):  # widths of layers are mostly multiples of 64, and sometimes anything
        n = log(lo, hi)
        return max(lo, min(hi, -(-n // 64) * 64)) if rng.random() < 0.6 else n

    which = rng.random()
    if which < 0.5:
        return {"op": "linear", "grad": rng.random() < 0.6, "M": log(1, 16384), "K": width(16, 4096),
                "N": width(16, 8192), "type": rng.choice(("f32", "bf16")),
                "act": rng.choice((None, "gelu", "gelu_tanh", "silu")), "bias": rng.random() < 0.7,
                "residual": rng.random() < 0.5, "p": rng.choice((0.0, 0.0, 0.1, 0.5))}
    if which < 0.7:
        return {"op": "dropout", "grad": rng.random() < 0.5, "M": log(1, 16384), "N": width(16, 8192),
                "type": rng.choice(("f32", "bf16")), "residual": rng.random() < 0.6,
                "p": rng.choice((0.05, 0.1, 0.123, 0.5))}
    return {"op": "norm", "pass": rng.choice(("forward", "train", "send")), "M": log(1, 16384), "N": width(16, 8192),
            "type": rng.choice(("f32", "bf16")), "residual": rng.random() < 0.6}


def work(case):
    m, n, size = case["M"], case["N"], 4 if case["type"] == "f32" else 2
    if case["op"] == "linear":
        k = case["K"]
        each = m * k + n * k + m * n  # x, w, y
        each += (n if case["bias"] else 0) + (m * n if case["residual"] else 0)
        if case["grad"]:  # dy, and the gradients of x, w and the bias
            each += m * n + m * k + n * k + (n if case["bias"] else 0)
        return {"bytes": size * each, "flops": (6 if case["grad"] else 2) * m * n * k}
    if case["op"] == "dropout":
        each = 2 + (1 if case["residual"] else 0) + (2 if case["grad"] else 0)
        return {"bytes": size * m * n * each, "flops": 2 * m * n}
    r = 2 if case["residual"] else 0  # the residual read, the sum written
    if case["pass"] == "send":  # the codes written and read, their values handed out in fp32
        return {"bytes": m * n * (size * (1 + r) + 2 + 4) + 16 * m + size * n, "flops": 8 * m * n}
    if case["pass"] == "forward":
        return {"bytes": size * (m * n * (2 + r) + n), "flops": 4 * m * n}
    # dy, the gradient along the residual stream, dx
    return {"bytes": size * (m * n * (2 + r + 2 + (1 if case["residual"] else 0)) + 2 * n), "flops": 12 * m * n}


# --------------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dev = {"device": "cuda", "generator": gen}
    m, n, kind = case["M"], case["N"], TYPES[case["type"]]
    s = {"case": case, "seed": (seed << 32) | 17, "bias": None, "residual": None}

    def stream(rows, cols):  # a residual stream: rows of different size, a few channels far larger than the others
        x = torch.randn(rows, cols, **dev)
        x *= torch.exp(0.5 * torch.randn(rows, 1, **dev))
        loud = torch.randperm(cols, **dev)[: max(1, cols // 200)]
        x[:, loud] *= 20.0
        return x

    if case["op"] == "linear":
        s["x"] = torch.randn(m, case["K"], **dev).to(kind)
        s["w"] = (torch.randn(n, case["K"], **dev) / math.sqrt(case["K"])).to(kind)
        if case["bias"]:
            s["bias"] = (torch.randn(n, **dev) * 0.1).to(kind)
    else:
        s["x"] = stream(m, n).to(kind)
        s["w"] = (1.0 + 0.2 * torch.randn(n, **dev)).to(kind)
    if case["residual"]:
        s["residual"] = stream(m, n).to(kind)
    if case.get("grad") or case.get("pass") == "train":
        s["dy"] = (torch.randn(m, n, **dev) * 1e-3).to(kind)
        if case["op"] == "norm" and case["residual"]:
            s["dh"] = (torch.randn(m, n, **dev) * 1e-3).to(kind)
    return s


# --------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return {"linear": _linear_own, "dropout": _dropout_own, "norm": _norm_own}[state["case"]["op"]](state)
    return {"linear": _linear_plain, "dropout": _dropout_plain, "norm": _norm_plain}[state["case"]["op"]](state)


def _linear_own(s):
    import paper_2401_07788_gb300 as mpc

    c = s["case"]
    keep = c["grad"] and c["act"] is not None
    y, z = mpc.mpc_linear_forward(s["x"], s["w"], s["bias"], s["residual"], act=c["act"], p=c["p"], seed=s["seed"],
                                  keep=keep)
    if not c["grad"]:
        return {"y": y}
    dx, dw, db = mpc.mpc_linear_backward(s["dy"], s["x"], s["w"], z, act=c["act"], p=c["p"], seed=s["seed"],
                                         need=(True, True, c["bias"]))
    return {"y": y, "dx": dx, "dw": dw} | ({"db": db} if c["bias"] else {})


def _linear_plain(s):
    c = s["case"]
    kind = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if c["bias"]:
        z += s["bias"].float()
    a, slope = _activation(z, c["act"], c["grad"])
    keep = _kept(s["seed"], z.numel(), c["p"], z.device).view(z.shape) if c["p"] else None
    if keep is not None:
        a = a * keep
    y = a if s["residual"] is None else a + s["residual"].float()
    if not c["grad"]:
        return {"y": y.to(kind)}
    dz = s["dy"].float()
    if keep is not None:
        dz = dz * keep
    if slope is not None:
        dz = dz * slope
    out = {"y": y.to(kind), "dx": (dz @ w).to(kind), "dw": (dz.t() @ x).to(kind)}
    if c["bias"]:
        out["db"] = dz.sum(0).to(kind)
    return out


def _activation(z, act, grad):
    """act(z), and act'(z) where the gradient is wanted."""
    if act is None:
        return z, None
    if act == "gelu":
        half = torch.erf(z * math.sqrt(0.5)).add_(1.0).mul_(0.5)
        slope = half + z * torch.exp(z * z * -0.5) * (1.0 / math.sqrt(2.0 * math.pi)) if grad else None
        return z * half, slope
    if act == "gelu_tanh":
        t = torch.tanh((z + z * z * z * 0.044715) * math.sqrt(2.0 / math.pi))
        half = (t + 1.0) * 0.5
        slope = None
        if grad:
            slope = half + z * (1.0 - t * t) * (z * z * (3.0 * 0.044715) + 1.0) * (0.5 * math.sqrt(2.0 / math.pi))
        return z * half, slope
    half = 1.0 / (torch.exp(-z) + 1.0)
    return z * half, (z * (1.0 - half) + 1.0) * half if grad else None


def _signed(x):
    """A 64-bit pattern as the int64 that holds it."""
    x &= (1 << 64) - 1
    return x - (1 << 64) if x >> 63 else x


def _kept(seed, n, p, device):
    """The factor of each of n entries: 0 where it is dropped, else what keeps the mean.  Four entries take the 16-bit
    parts, lowest first, of one splitmix64 output (counter: the entry's number over 4); an entry is dropped where
    its part is below p in 2^-16."""
    step = torch.arange(1, (n + 3) // 4 + 1, dtype=torch.int64, device=device)
    z = step * _signed(0x9E3779B97F4A7C15) + _signed(seed)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    part = z.view(torch.int16)[:n].to(torch.int32) & 0xFFFF
    level = int(math.floor(p * 65536.0 + 0.5))
    return (part >= level).float() * (65536.0 / (65536 - level) if level < 65536 else 0.0)


def _dropout_own(s):
    import paper_2401_07788_gb300 as mpc

    y = mpc.mpc_dropout(s["x"], s["case"]["p"], s["seed"], residual=s["residual"])
    if not s["case"]["grad"]:
        return {"y": y}
    return {"y": y, "dx": mpc.mpc_dropout(s["dy"], s["case"]["p"], s["seed"])}


def _dropout_plain(s):
    x = s["x"].float()
    keep = _kept(s["seed"], x.numel(), s["case"]["p"], x.device).view(x.shape)
    y = x * keep
    if s["residual"] is not None:
        y += s["residual"].float()
    out = {"y": y.to(s["x"].dtype)}
    if s["case"]["grad"]:
        out["dx"] = (s["dy"].float() * keep).to(s["x"].dtype)
    return out


def _norm_own(s):
    import paper_2401_07788_gb300 as mpc

    c = s["case"]
    if c["pass"] == "send":
        codes, scale, minv, h, _ = mpc.mpc_rms_norm_quant(s["x"], s["w"], EPS, residual=s["residual"])
        y = mpc.mpc_quant_decompress(codes, scale, minv, c["N"], 8)
        return {"y": y} | ({"h": h} if c["residual"] else {})
    y, h, rstd = mpc.mpc_rms_norm_forward(s["x"], s["w"], EPS, residual=s["residual"])
    out = {"y": y} | ({"h": h} if c["residual"] else {})
    if c["pass"] == "train":
        out["dx"], out["dw"] = mpc.mpc_rms_norm_backward(s["dy"], h, s["w"], rstd, dh=s.get("dh"))
    return out


def _norm_plain(s):
    c = s["case"]
    kind = s["x"].dtype
    h, w = s["x"].float(), s["w"].float()
    out = {}
    if c["residual"]:
        h = h + s["residual"].float()
        out["h"] = h.to(kind)
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    if c["pass"] == "send":
        # codes are decided on h w: the row's factor scales its range and its values alike
        u = h * w
        low = u.amin(1, keepdim=True)
        span = u.amax(1, keepdim=True) - low
        levels = torch.full_like(span, 255.0)
        code = torch.round((u - low) * (levels / span)).clamp_(0.0, 255.0)
        out["y"] = code * (span / levels * rstd) + low * rstd
        return out
    xhat = h * rstd
    out["y"] = (xhat * w).to(kind)
    if c["pass"] == "train":
        dy = s["dy"].float()
        g = dy * w
        dx = (g - xhat * (g * xhat).mean(1, keepdim=True)) * rstd
        if c["residual"]:
            dx += s["dh"].float()
        out["dx"], out["dw"] = dx.to(kind), (dy * xhat).sum(0).to(kind)
    return out


# --------------------------------------------------------------------------------------------------------
# 64 bits
# --------------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "linear" and work(case)["flops"] > 8e12:
        return None
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    return {"linear": _linear_exact, "dropout": _dropout_exact, "norm": _norm_exact}[case["op"]](case, s["seed"], wide)


def _keep_exact(case, seed):
    """The dropout factors from splitmix64 as published, on the host in unsigned 64-bit numbers."""
    n = case["M"] * case["N"]
    with np.errstate(over="ignore"):
        z = np.uint64(seed & (2 ** 64 - 1)) + (np.arange((n + 3) // 4, dtype=np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z ^= z >> np.uint64(31)
    parts = np.stack([(z >> np.uint64(16 * i)) & np.uint64(0xFFFF) for i in range(4)], axis=1).reshape(-1)[:n]
    level = int(round(case["p"] * 65536))
    kept = torch.from_numpy((parts >= np.uint64(level)).reshape(case["M"], case["N"])).cuda()
    return kept.double() / (1.0 - level / 65536.0)


def _linear_exact(case, seed, s):
    x = s["x"].requires_grad_(case["grad"])
    w = s["w"].requires_grad_(case["grad"])
    z = torch.einsum("mk,nk->mn", x, w)
    leaves = [x, w]
    if case["bias"]:
        b = s["bias"].requires_grad_(case["grad"])
        leaves.append(b)
        z = z + b
    if case["act"] == "gelu":
        a = z * torch.special.ndtr(z)
    elif case["act"] == "gelu_tanh":
        a = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    elif case["act"] == "silu":
        a = z * torch.sigmoid(z)
    else:
        a = z
    if case["p"]:
        a = a * _keep_exact(case, seed)
    y = a + s["residual"] if case["residual"] else a
    out = {"y": y.detach()}
    if case["grad"]:
        grads = torch.autograd.grad(y, leaves, s["dy"])
        out |= dict(zip(("dx", "dw", "db"), grads))
    return out


def _dropout_exact(case, seed, s):
    keep = _keep_exact(case, seed)
    out = {"y": torch.addcmul(s["residual"], s["x"], keep) if case["residual"] else s["x"] * keep}
    if case["grad"]:
        out["dx"] = s["dy"] * keep
    return out


def _norm_exact(case, seed, s):
    x = s["x"].requires_grad_(case["pass"] == "train")
    w = s["w"].requires_grad_(case["pass"] == "train")
    h = x + s["residual"] if case["residual"] else x
    size = torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["N"] + EPS)
    y = h / size * w
    out = {"h": h.detach()} if case["residual"] else {}
    if case["pass"] == "train":
        loss = (y * s["dy"]).sum()
        if case["residual"]:
            loss = loss + (h * s["dh"]).sum()
        out["dx"], out["dw"] = torch.autograd.grad(loss, (x, w))
    if case["pass"] == "send":
        # The codes are those of the library's quantiser, whose rule is one of single fp32 steps, for the fp32 tensor
        # (x + r) w; what they stand for follows in 64 bits.
        f32 = lambda t: t.float().cpu().numpy()  # noqa: E731
        u = f32(x) if not case["residual"] else f32(x) + f32(s["residual"])
        u = u * f32(w)
        low, high = u.min(1, keepdims=True), u.max(1, keepdims=True)
        code = np.rint((u - low) * (np.float32(255.0) / (high - low)))
        low, high, code = (torch.from_numpy(v).cuda().double() for v in (low, high, code))
        y = (low + code.clamp(0.0, 255.0) / 255.0 * (high - low)) / size
    out["y"] = y.detach()
    return out
