"""Measured cases of the training operators: the linear cross entropy of a last stage, and the AdamW step
(with the gradient norm it clips by) of any stage."""

import math
import random

import torch

own = False  # False: plain torch operations; True: the calls a user makes of the package

BLOCK = 256  # entries that share a scale in the 8-bit states
LR, B1, B2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one position scored against a 50257-entry vocabulary: a serving call, where latency counts
        {"name": "ce_score_1", "op": "ce", "grad": False, "T": 1, "D": 768, "V": 50257, "type": "bf16",
         "ignored": 0.0, "weights": False},
        # evaluation loss of a ragged batch in fp32
        {"name": "ce_eval_f32", "op": "ce", "grad": False, "T": 1000, "D": 768, "V": 50257, "type": "f32",
         "ignored": 0.2, "weights": False},
        # a small odd head (character or byte-pair vocabulary, width not a multiple of a tile), weighted tokens
        {"name": "ce_train_odd_f32", "op": "ce", "grad": True, "T": 129, "D": 203, "V": 5003, "type": "f32",
         "ignored": 0.1, "weights": True},
        # fine-tuning, batch 8 of 1024 tokens, hidden width 768, some positions padded
        {"name": "ce_train_768", "op": "ce", "grad": True, "T": 8192, "D": 768, "V": 50257, "type": "bf16",
         "ignored": 0.1, "weights": False},
        # the same head in the fp32 that the boundaries exchange, two sequences
        {"name": "ce_train_768_f32", "op": "ce", "grad": True, "T": 2048, "D": 768, "V": 50257, "type": "f32",
         "ignored": 0.0, "weights": False},
        # the largest head: wide hidden states, a 131072-entry vocabulary
        {"name": "ce_train_4096", "op": "ce", "grad": True, "T": 8192, "D": 4096, "V": 131072, "type": "bf16",
         "ignored": 0.0, "weights": False},
        # a handful of small tensors: a launch-bound step with clipping
        {"name": "adamw32_small_clip", "op": "adamw", "bits": 32, "count": 16, "largest": 5000, "param": "f32",
         "grad": "f32", "copy": False, "clip": True},
        # a whole stage in fp32 with clipping: eight layers of width 1024 and the embedding
        {"name": "adamw32_stage_clip", "op": "adamw", "bits": 32, "width": 1024, "layers": 8, "vocab": 50257,
         "param": "f32", "grad": "f32", "copy": False, "clip": True},
        # bf16 weights and gradients without a master copy, ragged tensors
        {"name": "adamw32_bf16", "op": "adamw", "bits": 32, "count": 60, "largest": 4000003, "param": "bf16",
         "grad": "bf16", "copy": False, "clip": False},
        # the stage with 8-bit states, bf16 gradients and a bf16 copy of the weights for the next forward pass
        {"name": "adamw8_stage", "op": "adamw", "bits": 8, "width": 1024, "layers": 8, "vocab": 50257,
         "param": "f32", "grad": "bf16", "copy": True, "clip": False},
        # ragged tensors with 8-bit states
        {"name": "adamw8_ragged", "op": "adamw", "bits": 8, "count": 40, "largest": 300007, "param": "f32",
         "grad": "f32", "copy": False, "clip": False},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))

    if rng.random() < 0.55:
        return {"op": "ce", "grad": rng.random() < 0.6, "T": log(1, 8192), "D": log(32, 4096),
                "V": log(500, 131072), "type": rng.choice(("f32", "bf16")),
                "ignored": rng.choice((0.0, 0.1, 0.5)), "weights": rng.random() < 0.3}
    bits = rng.choice((32, 8))
    param = rng.choice(("f32", "bf16"))
    case = {"op": "adamw", "bits": bits, "param": param, "grad": rng.choice(("f32", "bf16")),
            "copy": param == "f32" and rng.random() < 0.5, "clip": bits == 32 and rng.random() < 0.5}
    if rng.random() < 0.5:
        case.update(width=rng.choice((64, 128, 192, 320, 512, 640, 896, 1024)), layers=rng.randint(1, 8), vocab=log(500, 50257))
    else:
        case.update(count=rng.randint(1, 100), largest=log(10, 1000000))
    return case


# --------------------------------------------------------------------------------------------------------
# shapes
# --------------------------------------------------------------------------------------------------------

def _tensors(case):
    """(entries, decayed) of each tensor of an optimiser case."""
    if "width" in case:
        d = case["width"]
        layer = [(d, False), (d, False)] + [(d * d, True), (d, False)] * 4 + [(d, False), (d, False)]
        layer += [(4 * d * d, True), (4 * d, False), (4 * d * d, True), (d, False)]
        return [(case["vocab"] * d, True), (1024 * d, True)] + layer * case["layers"] + [(d, False), (d, False)]
    rng = random.Random(case["count"] * 1000003 + case["largest"])
    sizes = [max(1, int(math.exp(rng.uniform(0.0, math.log(case["largest"]))))) for _ in range(case["count"] - 1)]
    return [(n, i % 3 != 0) for i, n in enumerate(sizes + [case["largest"]])]


def _valid(case):
    return case["T"] - int(case["ignored"] * case["T"])


def work(case):
    if case["op"] == "ce":
        size = 4 if case["type"] == "f32" else 2
        t, d, v, n = case["T"], case["D"], case["V"], _valid(case)
        dense = size * d * (n + v)
        if not case["grad"]:
            return {"bytes": dense + 16 * t, "flops": 2 * n * d * v}
        return {"bytes": dense + size * d * (t + v) + 16 * t, "flops": 6 * n * d * v}
    n = sum(k for k, _ in _tensors(case))
    each = 2 * (4 if case["param"] == "f32" else 2) + (4 if case["grad"] == "f32" else 2) + (2 if case["copy"] else 0)
    # 8-bit states: codes read and written, then read once more for the values that are handed out in fp32
    each += 16 if case["bits"] == 32 else 4 + 2 + 8
    return {"bytes": n * each + (n * (4 if case["grad"] == "f32" else 2) if case["clip"] else 0), "flops": 15 * n}


# --------------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return _prepare_ce(case, gen) if case["op"] == "ce" else _prepare_adamw(case, gen)


def _prepare_ce(case, gen):
    T, D, V = case["T"], case["D"], case["V"]
    dev = {"device": "cuda", "generator": gen}
    # word frequencies fall off as a power law; hidden states partly predict their target
    targets = (torch.exp(torch.rand(T, **dev) * math.log(V)) - 1).long().clamp(0, V - 1)
    w = torch.randn(V, D, **dev) * (0.55 / math.sqrt(D))
    h = torch.randn(T, D, **dev)
    wt = w[targets]
    h += torch.rand(T, 1, **dev) * 12.0 * wt / wt.square().sum(1, keepdim=True).clamp_min(1e-6)
    gone = torch.randperm(T, **dev)[: T - _valid(case)]
    targets[gone] = -100
    h[gone] = float("nan")  # padding positions hold whatever the model left there
    s = {"case": case, "h": h.to(TYPES[case["type"]]), "w": w.to(TYPES[case["type"]]), "targets": targets,
         "weights": None}
    if case["weights"]:
        s["weights"] = (0.5 + torch.rand(T, **dev)) / T
    return s


def _prepare_adamw(case, gen):
    dev = {"device": "cuda", "generator": gen}
    sizes = _tensors(case)
    padded = [-(-n // BLOCK) * BLOCK for n, _ in sizes]
    starts = [0]
    for k in padded:
        starts.append(starts[-1] + k)
    N = starts[-1]
    inside = torch.zeros(N, dtype=torch.bool, device="cuda")
    for a, (n, _) in zip(starts, sizes):
        inside[a:a + n] = True
    param = (torch.randn(N, **dev) * 0.02 * inside).to(TYPES[case["param"]])
    # gradients of one tensor differ by orders of magnitude between its rows
    spread = torch.exp(torch.randn(N // BLOCK, 1, **dev) * 1.5) * 1e-4
    grad = ((torch.randn(N // BLOCK, BLOCK, **dev) * spread).view(N) * inside).to(TYPES[case["grad"]])
    m = torch.randn(N // BLOCK, BLOCK, **dev) * spread * 0.3 * inside.view(-1, BLOCK)
    v = (torch.rand(N // BLOCK, BLOCK, **dev) + 0.05) * spread.square() * inside.view(-1, BLOCK)
    s = {"case": case, "t": 100, "sizes": [n for n, _ in sizes], "starts": starts, "param": param, "grad": grad,
         "decay": [DECAY if d else 0.0 for _, d in sizes]}
    if case["copy"]:
        s["copy"] = torch.zeros(N, dtype=torch.bfloat16, device="cuda")
    if case["bits"] == 32:
        s["m"], s["v"] = m.view(N), v.view(N)
    else:
        s["m"], s["m_scale"], s["v"], s["v_scale"] = _encode(m, v)
        s["m_out"], s["v_out"] = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    keep = torch.tensor([1.0 - LR * d for d in s["decay"]], dtype=torch.float64).float()
    s["keep"] = keep.repeat_interleave(torch.tensor(padded) // BLOCK).cuda().view(-1, 1)
    if own:
        import paper_2401_07788_gb300 as mpc

        def views(x, blocks=False):
            return [x[a // BLOCK:a // BLOCK - (-n // BLOCK)] if blocks else x[a:a + n]
                    for a, n in zip(starts, s["sizes"])]

        low = {} if case["bits"] == 32 else {"m_scale": views(s["m_scale"], True), "v_scale": views(s["v_scale"], True)}
        s["plan"] = mpc.AdamWPlan(views(param), views(grad), views(s["m"]), views(s["v"]),
                                  copies=views(s["copy"]) if case["copy"] else None,
                                  weight_decay=s["decay"], **low)
        if case["bits"] == 8:
            s["m_views"], s["v_views"] = views(s["m_out"]), views(s["v_out"])
    return s


# --------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------

def run(state):
    if state["case"]["op"] == "ce":
        return _ce_own(state) if own else _ce_plain(state)
    return _adamw_own(state) if own else _adamw_plain(state)


def _ce_own(s):
    import paper_2401_07788_gb300 as mpc

    if not s["case"]["grad"]:
        loss, lse = mpc.mpc_linear_ce_forward(s["h"], s["w"], s["targets"])
        return {"loss": loss, "lse": lse}
    loss, dh, dw = mpc.mpc_linear_ce_train(s["h"], s["w"], s["targets"], s["weights"])
    return {"loss": loss, "dh": dh, "dw": dw}


def _ce_plain(s):
    valid = s["targets"] >= 0
    h = s["h"].float().masked_fill_(~valid[:, None], 0.0) if s["h"].dtype != torch.float32 else \
        s["h"].masked_fill(~valid[:, None], 0.0)
    w = s["w"].float()
    at = s["targets"].clamp_min(0)[:, None]
    logits = h @ w.t()
    top = logits.max(1, keepdim=True).values
    target = logits.gather(1, at)
    e = logits.sub_(top).exp_()
    z = e.sum(1, keepdim=True)
    lse = top + z.log()
    loss = ((lse - target)[:, 0]).masked_fill(~valid, 0.0)
    if not s["case"]["grad"]:
        return {"loss": loss, "lse": lse[:, 0].masked_fill(~valid, 0.0)}
    g = valid / valid.sum() if s["weights"] is None else s["weights"] * valid
    c = e.div_(z)
    c.scatter_add_(1, at, torch.full_like(z, -1.0))
    c.mul_(g[:, None])
    return {"loss": loss, "dh": (c @ w).to(s["h"].dtype), "dw": (c.t() @ h).to(s["w"].dtype)}


def _adamw_own(s):
    import paper_2401_07788_gb300 as mpc

    s["t"] += 1
    norm = mpc.mpc_grad_norm(s["plan"]) if s["case"]["clip"] else None
    mpc.mpc_adamw_step(s["plan"], LR, B1, B2, EPS, s["t"], grad_norm=norm, max_norm=1.0)
    if s["case"]["bits"] == 8:
        mpc.mpc_adamw_decode(s["plan"], s["m_views"], s["v_views"])
    return _adamw_outputs(s, norm)


def _adamw_outputs(s, norm):
    out = {"param": s["param"], "m": s["m"], "v": s["v"]}
    if s["case"]["bits"] == 8:
        out["m"], out["v"] = s["m_out"], s["v_out"]
    if norm is not None:
        out["norm"] = norm
    if s["case"]["copy"]:
        out["copy"] = s["copy"]
    return out


def _adamw_plain(s):
    s["t"] += 1
    low = s["case"]["bits"] == 8
    g = s["grad"].float().view(-1, BLOCK)
    norm = None
    if s["case"]["clip"]:
        norm = g.square().sum().sqrt().view(1)
        g = g * (1.0 / (norm + 1e-6)).clamp_max(1.0)
    if low:
        m, v = _decode(s["m"], s["m_scale"], s["v"], s["v_scale"])
    else:
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    m.mul_(B1).add_(g * (1.0 - B1))
    v.mul_(B2).add_((g * (1.0 - B2)).mul_(g))
    step = LR / (1.0 - B1 ** s["t"])
    under = v.sqrt().mul_(1.0 / math.sqrt(1.0 - B2 ** s["t"])).add_(EPS)
    p = s["param"].float().view(-1, BLOCK) * s["keep"]
    p.sub_(m.div(under).mul_(step))
    s["param"].copy_(p.view(-1))
    if s["case"]["copy"]:
        s["copy"].copy_(p.view(-1))
    if low:
        for name, x in zip(("m", "m_scale", "v", "v_scale"), _encode(m, v)):
            s[name].copy_(x)
        m, v = _decode(s["m"], s["m_scale"], s["v"], s["v_scale"])
        s["m_out"].copy_(m.view(-1))
        s["v_out"].copy_(v.view(-1))
    return _adamw_outputs(s, norm)


# The 8-bit states: m of a block as sign(c) (c/127)^2 s, v as (c/255)^4 s, s the block's largest; the code is the
# number of midpoints (of m/s, and of the square root of v/s) at or below the value.

def _midpoints(levels, device):
    c = torch.arange(1, levels + 1, dtype=torch.float32, device=device)
    return (2.0 * c * (c - 1.0) + 1.0) * (1.0 / (2.0 * levels * levels))


def _inverse(top):
    return torch.where(top < 2.0 ** -126, torch.zeros_like(top), 1.0 / top)


def _encode(m, v):
    top_m, top_v = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True)
    y = m.abs() * _inverse(top_m)
    code = torch.bucketize(y, _midpoints(127, m.device), right=True)
    cm = torch.where(m < 0, -code, code).to(torch.int8)
    y = v * _inverse(top_v)
    cv = torch.bucketize(y, _midpoints(255, m.device).square(), right=True)
    cv = torch.maximum(cv, (y > 0).to(cv.dtype)).to(torch.uint8)
    return cm.view(-1), top_m.view(-1), cv.view(-1), top_v.view(-1)


def _decode(cm, sm, cv, sv):
    c = cm.view(-1, BLOCK).float()
    m = (c * c.abs()).mul_(1.0 / 127.0 ** 2).mul_(sm.view(-1, 1))
    c = cv.view(-1, BLOCK).float()
    c = c * c
    return m, (c * c).mul_(1.0 / 255.0 ** 4).mul_(sv.view(-1, 1))


# --------------------------------------------------------------------------------------------------------
# 64 bits
# --------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _ce_exact(s) if case["op"] == "ce" else _adamw_exact(s)


def _ce_exact(s):
    case = s["case"]
    if work(case)["flops"] > 8e12:
        return None
    rows = (s["targets"] != -100).nonzero()[:, 0]
    T, D = s["h"].shape
    h = s["h"][rows].double().requires_grad_(case["grad"])
    w = s["w"].double().requires_grad_(case["grad"])
    y = s["targets"][rows]
    logits = torch.einsum("td,vd->tv", h, w)
    lse = torch.logsumexp(logits, 1)
    loss = lse - logits[torch.arange(len(rows), device=y.device), y]

    def whole(x):
        out = torch.zeros((T,) + x.shape[1:], dtype=torch.float64, device=x.device)
        out[rows] = x.detach()
        return out

    if not case["grad"]:
        return {"loss": whole(loss), "lse": whole(lse)}
    weights = torch.full_like(loss, 1.0 / max(1, len(rows))) if s["weights"] is None else s["weights"][rows].double()
    dh, dw = torch.autograd.grad((loss * weights).sum(), (h, w))
    return {"loss": whole(loss), "dh": whole(dh), "dw": dw}


def _adamw_exact(s):
    t = s["t"] + 1
    low = s["case"]["bits"] == 8
    rows = lambda x: x.double().view(-1, BLOCK)  # noqa: E731
    g, p = rows(s["grad"]), rows(s["param"])
    out = {}
    if s["case"]["clip"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = norm.view(1)
        g = g * min(1.0, 1.0 / (float(norm) + 1e-6))
    if low:
        c, k = rows(s["m"]) / 127.0, rows(s["v"]) / 255.0
        m, v = c.sign() * c ** 2 * s["m_scale"].double().view(-1, 1), k ** 4 * s["v_scale"].double().view(-1, 1)
    else:
        m, v = rows(s["m"]), rows(s["v"])
    m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g ** 2
    keep = torch.cat([torch.full(((n + BLOCK - 1) // BLOCK, 1), 1.0 - LR * d, dtype=torch.float64)
                      for n, d in zip(s["sizes"], s["decay"])]).cuda()
    p = p * keep - LR * (m / (1 - B1 ** t)) / ((v / (1 - B2 ** t)).sqrt() + EPS)
    out["param"] = p.view(-1)
    if s["case"]["copy"]:
        out["copy"] = p.view(-1)
    if low:
        # nearest of the 128 squares (m) and, in the square root, of the 256 squares (v), without ties
        a = m.abs() / m.abs().amax(1, keepdim=True).clamp_min(1e-300)
        lo = (a.sqrt() * 127.0).floor().clamp_max(126.0)
        c = torch.where(a * 127.0 ** 2 - lo ** 2 < (lo + 1) ** 2 - a * 127.0 ** 2, lo, lo + 1)
        m = m.sign() * (c / 127.0) ** 2 * m.abs().amax(1, keepdim=True)
        a = (v / v.amax(1, keepdim=True).clamp_min(1e-300)).sqrt()
        lo = (a.sqrt() * 255.0).floor().clamp_max(254.0)
        c = torch.where(a * 255.0 ** 2 - lo ** 2 < (lo + 1) ** 2 - a * 255.0 ** 2, lo, lo + 1)
        c = torch.where(v > 0, c.clamp_min(1.0), c)
        v = (c / 255.0) ** 4 * v.amax(1, keepdim=True)
    out["m"], out["v"] = m.view(-1), v.view(-1)
    return out
