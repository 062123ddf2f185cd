"""The AdamW step, its 8-bit states and the gradient norm on the GPU against the formulas in 64 bits.

Tolerances (u = 2^-24): m and v take three roundings of terms of one sign or two, so 4u of
b1|m| + (1-b1)|g| and of b2 v + (1-b2) g^2.  The step's quotient takes v's error halved by the root
and six more roundings, 16u of |m|'s bound over the divisor and of the quotient; param two roundings
of |p| more (2^-8 of the result in bf16).  An 8-bit code may be one off where the value lies within
2^-20 of a midpoint between two codes; otherwise it is the nearest.
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
B1, B2, EPS, LR = 0.9, 0.95, 1e-8, 3e-3


@pytest.fixture(scope="module")
def mpc():
    import __graft_entry__ as g

    g.build()
    import paper_2401_07788_gb300 as m

    torch.cuda.set_device(0)
    return m


def near(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    if bool(bad.any()):
        i = int(bad.nonzero()[0])
        raise AssertionError("%s: %d of %d off, first at %d: got %r want %r tolerance %r" % (
            what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(tol[i])))


def blocks(x):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)


def values(cm, sm, cv, sv):
    n = cm.numel()
    m = blocks(cm.double() / 127.0)
    v = blocks(cv.double() / 255.0)
    return ((m * m.abs() * sm.double()[:, None]).view(-1)[:n], (v ** 4 * sv.double()[:, None]).view(-1)[:n])


def nearest(y, levels):
    """The nearest square (c/levels)^2 to y, and whether y is too near a midpoint to tell."""
    lo = (y.sqrt() * levels).floor().clamp(0, levels - 1)
    mid = (2 * lo * (lo + 1) + 1) / (2 * levels ** 2)
    return torch.where(y >= mid, lo + 1, lo), (y / mid - 1).abs() < 2.0 ** -20


def reference(p, g, m, v, lr, decay, step, clip=1.0):
    g = g.double() * clip
    m0, v0 = m.double(), v.double()
    m1, v1 = B1 * m0 + (1 - B1) * g, B2 * v0 + (1 - B2) * g * g
    am = B1 * m0.abs() + (1 - B1) * g.abs()
    under = (v1 / (1 - B2 ** step)).sqrt() + EPS
    rate = lr / (1 - B1 ** step)
    p1 = p.double() * (1 - lr * decay) - rate * m1 / under
    ep = 4 * U * p.double().abs() + rate * am / under * 16 * U + 1e-37
    return m1, 4 * U * am + 1e-40, v1, 8 * U * v1 + 1e-40, p1, ep


def tensors(sizes, ptype, gtype, bits, seed=0, offset=0, zero=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def made(n, dtype, fn):
        big = torch.full((n + offset + 5,), 3, device="cuda").to(dtype)
        x = big[offset:offset + n]
        x.copy_(fn(n))
        return big, x

    def normal(s):
        return lambda n: torch.randn(n, device="cuda", generator=gen) * s * torch.exp(
            2 * torch.randn(n, device="cuda", generator=gen))

    out = []
    for n in sizes:
        t = {"p": made(n, ptype, normal(0.02)), "g": made(n, gtype, normal(1e-3))}
        if bits == 32:
            t["m"] = made(n, torch.float32, normal(0.0 if zero else 3e-4))
            t["v"] = made(n, torch.float32, lambda k: (torch.randn(k, device="cuda", generator=gen) * (0.0 if zero else 1e-3)) ** 2)
        else:
            k = -(-n // 256)
            t["m"] = made(n, torch.int8, lambda k: torch.randint(-127, 128, (k,), device="cuda", generator=gen) * (not zero))
            t["v"] = made(n, torch.uint8, lambda k: torch.randint(0, 256, (k,), device="cuda", generator=gen) * (not zero))
            t["sm"] = made(k, torch.float32, lambda k: torch.rand(k, device="cuda", generator=gen) * (0.0 if zero else 1e-3))
            t["sv"] = made(k, torch.float32, lambda k: torch.rand(k, device="cuda", generator=gen) * (0.0 if zero else 1e-6))
        t["c"] = made(n, torch.bfloat16, lambda k: torch.zeros(k, device="cuda"))
        out.append(t)
    return out


def plan_of(mpc, ts, copies=None, decay=0.0, bits=32):
    view = lambda k: [t[k][1] for t in ts]  # noqa: E731
    low = {"m_scale": view("sm"), "v_scale": view("sv")} if bits == 8 else {}
    return mpc.AdamWPlan(view("p"), view("g"), view("m"), view("v"), copies=copies, weight_decay=decay, **low)


SIZES = [1, 7, 8, 255, 256, 257, 2047, 2048, 2049, 4096, 0, 5000, 70001]
TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16),
         (torch.bfloat16, torch.float32)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype", TYPES)
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("zero", [False, True], ids=["warm", "cold"])
def test_step_against_64_bits(mpc, bits, ptype, gtype, offset, zero):
    ts = tensors(SIZES, ptype, gtype, bits, offset=offset, zero=zero)
    decay = [0.1 * (i % 3) for i in range(len(ts))]
    copies = [t["c"][1] if i % 2 else None for i, t in enumerate(ts)]
    step = 1 if zero else 37
    wants = []
    for t, d in zip(ts, decay):
        m, v = (t["m"][1], t["v"][1]) if bits == 32 else values(t["m"][1], t["sm"][1], t["v"][1], t["sv"][1])
        wants.append(reference(t["p"][1], t["g"][1], m.float() if bits == 8 else m, v.float() if bits == 8 else v, LR, d, step))
    plan = plan_of(mpc, ts, copies, decay, bits)
    mpc.mpc_adamw_step(plan, LR, B1, B2, EPS, step)
    if bits == 8:
        outs = [[torch.empty(t["p"][1].numel(), device="cuda") for t in ts] for _ in range(2)]
        mpc.mpc_adamw_decode(plan, *outs)
    for i, (t, (m, em, v, ev, p, ep)) in enumerate(zip(ts, wants)):
        low = 2.0 ** -8 * p.abs()
        near(t["p"][1], p, ep + low if ptype == torch.bfloat16 else ep, "param %d" % i)
        if copies[i] is not None:
            near(copies[i], p, ep + low, "copy %d" % i)
        if bits == 32:
            near(t["m"][1], m, em, "m %d" % i)
            near(t["v"][1], v, ev, "v %d" % i)
        elif m.numel():
            n = m.numel()
            bm, bv = blocks(m), blocks(v)
            tm, tv = bm.abs().amax(1), bv.amax(1)
            near(t["sm"][1], tm, 8 * U * tm + blocks(em).amax(1), "scale of m %d" % i)
            near(t["sv"][1], tv, 16 * U * tv + 1e-40, "scale of v %d" % i)
            cm, nm = nearest((bm.abs() / tm.clamp_min(1e-300)[:, None]), 127)
            cm = (cm * bm.sign()).view(-1)[:n]
            cv, nv = nearest((bv / tv.clamp_min(1e-300)[:, None]).sqrt(), 255)
            cv = torch.where(bv > 0, cv.clamp_min(1), cv).view(-1)[:n]
            # m's relative error grows where b1 m and (1-b1) g cancel: those codes are as good as em
            slack = (blocks(em) / tm.clamp_min(1e-300)[:, None] > 2.0 ** -22 * (bm.abs() / tm.clamp_min(1e-300)[:, None])).view(-1)[:n]
            off = (t["m"][1].double() - cm).abs()
            assert bool(((off == 0) | ((nm.view(-1)[:n] | slack) & (off <= 1))).all()), "codes of m %d" % i
            off = (t["v"][1].double() - cv).abs()
            assert bool(((off == 0) | (nv.view(-1)[:n] & (off <= 1))).all()), "codes of v %d" % i
            dm, dv = values(t["m"][1], t["sm"][1], t["v"][1], t["sv"][1])
            near(outs[0][i], dm, 8 * U * dm.abs() + 1e-44, "decoded m %d" % i)
            near(outs[1][i], dv, 8 * U * dv.abs() + 1e-44, "decoded v %d" % i)
        for name, (big, x) in t.items():  # what lies around each tensor
            if name != "c" or copies[i] is not None:
                assert bool((big[:offset] == 3).all()) and bool((big[offset + x.numel():] == 3).all()), name
    assert mpc.mpc_get_status() == 0


@pytest.mark.parametrize("count", [47, 49, 401, 1700])
def test_long_lists(mpc, count):
    """Lists that take the short and the long table, several tables and several batches."""
    sizes = [(37 * i) % 301 for i in range(count)]
    ts = tensors(sizes, torch.float32, torch.float32, 32, seed=count)
    wants = [reference(t["p"][1], t["g"][1], t["m"][1], t["v"][1], LR, 0.1, 5) for t in ts]
    total = sum(float(t["g"][1].double().square().sum()) for t in ts)
    plan = plan_of(mpc, ts, decay=0.1)
    norm = mpc.mpc_grad_norm(plan)
    assert abs(float(norm) - math.sqrt(total)) <= 1e-6 * math.sqrt(total)
    mpc.mpc_adamw_step(plan, LR, B1, B2, EPS, 5)
    for i, (t, (m, em, v, ev, p, ep)) in enumerate(zip(ts, wants)):
        near(t["p"][1], p, ep, "param %d" % i)
        near(t["m"][1], m, em, "m %d" % i)
        near(t["v"][1], v, ev, "v %d" % i)


def test_small_second_moments_keep_a_code(mpc):
    """A v far below its block's largest must not become 0: the step would divide by eps."""
    g = torch.full((512,), 1e-6, device="cuda")
    g[0] = 1.0
    g[256:] = 0.0
    p = torch.zeros(512, device="cuda")
    plan = mpc.AdamWPlan([p], [g], state_bits=8)
    mpc.mpc_adamw_step(plan, 1e-3, 0.9, 0.999, 1e-12, 1)
    assert int(plan.v[0][:256].min()) >= 1 and not plan.v[0][256:].any()
    g.zero_()
    before = p.clone()
    mpc.mpc_adamw_step(plan, 1e-3, 0.9, 0.999, 1e-12, 2)
    assert float((p - before).abs().max()) <= 1.1e-3


def test_blocks_of_tiny_and_equal_values(mpc):
    """A block below the normal range codes as zero; a block of equal values as its largest code."""
    g = torch.full((768,), 1e-30, device="cuda")
    g[256:512] = 0.5
    g[512:] = -0.5
    plan = mpc.AdamWPlan([torch.zeros(768, device="cuda")], [g], state_bits=8)
    mpc.mpc_adamw_step(plan, 1e-3, B1, B2, EPS, 1)
    assert not plan.v[0][:256].any()
    assert bool((plan.m[0][256:512] == 127).all()) and bool((plan.m[0][512:] == -127).all())
    assert bool((plan.v[0][256:] == 255).all())


@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [1.0, 1e-6, 0.0])
def test_norm_and_clip(mpc, gtype, scale):
    ts = tensors([5, 300, 0, 40001, 1], torch.float32, gtype, 32, seed=4)
    for t in ts:
        t["g"][1].mul_(scale * 100)
    total = math.sqrt(sum(float(t["g"][1].double().square().sum()) for t in ts))
    plan = plan_of(mpc, ts)
    norm = mpc.mpc_grad_norm(plan)
    # a thread sums at most 8 squares and its groups of 8 in fp32: 2^-20 leaves room for 16 roundings
    assert abs(float(norm) - total) <= 2.0 ** -20 * total
    clip = min(1.0, 0.5 / (total + 1e-6))
    wants = [reference(t["p"][1], t["g"][1], t["m"][1], t["v"][1], LR, 0.0, 9, clip) for t in ts]
    mpc.mpc_adamw_step(plan, LR, B1, B2, EPS, 9, grad_norm=norm, max_norm=0.5)
    for i, (t, (m, em, v, ev, p, ep)) in enumerate(zip(ts, wants)):
        # the clip factor's own error (norm, sum, quotient) comes on top, times two in v
        near(t["m"][1], m, em + 2.0 ** -19 * m.abs() + 2.0 ** -19 * (1 - B1) * clip * t["g"][1].double().abs(), "m %d" % i)
        near(t["v"][1], v, ev + 2.0 ** -18 * v, "v %d" % i)
        near(t["p"][1], p, ep + 2.0 ** -17 * LR * 10, "param %d" % i)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_norm_that_is_not_finite_skips_the_step(mpc, bad, bits):
    ts = tensors([300, 5000], torch.float32, torch.float32, bits, seed=5)
    ts[1]["g"][1][77] = bad
    before = [{k: x.clone() for k, (_, x) in t.items()} for t in ts]
    plan = plan_of(mpc, ts, bits=bits)
    norm = mpc.mpc_grad_norm(plan)
    assert not math.isfinite(float(norm))
    mpc.mpc_adamw_step(plan, LR, B1, B2, EPS, 3, grad_norm=norm, max_norm=1.0)
    for t, b in zip(ts, before):
        for k, x in b.items():
            if k != "g":
                assert torch.equal(t[k][1], x), k


def test_results_repeat_on_any_stream_and_in_a_graph(mpc):
    runs = []
    for mode in range(3):
        ts = tensors(SIZES, torch.float32, torch.float32, 8, seed=6)
        plan = plan_of(mpc, ts, decay=0.1, bits=8)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        if mode == 0:
            norm = mpc.mpc_grad_norm(plan)
            mpc.mpc_adamw_step(plan, LR, B1, B2, EPS, 4, grad_norm=norm, max_norm=0.1)
        elif mode == 1:
            norm = mpc.mpc_grad_norm(plan, stream=side)
            mpc.mpc_adamw_step(plan, LR, B1, B2, EPS, 4, grad_norm=norm, max_norm=0.1, stream=side)
        else:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                norm = mpc.mpc_grad_norm(plan)
                mpc.mpc_adamw_step(plan, LR, B1, B2, EPS, 4, grad_norm=norm, max_norm=0.1)
            g.replay()
        torch.cuda.synchronize()
        runs.append([norm] + [t[k][1] for t in ts for k in ("p", "m", "v", "sm", "sv")])
    for a, b, c in zip(*runs):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer(mpc, bits):
    """Against torch's AdamW in 64 bits over a few steps (fp32 states), clipped, in two groups; a
    saved and restored optimizer continues bit for bit."""
    torch.manual_seed(0)
    made = [torch.randn(33, 65, device="cuda"), torch.randn(65, device="cuda"), torch.randn(700, device="cuda")]

    def build():
        ps = [torch.nn.Parameter(x.clone()) for x in made]
        copies = {ps[0]: torch.empty(33, 65, dtype=torch.bfloat16, device="cuda")}
        opt = mpc.AdamW([{"params": ps[:1], "weight_decay": 0.1}, {"params": ps[1:], "weight_decay": 0.0, "lr": 2e-3}],
                        lr=1e-3, betas=(B1, B2), state_bits=bits, max_norm=1.0, copies=copies)
        return ps, opt, copies

    ps, opt, copies = build()
    ref = [torch.nn.Parameter(x.double()) for x in made]
    ropt = torch.optim.AdamW([{"params": ref[:1], "weight_decay": 0.1}, {"params": ref[1:], "weight_decay": 0.0, "lr": 2e-3}],
                             lr=1e-3, betas=(B1, B2))
    grads = [[torch.randn_like(x) * (k + 1) for x in made] for k in range(6)]

    def advance(ps, opt, k):
        for i, p in enumerate(ps):
            p.grad = None if (i == 2 and k == 3) else grads[k][i].to(p.dtype).clone()
        opt.step()

    saved = None
    for k in range(6):
        if k == 4:
            saved = ([p.detach().clone() for p in ps], opt.state_dict())
            saved = (saved[0], torch.utils._pytree.tree_map(lambda x: x.clone() if isinstance(x, torch.Tensor) else x, saved[1]))
        advance(ps, opt, k)
        for i, p in enumerate(ref):
            p.grad = None if (i == 2 and k == 3) else grads[k][i].double()
        torch.nn.utils.clip_grad_norm_([p for p in ref if p.grad is not None], 1.0)
        ropt.step()
    if bits == 32:
        for a, b in zip(ps, ref):
            assert float((a.detach().double() - b.detach()).abs().max()) < 1e-6
    else:
        for a, b in zip(ps, ref):  # coded states: the same descent, to a few per cent of its length
            moved = (b.detach() - a.detach().double()).norm() / (b.detach() - made[[33 * 65, 65, 700].index(b.numel())].double()).norm()
            assert float(moved) < 0.1
    assert torch.equal(copies[ps[0]], ps[0].detach().bfloat16())
    qs, opt2, _ = build()
    with torch.no_grad():
        for q, x in zip(qs, saved[0]):
            q.copy_(x)
    opt2.load_state_dict(saved[1])
    for k in (4, 5):
        advance(qs, opt2, k)
    for p, q in zip(ps, qs):
        assert torch.equal(p, q)
