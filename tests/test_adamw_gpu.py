"""resbm_adamw_step and resbm_grad_norm against their definitions in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, half a step of fp32 relative to the value). m: two products and a sum, and the
rounded coefficients: 6 u of |b1 m| + |(1 - b1) g|; v: one product more, all terms positive: 8 u of v. The new weight: the
decay 3 u of |w|, the quotient 16 u of |update| beside what m's error makes of it, and the weight's own rounding (half a
step of its type). With 8-bit states the scale has the error of the block's largest value and two roundings, and a code is
off by half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below 2^-6 of it). A norm: squares in fp32 over at most
8 x 4 elements a thread (all positive: 33 u), the rest in 64 bits; the root halves it, two roundings more."""
import pytest
import torch

from paper_2604_11947_gb300 import resbm

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
U = 2.0 ** -24
B = resbm.RESBM_STATE_BLOCK
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = [1, 7, 255, 256, 257, 1000, 2048, 2049, 4096, 70001]


def model(sizes, w="bf16", g="bf16", bits=32, master=False, seed=0, offset=0, warm=True):
    """A list of tensors in the states that a step meets (warm) or before the first (zeros), each behind `offset` elements."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda n: torch.randn(n, generator=gen, device="cuda")

    def put(x, dtype):
        buf = torch.full((offset + x.numel() + 9,), 77.0, device="cuda").to(dtype)
        t = buf[offset:offset + x.numel()]
        t.copy_(x)
        return t

    s = {k: [] for k in ("w", "g", "m", "v", "m_scale", "v_scale", "master")}
    for n in sizes:
        x, size = 0.05 * rnd(n), torch.exp(2 * rnd(1))
        s["w"].append(put(x, DT[w]))
        s["master"].append(put(x, torch.float32))
        s["g"].append(put(1e-3 * size * rnd(n), DT[g]))
        m, v = (3e-4 * size * rnd(n), (1e-3 * size * (rnd(n).abs() + 0.1)) ** 2) if warm else (torch.zeros(n, device="cuda"),) * 2
        if bits == 32:
            s["m"].append(put(m, torch.float32))
            s["v"].append(put(v, torch.float32))
        else:
            for k, y in (("m", m), ("v", v.sqrt())):
                blocks = torch.nn.functional.pad(y, (0, -n % B)).view(-1, B)
                scale = blocks.abs().amax(dim=1) / 448
                code = (blocks / scale.clamp_min(1e-30)[:, None]).clamp(-448, 448).to(E4M3).view(-1)[:n]
                s[k].append(put(code.float(), E4M3))
                s[k + "_scale"].append(put(scale, torch.float32))
    if bits == 32:
        s["m_scale"] = s["v_scale"] = None
    if not master:
        s["master"] = None
    return s


def plan_of(s):
    return resbm.AdamWPlan(s["w"], s["g"], s["m"], s["v"], s["m_scale"], s["v_scale"], s["master"])


def copy_of(s):
    return {k: None if x is None else [t.clone() for t in x] for k, x in s.items()}


def wide(s, k, i):
    x = s[k][i].double()
    if s[k + "_scale"] is not None:
        x = x * s[k + "_scale"][i].double().repeat_interleave(B)[:x.numel()]
    return x


def expect(s, i, t, h=HYPER, c=1.0):
    """New w, m, v of tensor i in 64 bits, and how far fp32 may be off"""
    g = s["g"][i].double() * c
    m0, v0 = wide(s, "m", i), wide(s, "v", i)
    if s["m_scale"] is not None:
        v0 = v0 * v0
    m, v = h["beta1"] * m0 + (1 - h["beta1"]) * g, h["beta2"] * v0 + (1 - h["beta2"]) * g * g
    me = 6 * U * ((h["beta1"] * m0).abs() + ((1 - h["beta1"]) * g).abs())
    w0 = (s["master"] or s["w"])[i].double()
    step = h["lr"] / (1 - h["beta1"] ** t)
    denom = (v / (1 - h["beta2"] ** t)).sqrt() + h["eps"]
    update = step * m / denom
    w = w0 * (1 - h["lr"] * h["weight_decay"]) - update
    we = 4 * U * w0.abs() + 16 * U * update.abs() + step * me / denom + 1e-37
    return w, we, m, me, v


def check_step(before, s, t, h=HYPER, c=1.0):
    for i in range(len(s["w"])):
        w, we, m, me, v = expect(before, i, t, h, c)
        eps = torch.finfo(s["w"][i].dtype).eps / 2
        off = (s["w"][i].double() - w).abs()
        assert bool((off <= we + eps * (w.abs() + we)).all()), ("w", i, float((off / (we + eps * w.abs())).max()))
        if s["master"] is not None:
            off = (s["master"][i].double() - w).abs()
            assert bool((off <= we + U * w.abs()).all()), ("master", i)
            assert torch.equal(s["w"][i], s["master"][i].to(s["w"][i].dtype))
        if s["m_scale"] is None:
            assert bool(((s["m"][i].double() - m).abs() <= me + 1e-42).all()), ("m", i)
            assert bool(((s["v"][i].double() - v).abs() <= 8 * U * v + 1e-42).all()), ("v", i)
            continue
        for k, x, xe in (("m", m, me), ("v", v.sqrt(), 6 * U * v.sqrt())):
            n = x.numel()
            blocks = lambda y: torch.nn.functional.pad(y, (0, -n % B)).view(-1, B)
            scale = blocks(x.abs()).amax(dim=1).clamp_min(2.0 ** -100) / 448
            slack = blocks(xe).amax(dim=1) / 448
            got = s[k + "_scale"][i].double()
            assert bool(((got - scale).abs() <= slack + 3 * U * scale).all()), (k, "scale", i)
            per = scale.repeat_interleave(B)[:n]
            off = (wide(s, k, i) - x).abs()
            tol = torch.maximum(x.abs() * 2.0 ** -4, per * 2.0 ** -10) * (1 + 2.0 ** -10) + 2 * xe + 8 * U * x.abs()
            if k == "v":   # a value above zero keeps a code above zero
                tol = torch.where(x < per * 2.0 ** -9, per * 2.0 ** -9 * (1 + 2.0 ** -10), tol)
                assert bool((s["v"][i].float()[x > 1e-38] > 0).all())
            assert bool((off <= tol).all()), (k, i, float((off / tol.clamp_min(1e-300)).max()))


def untouched(s, offset):
    """The elements around every tensor, in the buffer that holds it"""
    for k, x in s.items():
        for t in x or ():
            base = t._base if t._base is not None else t
            if base.numel() > t.numel():
                fill = torch.tensor(77.0).to(t.dtype).float()
                rest = torch.cat((base[:offset].float(), base[offset + t.numel():].float())).cpu()
                assert bool((rest == fill).all()), k


FORMS = [(w, g, bits, master) for w, g, master in (("bf16", "bf16", False), ("bf16", "f32", False), ("bf16", "f32", True), ("bf16", "bf16", True),
                                                   ("f32", "f32", False), ("f32", "bf16", False)) for bits in (32, 8)]


@pytest.mark.parametrize("offset", [0, 1, 4])
@pytest.mark.parametrize("w,g,bits,master", FORMS)
def test_step_matches_64_bits(w, g, bits, master, offset):
    s = model(SIZES, w, g, bits, master, offset=offset)
    plan = plan_of(s)
    for t in (1000, 1001):
        before = copy_of(s)
        resbm.resbm_adamw_step(plan, step=t, **HYPER)
        torch.cuda.synchronize()
        check_step(before, s, t)
        untouched(s, offset)
        assert all(torch.equal(a.view(torch.uint8) if a.element_size() == 1 else a, b.view(torch.uint8) if b.element_size() == 1 else b)
                   for a, b in zip(before["g"], s["g"]))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 31, 32, 33, 447, 448, 449, 1000])
def test_counts(count, bits):
    """One launch's list and more than one, empty tensors among them"""
    sizes = [(37 * i) % 701 for i in range(count)]
    s = model(sizes, bits=bits)
    before = copy_of(s)
    n0 = resbm.resbm_kernel_launches()
    resbm.resbm_adamw_step(plan_of(s), step=5, **HYPER)
    assert resbm.resbm_kernel_launches() - n0 == -(-sum(n > 0 for n in sizes) // (32 if count <= 32 else 448))
    check_step(before, s, 5)
    untouched(s, 0)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_steps_and_zero_gradients(bits):
    """From zeros; then gradients of zero, and a tensor whose gradients were always zero (only decayed)."""
    s = model([1000, 300, 513], bits=bits, warm=False)
    s["g"][1].zero_()
    w1 = s["w"][1].clone()
    plan = plan_of(s)
    for t in range(1, 6):
        if t == 4:
            s["g"][0].zero_()
        before = copy_of(s)
        resbm.resbm_adamw_step(plan, step=t, **HYPER)
        check_step(before, s, t)
        w1 = (w1.float() * (1 - HYPER["lr"] * HYPER["weight_decay"])).to(w1.dtype)
    assert torch.equal(s["w"][1], w1)
    for k in ("m", "v"):
        assert bool((s[k][1].float() == 0).all())


def test_tiny_and_large_gradients():
    """Gradients over the whole of fp32's squares, 8 bits: no division by eps alone, nothing infinite."""
    for bits in (32, 8):
        s = model([2048], "f32", "f32", bits, warm=False)
        s["g"][0].copy_(torch.logspace(-18, 15, 2048, device="cuda")[torch.randperm(2048, device="cuda")])
        w0 = s["w"][0].clone()
        plan = plan_of(s)
        for t in (1, 2, 3):
            before = copy_of(s)
            resbm.resbm_adamw_step(plan, step=t, lr=1e-3, beta1=0.9, beta2=0.999, eps=0.0 if bits == 32 else 1e-12, weight_decay=0.0)
            assert bool(torch.isfinite(s["w"][0]).all())
        # constant gradients: every element moves by at most lr a step (1 + what v's rounding up of tiny values leaves)
        assert float((s["w"][0] - w0).abs().max()) <= 3 * 1e-3 * 1.15


def test_hyperparameter_edges():
    for h in (dict(lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.5), dict(lr=1e-2, beta1=0.0, beta2=0.0, eps=1e-8, weight_decay=0.0),
              dict(lr=1e-2, beta1=0.0, beta2=0.95, eps=1e-6, weight_decay=0.0)):
        for t in (1, 10 ** 7):
            s = model([777, 4096], "f32", "f32")
            before = copy_of(s)
            resbm.resbm_adamw_step(plan_of(s), step=t, **h)
            check_step(before, s, t, h)


def test_values_from_the_device_and_graph():
    """lr, step and the gradients' factor read by the kernel: the same step as with the values given, also when captured
    and replayed with others, on another stream."""
    one = lambda x, dt=torch.float32: torch.tensor([x], dtype=dt, device="cuda")
    lr, step, c = one(1e-3), one(1, torch.int64), one(0.5)
    s = model(SIZES, "f32", "f32")
    plan = plan_of(s)
    start = copy_of(s)
    args = dict(HYPER, lr=0.0)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        resbm.resbm_adamw_step(plan, lr_dev=lr, step_dev=step, grad_scale=c, **args)
    assert all(torch.equal(a, b) for k in ("w", "m", "v") for a, b in zip(start[k], s[k]))
    for t, rate, f in ((1, 1e-3, 0.5), (2, 2e-3, 1.0), (70000, 5e-4, 0.125)):
        step.fill_(t)
        lr.fill_(rate)
        c.fill_(f)
        before = copy_of(s)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        side.synchronize()
        # (1 - beta^t from expm1f of a rounded exponent: a few roundings more than the host's)
        check_step(before, s, t, dict(HYPER, lr=float(lr)), float(c))
    for bad in (float("nan"), float("inf")):
        c.fill_(bad)
        before = copy_of(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for k in ("w", "m", "v") for a, b in zip(before[k], s[k]))


@pytest.mark.parametrize("bits", [32, 8])
def test_nan_gradients_are_seen(bits):
    s = model([1000], "f32", "f32", bits)
    s["g"][0][300] = float("nan")
    resbm.resbm_adamw_step(plan_of(s), step=3, **HYPER)
    assert bool(torch.isnan(s["w"][0][300])) and int(torch.isnan(s["w"][0]).sum()) == 1
    m = wide(s, "m", 0)
    assert bool(torch.isnan(m[300])) and not bool(torch.isnan(m[:256]).any()) and not bool(torch.isnan(m[512:]).any())


def test_reproducible_and_set_grads():
    a, b = model(SIZES, bits=8), model(SIZES, bits=8)
    resbm.resbm_adamw_step(plan_of(a), step=9, **HYPER)
    moved = [g.clone() for g in b["g"]]
    plan = plan_of(b)
    for g in b["g"]:
        g.fill_(123.0)
    plan.set_grads(moved)
    resbm.resbm_adamw_step(plan, step=9, **HYPER)
    for k in ("w", "m", "v", "m_scale", "v_scale"):
        for x, y in zip(a[k], b[k]):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k
    with pytest.raises(ValueError):
        plan.set_grads(moved[:-1])
    with pytest.raises(ValueError):
        plan.set_grads([g.float() for g in moved])
    with pytest.raises(resbm.ResbmError):
        plan.set_grads(b["w"])       # what the step writes is no gradient
    with pytest.raises(resbm.ResbmError):
        resbm.resbm_adamw_step(plan, step=9, **HYPER)


def norm_of(grads, c=1.0):
    return float(torch.stack([g.double().square().sum() for g in grads]).sum().sqrt())


@pytest.mark.parametrize("g", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("sizes", [[1], [5, 300], SIZES, [3_000_001], [1000] * 700, [0, 0, 9], []])
def test_grad_norm(sizes, g, offset):
    s = model(sizes, g=g, offset=offset)
    plan = resbm.AdamWPlan(None, s["g"])
    ws = resbm.grad_norm_workspace(plan)
    out = torch.full((2,), -1.0, device="cuda")
    want = norm_of(s["g"]) if sum(sizes) else 0.0
    for max_norm in (0.0, 1e-3, 1e6):
        ws.fill_(0x7F)   # what the workspace holds does not matter
        resbm.resbm_grad_norm(plan, max_norm, out, ws)
        got, coef = out.tolist()
        assert abs(got - want) <= 20 * U * want
        c = min(1.0, max_norm / (want + 1e-6)) if max_norm else 1.0
        assert abs(coef - c) <= 24 * U * c
    first = out.clone()
    resbm.resbm_grad_norm(plan, 1e6, out, ws)
    assert torch.equal(first, out)


def test_grad_norm_of_several_plans_and_special_values():
    a, b = model(SIZES, g="bf16"), model([70001, 3], g="f32", seed=4)
    plans = [plan_of(a), resbm.AdamWPlan(None, b["g"])]
    ws = resbm.grad_norm_workspace(plans)
    out = torch.empty(2, device="cuda")
    resbm.resbm_grad_norm(plans, 1.0, out, ws)
    want = norm_of(a["g"] + b["g"])
    assert abs(float(out[0]) - want) <= 20 * U * want
    for bad in (float("nan"), float("inf"), 1e25):   # (the square of 1e25 is no fp32)
        b["g"][1][2] = bad
        resbm.resbm_grad_norm(plans, 1.0, out, ws)
        assert not bool(torch.isfinite(out[0])) and bool(torch.isnan(out[1]))
        before = copy_of(a)
        resbm.resbm_adamw_step(plans[0], step=3, grad_scale=out[1:], **HYPER)   # ... so that the step changes nothing
        assert all(torch.equal(x, y) for k in ("w", "m", "v") for x, y in zip(before[k], a[k]))
    with pytest.raises(resbm.ResbmError):
        resbm.resbm_adamw_step(plans[1], step=1, **HYPER)      # gradients only


@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_step_in_a_graph(bits):
    """The norm and the step that reads its coefficient, captured together and replayed with other gradients."""
    s = model(SIZES, "bf16", "f32", bits, True)
    plan = plan_of(s)
    ws, out = resbm.grad_norm_workspace(plan), torch.empty(2, device="cuda")
    step = torch.tensor([0], dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step += 1
        resbm.resbm_grad_norm(plan, 0.25, out, ws)
        resbm.resbm_adamw_step(plan, step_dev=step, grad_scale=out[1:], **HYPER)
    for t in (1, 2, 3):
        for g in s["g"]:
            g.mul_(1.5)
        before = copy_of(s)
        graph.replay()
        torch.cuda.synchronize()
        want = norm_of(s["g"])
        c = min(1.0, 0.25 / (want + 1e-6))   # (1 in the first of the three)
        assert abs(float(out[0]) - want) <= 20 * U * want and abs(float(out[1]) - c) <= 24 * U * c
        check_step(before, s, t, HYPER, float(out[1]))


def test_binding_refusals():
    f = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
    ok = dict(params=[f(300)], grads=[f(300)], m=[f(300)], v=[f(300)])
    resbm.AdamWPlan(**ok)
    for bad in (dict(grads=[f(299)]), dict(m=None), dict(m=[f(300, dtype=torch.bfloat16)]), dict(params=[f(600)[::2]]), dict(grads=[f(300).half()]), dict(v=[f(300), f(300)]),
                dict(params=[torch.zeros(300)]), dict(master=[f(300)]), dict(m_scale=[f(2)], v_scale=[f(2)]), dict(params=None),
                dict(m=[f(300, dtype=torch.uint8)], v=[f(300, dtype=torch.uint8)]),
                dict(m=[f(300, dtype=torch.uint8)], v=[f(300, dtype=torch.uint8)], m_scale=[f(1)], v_scale=[f(1)])):
        with pytest.raises(ValueError):
            resbm.AdamWPlan(**{**ok, **bad})
    with pytest.raises(resbm.ResbmError):
        resbm.AdamWPlan([ok["params"][0]] * 2, ok["grads"] * 2, ok["m"] * 2, ok["v"] * 2)   # the same tensor twice
    plan = resbm.AdamWPlan(**ok)
    with pytest.raises(ValueError):
        resbm.resbm_adamw_step(plan, 1e-3, step_dev=f(1))
    with pytest.raises(ValueError):
        resbm.resbm_adamw_step(plan, 1e-3, grad_scale=torch.ones(1))
    with pytest.raises(resbm.ResbmError):
        resbm.resbm_adamw_step(plan, 1e-3, step=0)
    with pytest.raises(ValueError):
        resbm.resbm_grad_norm(plan, 1.0, f(3), f(64))
    with pytest.raises(resbm.ResbmError):
        resbm.resbm_grad_norm(plan, 1.0, f(2), f(1, dtype=torch.uint8))


@pytest.mark.parametrize("bits", [32, 8])
def test_offsets_past_32_bits(bits):
    """One tensor of over 2^31 elements: its first, middle and last elements, and its norm."""
    n = (1 << 31) + 70001
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB")
    gen = torch.Generator(device="cuda").manual_seed(3)
    t = lambda dtype: torch.zeros(n, dtype=dtype, device="cuda")
    w, g, m, v = t(torch.bfloat16), t(torch.bfloat16), t(torch.uint8 if bits == 8 else torch.float32), t(torch.uint8 if bits == 8 else torch.float32)
    scales = [torch.zeros(-(-n // B), device="cuda") for _ in range(2)] if bits == 8 else [None, None]
    spots = [slice(0, 1000 * B), slice((1 << 31) - 500 * B, (1 << 31) + 200 * B), slice(n // B * B - 100 * B, n)]
    for at in spots:
        for x, size in ((w, 0.1), (g, 1e-2)):
            x[at] = (size * torch.randn(x[at].numel(), generator=gen, device="cuda")).to(x.dtype)
    start, grads = [w[at].clone() for at in spots], [g[at].clone() for at in spots]
    plan = resbm.AdamWPlan([w], [g], [m], [v], *[[x] if x is not None else None for x in scales])
    ws, out = resbm.grad_norm_workspace(plan), torch.empty(2, device="cuda")
    resbm.resbm_grad_norm(plan, 0.0, out, ws)
    covered = torch.cat([g[spots[0]], g[spots[1].start:]]) if spots[2].start < spots[1].stop else torch.cat([g[at] for at in spots])
    want = norm_of([covered])
    assert abs(float(out[0]) - want) <= 20 * U * want
    resbm.resbm_adamw_step(plan, step=1, **HYPER)
    for at, w0, g0 in zip(spots, start, grads):
        k = w0.numel()
        blank = lambda x: [torch.zeros(x, device="cuda")]
        before = {"w": [w0], "g": [g0], "m": blank(k), "v": blank(k), "m_scale": None, "v_scale": None, "master": None}
        part = slice(at.start // B, -(-at.stop // B))
        view = lambda x: [x[at].view(E4M3) if bits == 8 else x[at]]
        after = {"w": [w[at]], "g": [g0], "m": view(m), "v": view(v), "m_scale": [scales[0][part]] if bits == 8 else None,
                 "v_scale": [scales[1][part]] if bits == 8 else None, "master": None}
        if bits == 8:
            before |= {"m_scale": [torch.zeros_like(scales[0][part])], "v_scale": [torch.zeros_like(scales[1][part])]}
        check_step(before, after, 1)
    assert bool((w[spots[0].stop:spots[0].stop + 1000] == 0).all())


def test_the_workspace_goes_by_the_count_alone():
    """Gradients that move off the alignment need no other workspace."""
    s = model([3_000_000, 500_000, 70_000], "f32", "f32")
    plan = plan_of(s)
    ws, out = resbm.grad_norm_workspace(plan), torch.empty(2, device="cuda")
    moved = [torch.empty(g.numel() + 1, device="cuda")[1:] if i != 1 else g for i, g in enumerate(s["g"])]
    for a, b in zip(moved, s["g"]):
        a.copy_(b)
    plan.set_grads(moved)
    assert resbm.grad_norm_workspace(plan).numel() == ws.numel()
    resbm.resbm_grad_norm(plan, 0.0, out, ws)
    want = norm_of(s["g"])
    assert abs(float(out[0]) - want) <= 20 * U * want
    s["g"] = moved
    before = copy_of(s)
    resbm.resbm_adamw_step(plan, step=4, **HYPER)
    check_step(before, s, 4)
