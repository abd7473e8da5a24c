"""Chains of AdamW steps beside the same arithmetic in IEEE fp32: the states that a step leaves are what the next one reads, so
that a rounding that differs once is a difference that stays (an 8-bit code that goes the other way is up to 1 / 8 off).

The reference rounds to fp32 after every operation: it computes each in 64 bits from fp32 values and rounds the result once.
For sums, products, quotients and roots of fp32 values that is IEEE's own result (53 bits are at least twice 24 and two more).
The running means, their scales and their codes have no other freedom, so they have to be equal bit for bit."""
import pytest
import torch

from paper_2604_11947_gb300 import resbm
from test_adamw_gpu import B, E4M3, FORMS, HYPER, copy_of, model, plan_of

pytestmark = pytest.mark.gpu
SIZES = [1, 255, 257, 2048, 4099, 70001]
STEPS = 20


def f(x):
    """x (64 bits) rounded to fp32, as a number in 64 bits"""
    return x.float().double()


def const(x):
    return float(torch.tensor(x, dtype=torch.float32))


def decode(code, scale):
    """e4m3 codes in units of their blocks' scales, rounded to fp32"""
    return f(code.double() * scale.double().repeat_interleave(B)[:code.numel()])


def encode(x, least=False):
    """Codes and scales of x; least: a value above zero keeps a code above zero"""
    blocks = torch.nn.functional.pad(x.abs(), (0, -x.numel() % B)).view(-1, B)
    most = blocks.amax(dim=1).clamp_min(2.0 ** -100)
    inv = f(f(1 / most) * 448).repeat_interleave(B)[:x.numel()]
    y = f(x * inv)
    if least:
        y = torch.where(x > 0, y.clamp_min(2.0 ** -9), y)
    return y.clamp(-448, 448).float().to(E4M3), f(most * const(1 / 448)).float()


def means(s, i, h=HYPER):
    """m and v of tensor i after a step, rounded after every operation"""
    b1, b2, c1, c2 = const(h["beta1"]), const(h["beta2"]), const(1 - h["beta1"]), const(1 - h["beta2"])
    g = s["g"][i].double()
    if s["m_scale"] is None:
        m, v = s["m"][i].double(), s["v"][i].double()
    else:
        m, v = decode(s["m"][i], s["m_scale"][i]), decode(s["v"][i], s["v_scale"][i])
        v = f(v * v)
    return f(f(m * b1) + f(g * c1)), f(f(v * b2) + f(f(g * g) * c2))


def same(a, b):
    return torch.equal(a.view(torch.uint8) & 0x7F, b.view(torch.uint8) & 0x7F) if a.element_size() == 1 else torch.equal(a, b)


def fresh_gradients(s, t):
    gen = torch.Generator(device="cuda").manual_seed(1000 + t)
    for g in s["g"]:
        g.copy_(1e-3 * torch.exp(torch.randn(1, generator=gen, device="cuda")) * torch.randn(g.numel(), generator=gen, device="cuda"))


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("w,g,bits,master", FORMS)
def test_running_means_round_every_product(w, g, bits, master, offset):
    """Twenty steps: m (codes and scales, or fp32) and fp32 v are the reference's own bits."""
    s = model(SIZES, w, g, bits, master, offset=offset)
    plan, mine = plan_of(s), copy_of(s)
    for t in range(1, STEPS + 1):
        fresh_gradients(s, t)
        mine["g"] = s["g"]
        resbm.resbm_adamw_step(plan, step=t + 100, **HYPER)
        for i in range(len(SIZES)):
            m, v = means(mine, i)
            if bits == 32:
                mine["m"][i], mine["v"][i] = m.float(), v.float()
                assert same(s["v"][i], mine["v"][i]), (t, i)
            else:
                mine["m"][i], mine["m_scale"][i] = encode(m)
                assert same(s["m_scale"][i], mine["m_scale"][i]), (t, i)
            assert same(s["m"][i], mine["m"][i]), (t, i)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("w,g,bits,master", [form for form in FORMS if form[2] == 8])
def test_stored_roots_and_weights_after_many_steps(w, g, bits, master, offset):
    """Twenty steps with 8-bit states: sqrt(v)'s codes and scales are the reference's own bits, and the weights are off by no
    more than the steps' roundings together: 16 u of each update and 4 u of the weight (u = 2^-24, as for one step), and,
    where the weight itself is what is kept, one rounding to its type a step."""
    s = model(SIZES, w, g, bits, master, offset=offset)
    plan, mine = plan_of(s), copy_of(s)
    kept = "master" if master else "w"
    weight = [x.double() for x in mine[kept]]
    slack = [torch.zeros_like(x) for x in weight]
    u = 2.0 ** -24
    half = torch.finfo(s[kept][0].dtype).eps / 2
    for t in range(1, STEPS + 1):
        fresh_gradients(s, t)
        mine["g"] = s["g"]
        resbm.resbm_adamw_step(plan, step=t + 100, **HYPER)
        for i in range(len(SIZES)):
            m, v = means(mine, i)
            root = f(v.sqrt())
            mine["m"][i], mine["m_scale"][i] = encode(m)
            mine["v"][i], mine["v_scale"][i] = encode(root, least=True)
            assert same(s["v_scale"][i], mine["v_scale"][i]), (t, i)
            assert same(s["v"][i], mine["v"][i]), (t, i)
            n = t + 100
            update = HYPER["lr"] / (1 - HYPER["beta1"] ** n) * m / (root / (1 - HYPER["beta2"] ** n) ** 0.5 + HYPER["eps"])
            weight[i] = weight[i] * (1 - HYPER["lr"] * HYPER["weight_decay"]) - update
            slack[i] += 4 * u * weight[i].abs() + 16 * u * update.abs()
            if half > u:
                slack[i] += half * (weight[i].abs() + slack[i])
    for i in range(len(SIZES)):
        off = (s[kept][i].double() - weight[i]).abs()
        assert bool((off <= slack[i] + half * weight[i].abs()).all()), (i, float((off / slack[i]).max()))


def test_small_and_large_second_moments_in_8_bits():
    """Roots over the whole range: gradients whose squares leave fp32 at either end. Above zero stays above zero; an overflow
    is seen, as NaN, in its own block and weight only."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    for size in (1e-17, 1e-12, 1e-6, 1.0, 1e6, 1e12):
        s = model([3 * B], "f32", "f32", 8, warm=False)
        s["g"][0].copy_(size * (1 + torch.rand(3 * B, generator=gen, device="cuda")))
        mine = copy_of(s)
        resbm.resbm_adamw_step(plan_of(s), step=1, lr=1e-3, beta1=0.0, beta2=0.5, eps=0.0, weight_decay=0.0)
        v = f(f(mine["g"][0].double() ** 2) * 0.5)
        code, scale = encode(f(v.sqrt()), least=True)
        if size > 1e-15:
            assert same(s["v"][0], code) and same(s["v_scale"][0], scale)
        assert bool((s["v"][0].float() > 0).all())
    s = model([3 * B], "f32", "f32", 8)
    s["g"][0][B + 5] = 1e25
    resbm.resbm_adamw_step(plan_of(s), step=1, **HYPER)
    root = s["v"][0].float() * s["v_scale"][0].repeat_interleave(B)
    assert torch.isnan(root).view(3, B).all(dim=1).tolist() == [False, True, False]
    assert torch.isnan(s["w"][0]).nonzero().flatten().tolist() == [B + 5]


def test_8_bit_second_moments_change_by_half_a_step_or_not_at_all():
    """What the header says of them, on constant gradients of one at beta2 = 0.999: an element whose gradients fall to a fifth keeps
    its code (0.05 % a step), while fp32 states follow; one of twenty times the others' (18 % in one step) shows at once."""
    h = dict(HYPER, beta1=0.0, beta2=0.999)
    left = {}
    for bits in (32, 8):
        s = model([B], "f32", "f32", bits, warm=False)
        plan = plan_of(s)
        s["g"][0].fill_(1.0)
        resbm.resbm_adamw_step(plan, step=1, **dict(h, beta2=0.0))      # v = 1
        s["g"][0][5] = 0.2
        for t in range(2, 502):
            resbm.resbm_adamw_step(plan, step=t, **h)
        root = s["v"][0].sqrt() if bits == 32 else s["v"][0].float() * s["v_scale"][0]
        left[bits] = float(root[5])
        assert abs(float(root[6]) - 1) <= 1e-3
        s["g"][0][5] = 1.0
        s["g"][0][7] = 20.0
        resbm.resbm_adamw_step(plan, step=502, **h)
        root = s["v"][0].sqrt() if bits == 32 else s["v"][0].float() * s["v_scale"][0]
        assert abs(float(root[7]) - 1.399 ** 0.5) <= 2e-3
    # 500 steps of 0.999 v + 0.001 / 25 from 1
    v = 0.04 + 0.96 * 0.999 ** 500
    assert abs(left[32] - v ** 0.5) <= 1e-4 and abs(left[8] - 1) <= 1e-3
