"""optim.AdamW (the library's step as a torch optimizer) and the pipeline's fused norms: against 64 bits, against torch, and
together in training steps as they are used."""
import copy
import weakref

import pytest
import torch

from paper_2604_11947_gb300 import optim, pipeline, resbm
from test_adamw_gpu import U, check_step, norm_of

pytestmark = pytest.mark.gpu
H = dict(lr=2e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.05)
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.05)


def params_of(sizes, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.nn.Parameter((0.1 * torch.randn(n, generator=g, device="cuda")).to(dtype)) for n in sizes]


def set_grads(params, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for p in params:
        p.grad = (1e-2 * torch.randn(p.shape, generator=g, device="cuda")).to(p.dtype)


def columns(opt, params):
    """The optimizer's tensors as test_adamw_gpu's lists"""
    st = [opt.state[p] for p in params]
    c = lambda k: [s[k].reshape(-1).clone() for s in st] if k in st[0] else None
    return {"w": [p.detach().reshape(-1).clone() for p in params], "g": [p.grad.reshape(-1).clone() for p in params], "m": c("exp_avg"), "v": c("exp_avg_sq"),
            "m_scale": c("exp_avg_scale"), "v_scale": c("exp_avg_sq_scale"), "master": c("master")}


@pytest.mark.parametrize("bits,master", [(32, False), (8, False), (32, True), (8, True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_match_64_bits(dtype, bits, master):
    params = params_of([1, 300, 256, 5000], dtype)
    opt = optim.AdamW(params, state_bits=bits, master=master, **H)
    set_grads(params, 1)
    opt.step()
    for t in range(2, 5):
        if t == 3:
            opt.zero_grad(set_to_none=True)      # gradients in other memory
        set_grads(params, t)
        before = columns(opt, params)
        opt.step()
        check_step(before, columns(opt, params), t, HYPER)
        assert all(opt.state[p]["step"] == t for p in params)


def test_fp32_follows_torch():
    """Twenty steps beside torch.optim.AdamW in fp32: every step's update agrees to 24 roundings of the update and one of
    the weight (the two differ in the order of a few operations), so twenty differ by at most the sum."""
    a, b = params_of([64, 1000], torch.float32), params_of([64, 1000], torch.float32)
    mine, theirs = optim.AdamW(a, **H), torch.optim.AdamW(b, **H)
    for t in range(20):
        set_grads(a, t)
        set_grads(b, t)
        mine.step()
        theirs.step()
    for x, y in zip(a, b):
        # |update| <= lr |m| / sqrt(v) / (corrections), at most 7.3 lr for these betas
        tol = 20 * (24 * U * 7.3 * H["lr"] + 4 * U * x.abs())
        assert bool(((x - y).abs() <= tol).all()), float(((x - y).abs() / tol).max())


def test_clipping_groups_and_late_parameters():
    """Two groups of their own lr and decay, types mixed, a parameter that gets its first gradient late: the norm is of all
    gradients together, every parameter counts its own steps."""
    f, h = params_of([700, 64], torch.float32), params_of([1000, 300, 5], torch.bfloat16)
    opt = optim.AdamW([{"params": f + h[:1]}, {"params": h[1:], "lr": 5e-3, "weight_decay": 0.0}], max_grad_norm=0.05, **H)
    late = h[2]
    for t in range(1, 4):
        set_grads(f + h, t)
        if t == 1:
            late.grad = None
        live = [p for p in f + h if p.grad is not None]
        before = {p: columns(opt, [p]) for p in live if opt.state[p]}
        w0 = late.detach().clone()
        opt.step()
        want = norm_of([p.grad for p in live])
        assert abs(float(opt.grad_norm[0]) - want) <= 20 * U * want and float(opt.grad_norm[1]) < 1
        if t == 1:
            assert torch.equal(late, w0) and not opt.state[late]
        for p, b in before.items():
            group = H if any(p is x for x in f + h[:1]) else dict(H, lr=5e-3, weight_decay=0.0)
            hyper = dict(HYPER, lr=group["lr"], weight_decay=group["weight_decay"])
            check_step(b, columns(opt, [p]), opt.state[p]["step"], hyper, float(opt.grad_norm[1]))
    assert opt.state[late]["step"] == 2 and opt.state[f[0]]["step"] == 3
    # a norm that is no number: nothing moves
    f[0].grad[3] = float("nan")
    before = [p.detach().clone() for p in f + h]
    opt.step()
    assert all(torch.equal(a, b) for a, b in zip(before, f + h))


@pytest.mark.parametrize("bits,master", [(32, False), (8, True)])
def test_state_dict_goes_on_where_it_was(bits, master):
    params = params_of([300, 5000], torch.bfloat16)
    opt = optim.AdamW(params, state_bits=bits, master=master, **H)
    for t in range(3):
        set_grads(params, t)
        opt.step()
    others = [torch.nn.Parameter(p.detach().clone()) for p in params]
    again = optim.AdamW(others, state_bits=bits, master=master, lr=1.0)
    again.load_state_dict(copy.deepcopy(opt.state_dict()))
    assert again.param_groups[0]["lr"] == H["lr"]
    for t in range(3, 6):
        set_grads(params, t)
        set_grads(others, t)
        opt.step()
        again.step()
    for p, q in zip(params, others):
        assert torch.equal(p, q)
        for k, v in opt.state[p].items():
            o = again.state[q][k]
            assert o.dtype == v.dtype and torch.equal(o.view(torch.uint8), v.view(torch.uint8)) if torch.is_tensor(v) else o == v
    with pytest.raises(ValueError):
        optim.AdamW(others, state_bits=40 - bits, master=master).load_state_dict(opt.state_dict())
    with pytest.raises(ValueError):
        optim.AdamW(others, state_bits=bits, master=not master).load_state_dict(opt.state_dict())


def test_gradients_are_let_go():
    """After the step nothing of the optimizer holds the gradients' memory; gradients that stay where they are serve again."""
    params = params_of([1000, 300], torch.float32)
    opt = optim.AdamW(params, max_grad_norm=1.0, **H)
    set_grads(params, 1)
    for t in (2, 3):
        before = columns(opt, params) if t > 2 else None
        opt.step()
        if before:
            check_step(before, columns(opt, params), 2, HYPER, float(opt.grad_norm[1]))
        for p in params:
            p.grad.mul_(0.5)
    held = [weakref.ref(p.grad) for p in params]
    opt.zero_grad(set_to_none=True)
    assert all(h() is None for h in held)
    plan = resbm.AdamWPlan(None, [torch.ones(5, device="cuda")])
    ws, out = resbm.grad_norm_workspace(plan), torch.empty(2, device="cuda")
    plan.release_grads()
    with pytest.raises(ValueError):
        resbm.resbm_grad_norm(plan, 1.0, out, ws)
    plan.set_grads([torch.full((5,), 2.0, device="cuda")])
    resbm.resbm_grad_norm(plan, 0.0, out, ws)
    assert abs(float(out[0]) - 20 ** 0.5) <= 4 * U * 20 ** 0.5


def test_refusals():
    p = params_of([10], torch.float32)
    for bad in (dict(state_bits=16), dict(max_grad_norm=0.0), dict(max_grad_norm=float("inf")), dict(lr=-1.0), dict(betas=(0.9, 1.0))):
        with pytest.raises(ValueError):
            optim.AdamW(p, **bad)
    cpu = [torch.nn.Parameter(torch.zeros(4))]
    cpu[0].grad = torch.zeros(4)
    with pytest.raises(ValueError):
        optim.AdamW(cpu).step()
    half = [torch.nn.Parameter(torch.zeros(4, dtype=torch.float16, device="cuda"))]
    half[0].grad = torch.zeros_like(half[0])
    with pytest.raises(ValueError):
        optim.AdamW(half).step()
    opt = optim.AdamW(p)
    set_grads(p, 1)
    opt.step()
    before = p[0].detach().clone()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(graph):
            opt.step()
    torch.cuda.synchronize()
    assert torch.equal(before, p[0])


# ---- the norm with its backward, and everything together ------------------------------------------
def reference(x, a, gamma, dh, dn, eps=pipeline.NORM_EPS):
    """h, n and the gradients in 64 bits, from the stored h"""
    h = (x.float() + a.float()).to(x.dtype).double()
    s = (h.square().mean(dim=1, keepdim=True) + eps).rsqrt()
    g = dn.double() * gamma.double()
    d = dh.double() + s * g - h * s ** 3 * (g * h).mean(dim=1, keepdim=True)
    return h, h * s * gamma.double(), d, (dn.double() * h * s).sum(dim=0)


@pytest.mark.parametrize("dtype,T,d", [(torch.float32, 33, 100), (torch.float32, 7, 1001), (torch.bfloat16, 300, 512), (torch.bfloat16, 5, 77), (torch.float32, 1, 64)])
def test_add_norm_gradients(dtype, T, d):
    """Forward and backward of pipeline.add_norm: the gradient that x and a share, gamma's, each against the formula; an
    input broadcast over the rows gets the sum of theirs."""
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)
    x, a, gamma, dh, dn = rnd(T, d), rnd(T, d), rnd(d), rnd(T, d), rnd(T, d)
    for t in (x, a, gamma):
        t.requires_grad_()
    h, n = pipeline.add_norm(x, a, gamma)
    torch.autograd.backward((h, n), (dh, dn))
    _, wn, wd, wg = reference(x.detach(), a.detach(), gamma.detach(), dh, dn)
    eps = torch.finfo(dtype).eps / 2
    # sums over d in fp32: at most d / 32 + 40 terms one after the other; 40 operations more along the way
    terms = (d / 32 + 80) * U
    size = wd.abs().amax() + dn.abs().amax() * gamma.abs().amax() * 4
    assert bool(((n.double() - wn).abs() <= eps * wn.abs() + terms * (wn.abs() + 1)).all())
    assert bool(((x.grad.double() - wd).abs() <= eps * wd.abs() + terms * size).all())
    assert torch.equal(x.grad, a.grad)
    assert bool(((gamma.grad.double() - wg).abs() <= eps * wg.abs() + (T + 40) * U * (dn.double().abs() * wn.abs().amax()).sum(dim=0) + 1e-6).all())
    # one of the two outputs only, and no addition
    for which in (0, 1):
        y, b, gm = (t.detach().clone().requires_grad_() for t in (x, a, gamma))
        pipeline.add_norm(y, b, gm)[which].backward(dh if which == 0 else dn)
        z = torch.zeros_like(dn)
        want = reference(x.detach(), a.detach(), gamma.detach(), dh if which == 0 else z, z if which == 0 else dn)[2]
        assert bool(((y.grad.double() - want).abs() <= eps * want.abs() + terms * size).all()) and torch.equal(y.grad, b.grad)
        assert (gm.grad is None) == (which == 0)
    y = x.detach().clone().requires_grad_()
    pipeline.add_norm(y, None, gamma.detach())[1].backward(dn)
    want = reference(x.detach(), torch.zeros_like(x), gamma.detach(), torch.zeros_like(dn), dn)[2]
    assert bool(((y.grad.double() - want).abs() <= eps * want.abs() + terms * size).all())
    row = a.detach()[:1].clone().requires_grad_()
    h, n = pipeline.add_norm(x.detach(), row.expand(T, d), gamma.detach())
    torch.autograd.backward((h, n), (dh, dn))
    want = reference(x.detach(), row.detach().expand(T, d), gamma.detach(), dh, dn)[2].sum(dim=0, keepdim=True)
    assert bool(((row.grad.double() - want).abs() <= eps * (want.abs() + 3 * T * size) + terms * size * T).all())


def test_add_norm_gradients_by_differences():
    """Central differences of a loss in 64 bits along random directions (fp32 tensors): with steps of 2^-7 the loss, a sum of
    T d terms of size one, moves by far more than fp32's rounding of the outputs, and the third derivative leaves under
    1 % of the slope's size."""
    g = torch.Generator(device="cuda").manual_seed(9)
    T, d = 6, 40
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, a, gamma, u, v = rnd(T, d), rnd(T, d), rnd(d), rnd(T, d), rnd(T, d)
    loss = lambda X, A, G: sum((o.double() * w.double()).sum() for o, w in zip(pipeline.add_norm(X, A, G), (u, v)))
    leaves = [t.clone().requires_grad_() for t in (x, a, gamma)]
    loss(*leaves).backward()
    for i in range(3):
        way = torch.randn(leaves[i].shape, generator=g, device="cuda")
        way /= way.norm()
        at = lambda e: loss(*[t.detach() + (e * way if k == i else 0) for k, t in enumerate(leaves)])
        slope = float(at(2.0 ** -7) - at(-2.0 ** -7)) * 2.0 ** 6
        grad = leaves[i].grad.double()
        assert abs(slope - float((grad * way).sum())) <= 1e-2 * float(grad.norm()), (i, slope)


def test_add_norm_captured_both_ways():
    """Forward and backward in one CUDA graph, replayed with other inputs; nothing eager of the same leaves is alive."""
    T, d = 64, 300
    leaves = [torch.zeros(T, d, device="cuda", requires_grad=True), torch.zeros(T, d, device="cuda", requires_grad=True),
              torch.ones(d, device="cuda", requires_grad=True)]
    dh, dn = torch.zeros(T, d, device="cuda"), torch.zeros(T, d, device="cuda")

    def both_ways():
        h, n = pipeline.add_norm(*leaves)
        torch.autograd.backward((h, n), (dh, dn))
        return h.detach(), n.detach()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both_ways()
    torch.cuda.current_stream().wait_stream(side)
    for t in leaves:
        t.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, n = both_ways()
    g = torch.Generator(device="cuda").manual_seed(11)
    for _ in range(2):
        new = [torch.randn(t.shape, generator=g, device="cuda") for t in leaves]
        with torch.no_grad():
            for t, x in zip(leaves, new):
                t.copy_(x)
        for t in (dh, dn):
            t.copy_(torch.randn(T, d, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        eager = [x.clone().requires_grad_() for x in new]
        eh, en = pipeline.add_norm(*eager)
        torch.autograd.backward((eh, en), (dh, dn))
        assert torch.equal(h, eh) and torch.equal(n, en)
        assert all(torch.equal(t.grad, e.grad) for t, e in zip(leaves, eager))


def test_add_norm_has_no_second_derivative():
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    n = pipeline.add_norm(x, x, torch.ones(8, device="cuda"))[1]
    (g,) = torch.autograd.grad(n.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("wiring", ["A", "B"])
@pytest.mark.parametrize("fuse_norm", [True, False])
def test_fused_norms_match_the_unfused_model(wiring, fuse_norm):
    """The same model with the norms fused with the additions before them and without: the loss and every gradient agree to
    bf16 noise (the two round at the same places but for the norm's own)."""
    cfg = pipeline.PipelineConfig(layers=4, d=512, heads=4, ffn=1024, vocab=1000, stages=2, r=16, m=16, batch=2, seq=256,
                                  wiring=wiring, fuse_norm=fuse_norm)
    tokens = pipeline.synthetic_tokens(cfg)
    grads, losses = [], []
    for fuse in (True, False):
        model = pipeline.PipelineModel(cfg.with_(fuse_add_norm=fuse))
        losses.append(float(pipeline.train_step(model, tokens).detach()))
        grads.append({k: p.grad.float().clone() for k, p in model.named_parameters()})
    assert abs(losses[0] - losses[1]) < 1e-3 * abs(losses[1])
    for k in grads[1]:
        a, b = grads[0][k], grads[1][k]
        rel = float((a - b).norm() / b.norm().clamp_min(1e-30))
        assert rel < 3e-2, (k, rel)
    assert resbm.resbm_device_error() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_training_steps_together(bits):
    """Fused norms forward and backward, the gradients' norm and the clipped step, as a training program runs them: after
    each of three steps every tensor of the model is what the definition makes of the gradients that the step met."""
    cfg = pipeline.PipelineConfig(layers=2, d=256, heads=4, ffn=512, vocab=200, stages=2, r=16, m=16, batch=2, seq=64,
                                  fuse_add_norm=True)
    model = pipeline.PipelineModel(cfg)
    tokens = pipeline.synthetic_tokens(cfg)
    params = list(model.parameters())
    opt = optim.AdamW(params, state_bits=bits, max_grad_norm=0.5, **H)
    for t in range(1, 4):
        pipeline.train_step(model, tokens)
        before = columns(opt, params) if t > 1 else None
        opt.step()
        want = norm_of([p.grad for p in params])
        assert abs(float(opt.grad_norm[0]) - want) <= 20 * U * want
        if before:
            check_step(before, columns(opt, params), t, HYPER, float(opt.grad_norm[1]))
    assert resbm.resbm_device_error() == 0


def test_train_curve_with_the_library_optimizer():
    """The convergence comparison's loop runs with it (4 steps), its loss finite at every step."""
    data, _ = pipeline.markov_batches(pipeline.CONVERGENCE, 4)
    for bits in (32, 8):
        curve = pipeline.train_curve(pipeline.CONVERGENCE.with_(fuse_add_norm=True), data, 4, every=1,
                                     optimizer=lambda p, lr: optim.AdamW(p, lr=lr, state_bits=bits, max_grad_norm=1.0))
        assert len(curve) == 4 and all(loss == loss and abs(loss) < 100 for _, loss in curve)
