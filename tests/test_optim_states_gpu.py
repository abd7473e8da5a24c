"""optim.AdamW where a program changes what the optimizer holds between steps: states cleared, replaced, moved; every step is
checked against its definition in 64 bits from the tensors in opt.state and in the parameters, and against torch's where torch
says what happens."""
import copy
import gc
import weakref

import pytest
import torch

from paper_2604_11947_gb300 import optim
from test_adamw_gpu import check_step
from test_optim_gpu import H, HYPER, columns, params_of, set_grads

pytestmark = pytest.mark.gpu
FORMS = [(torch.float32, 32, False), (torch.bfloat16, 8, False), (torch.bfloat16, 32, True), (torch.bfloat16, 8, True)]
SIZES = [1, 300, 256, 5000]


def grads_in_place(params, t):
    """New values where the gradients are"""
    gen = torch.Generator(device="cuda").manual_seed(t)
    for p in params:
        if p.grad is None:
            p.grad = torch.zeros_like(p)
        p.grad.copy_(1e-2 * torch.randn(p.shape, generator=gen, device="cuda"))


def stepped(opt, params, t, step=None):
    """One step with new gradients in place, checked from the state before it; `step`: which it is to the states"""
    grads_in_place(params, t)
    before = columns(opt, params) if all(opt.state[p] for p in params) else None
    opt.step()
    after = columns(opt, params)
    if before is not None:
        check_step(before, after, step or t, HYPER)
    assert all(opt.state[p]["step"] == (step or t) for p in params)
    return after


@pytest.mark.parametrize("dtype,bits,master", FORMS)
def test_cleared_states_start_again(dtype, bits, master):
    """opt.state.clear(): the next step is the first one of new moments, as a new optimizer's on the same parameters."""
    params = params_of(SIZES, dtype)
    opt = optim.AdamW(params, state_bits=bits, master=master, **H)
    for t in range(1, 6):
        stepped(opt, params, t)
    opt.state.clear()
    others = [torch.nn.Parameter(p.detach().clone()) for p in params]
    fresh = optim.AdamW(others, state_bits=bits, master=master, **H)
    for t in range(1, 4):
        stepped(opt, params, t)
        grads_in_place(others, t)
        fresh.step()
        for p, q in zip(params, others):
            assert torch.equal(p, q)
            for k, v in opt.state[p].items():
                o = fresh.state[q][k]
                assert torch.equal(v.view(torch.uint8), o.view(torch.uint8)) if torch.is_tensor(v) else v == o, k
    assert all(bool((opt.state[p]["exp_avg"].float() != 0).any()) for p in params)


@pytest.mark.parametrize("dtype,bits,master", FORMS)
def test_states_that_move(dtype, bits, master):
    """Off the device and back, in one entry or all of them, as new tensors or under the same ones: the step goes on from what
    opt.state holds and leaves its result there."""
    params = params_of(SIZES, dtype)
    opt = optim.AdamW(params, state_bits=bits, master=master, **H)
    for t in range(1, 3):
        stepped(opt, params, t)
    for t, move in enumerate((lambda st, k: st.__setitem__(k, st[k].cpu().cuda()), lambda st, k: st.__setitem__(k, st[k].clone()),
                              lambda st, k: setattr(st[k], "data", st[k].data.clone())), 3):
        for p in params:
            for k, v in list(opt.state[p].items()):
                if torch.is_tensor(v):
                    move(opt.state[p], k)
        stepped(opt, params, t)
    opt.state[params[1]]["exp_avg"] = opt.state[params[1]]["exp_avg"].clone()
    stepped(opt, params, 6)
    opt.state[params[2]].clear()     # one parameter starts again, the others go on
    grads_in_place(params, 7)
    before = columns(opt, params[:2] + params[3:])
    opt.step()
    check_step(before, columns(opt, params[:2] + params[3:]), 7, HYPER)
    assert opt.state[params[2]]["step"] == 1 and bool((opt.state[params[2]]["exp_avg"].float() != 0).any())


def test_states_on_another_device_are_refused():
    params = params_of([300], torch.float32)
    opt = optim.AdamW(params, **H)
    stepped(opt, params, 1)
    opt.state[params[0]]["exp_avg"] = opt.state[params[0]]["exp_avg"].cpu()
    with pytest.raises(ValueError):
        opt.step()
    opt.state[params[0]]["exp_avg"] = opt.state[params[0]]["exp_avg"].cuda()
    stepped(opt, params, 2)


def test_resized_parameters_are_refused():
    """A parameter that became shorter where it lies: its states are of another size, and nothing behind it is written."""
    params = params_of([300], torch.float32)
    opt = optim.AdamW(params, **H)
    stepped(opt, params, 1)
    whole, grad = params[0].data, params[0].grad
    params[0].grad = None
    params[0].data = whole[:100]
    params[0].grad = grad[:100]
    before = whole.clone()
    with pytest.raises(ValueError):
        opt.step()
    torch.cuda.synchronize()
    assert torch.equal(whole, before)


def test_states_are_let_go():
    """Between steps only opt.state holds the moments: a program that drops them or moves them off has their memory."""
    params = params_of([1000, 300], torch.bfloat16)
    opt = optim.AdamW(params, state_bits=8, master=True, max_grad_norm=1.0, **H)
    for t in (1, 2):
        grads_in_place(params, t)
        opt.step()
    held = [weakref.ref(v) for p in params for v in opt.state[p].values() if torch.is_tensor(v)]
    opt.state.clear()
    gc.collect()
    assert all(h() is None for h in held)


def test_refused_gradients_leave_no_trace():
    """Gradients that overlap what the step writes are refused; the step after, with gradients where they were, goes on."""
    params = params_of([300, 64], torch.float32)
    opt = optim.AdamW(params, **H)
    stepped(opt, params, 1)
    good = params[0].grad
    params[0].grad = params[0].detach()[:]
    with pytest.raises(RuntimeError):
        opt.step()
    params[0].grad = good
    stepped(opt, params, 2)


def test_a_copied_optimizer_has_its_own_states():
    """copy.deepcopy of an optimizer with its parameters: both go on by themselves."""
    params = params_of([300], torch.float32)
    opt = optim.AdamW(params, **H)
    stepped(opt, params, 1)
    twin = copy.deepcopy(opt)
    others = twin.param_groups[0]["params"]
    assert others[0] is not params[0]
    stepped(opt, params, 2)
    stepped(twin, others, 2)
    assert torch.equal(params[0], others[0])


def test_plans_of_other_lists_are_let_go():
    """A list that is not stepped has no plan afterwards; parameters that took turns go on with the right moments."""
    a, b = params_of([300, 64], torch.float32), params_of([1000], torch.float32, seed=1)
    opt = optim.AdamW(a + b, **H)
    stepped(opt, a, 1)             # (b has no gradient yet)
    grads_in_place(a, 2)
    grads_in_place(b, 2)
    opt.step()
    assert len(opt._plans) == 2 and opt.state[b[0]]["step"] == 1
    main = next(plan for key, (plan, *_) in opt._plans.items() if plan.count == 2)
    b[0].grad = None
    stepped(opt, a, 3)
    assert [plan for plan, *_ in opt._plans.values()] == [main]
    for p in a:
        p.grad = None
    stepped(opt, b, 2)
    assert [plan.count for plan, *_ in opt._plans.values()] == [1]
    # b, a step behind, first in the step's order: a's plan is still a's
    opt.param_groups[0]["params"] = b + a
    for t in (4, 5):
        grads_in_place(a + b, t)
        before = columns(opt, a)
        opt.step()
        check_step(before, columns(opt, a), t, HYPER)
        kept = {plan.count: plan for plan, *_ in opt._plans.values()}
        assert len(kept) == 2 and (t == 4 or kept[2] is last)
        last = kept[2]


def test_removed_parameters_are_let_go():
    params = params_of([300, 1000], torch.float32)
    opt = optim.AdamW(params, max_grad_norm=1.0, **H)
    for t in (1, 2):
        grads_in_place(params, t)
        opt.step()
    gone = params.pop()
    held = [weakref.ref(gone)] + [weakref.ref(v) for v in opt.state[gone].values() if torch.is_tensor(v)]
    opt.param_groups[0]["params"] = params
    del opt.state[gone], gone
    grads_in_place(params, 3)
    opt.step()
    gc.collect()
    assert all(h() is None for h in held)


@pytest.mark.parametrize("kind", ["here", "torch"])
def test_a_backward_through_changed_weights_is_refused(kind):
    """As after any change in place: what autograd kept of a weight before the step is not what the step left."""
    params = params_of([300, 64], torch.float32)
    make = optim.AdamW if kind == "here" else torch.optim.AdamW
    opt = make(params, **H)
    set_grads(params, 1)
    still = params_of([64], torch.float32, seed=3)[0]
    stale = sum((p * p).sum() for p in params)
    other = (still * still).sum()
    versions = [p._version for p in params]
    opt.step()
    assert all(p._version > v for p, v in zip(params, versions))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        stale.backward()
    other.backward()
    sum((p * p).sum() for p in params).backward()


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_that_become_bf16_get_master_copies(bits):
    params = params_of(SIZES, torch.float32)
    opt = optim.AdamW(params, state_bits=bits, master=True, **H)
    stepped(opt, params, 1)
    assert all("master" not in opt.state[p] for p in params)
    for p in params:
        p.grad = None
        p.data = p.data.bfloat16()
    grads_in_place(params, 2)
    before = columns(opt, params)
    before["master"] = [w.float() for w in before["w"]]
    opt.step()
    assert all(opt.state[p]["master"].dtype == torch.float32 for p in params)
    check_step(before, columns(opt, params), 2, HYPER)
    stepped(opt, params, 3)
    again = optim.AdamW(params, state_bits=bits, master=True, **H)
    again.load_state_dict(copy.deepcopy(opt.state_dict()))
    stepped(again, params, 4)


def test_a_refused_step_holds_nothing():
    """Where a list of the step is refused, nothing is changed and the other lists' gradients are let go too."""
    a, b = params_of([300], torch.float32), params_of([64], torch.bfloat16, seed=1)
    opt = optim.AdamW(a + b, **H)
    for t in (1, 2):
        grads_in_place(a + b, t)
        opt.step()
    before = [p.detach().clone() for p in a + b]
    b[0].grad = b[0].detach()[:]
    with pytest.raises(RuntimeError):
        opt.step()
    assert all(torch.equal(p, q) for p, q in zip(a + b, before)) and opt.state[a[0]]["step"] == 2
    held = weakref.ref(a[0].grad)
    opt.zero_grad(set_to_none=True)
    assert held() is None


@pytest.mark.parametrize("bits,master", [(32, False), (8, True)])
def test_empty_parameters_and_scalars(bits, master):
    params = [torch.nn.Parameter(torch.full(shape, 0.5, device="cuda", dtype=torch.bfloat16)) for shape in ((0,), (), (3, 0), (2, 5))]
    opt = optim.AdamW(params, state_bits=bits, master=master, max_grad_norm=1.0, **H)
    for t in (1, 2):
        grads_in_place(params, t)
        before = columns(opt, params) if t > 1 else None
        opt.step()
        if before:
            for i in (1, 3):
                one = lambda s: {k: None if x is None else [x[i]] for k, x in s.items()}
                check_step(one(before), one(columns(opt, params)), t, HYPER, float(opt.grad_norm[1]))
    only = optim.AdamW(params[:1], state_bits=bits, master=master, max_grad_norm=1.0, **H)
    params[0].grad = torch.zeros_like(params[0])
    only.step()
    assert only.grad_norm.tolist() == [0.0, 1.0]
