"""The C ABI of include/resbm_train.h on the host, without a GPU: the library exports every declared function, its
structures have the header's layout, and bad arguments are refused before the device is touched (fake, aligned,
never dereferenced device addresses)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2604_11947_gb300 import build, resbm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, BIG = 1 << 40, 1 << 34
INVALID, WORKSPACE, UNSUPPORTED = resbm.RESBM_ERR_INVALID_ARG, resbm.RESBM_ERR_WORKSPACE, resbm.RESBM_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build()
    return resbm.load()


def test_exports_every_declared_symbol(lib):
    src = open(os.path.join(ROOT, "include", "resbm_train.h")).read()
    names = sorted(set(re.findall(r"RESBM_API\s+[\w\s\*]*?\b(resbm_\w+)\s*\(", src)))
    assert sorted(resbm.TRAIN_EXPORTS) == names
    for n in names:
        assert hasattr(lib, n), n
    assert int(re.search(r"RESBM_STATE_BLOCK (\d+)", src).group(1)) == resbm.RESBM_STATE_BLOCK
    for n, v in re.findall(r"\b(RESBM_STATE_(?:NONE|F32|E4M3)) = (\d+)", src):
        assert getattr(resbm, n) == int(v)


def test_struct_layout_matches_header():
    assert ctypes.sizeof(resbm.resbm_add_norm_desc) == 6 * 8 + 4 * 4
    assert ctypes.sizeof(resbm.resbm_adamw_desc) == 16
    assert ctypes.sizeof(resbm.resbm_adamw_tensor) == 64
    assert ctypes.sizeof(resbm.resbm_adamw_hyper) == 5 * 8 + 8 + 3 * 8


def norm(lib, X=A, Am=A + BIG, gamma=A + 2 * BIG, H=A + 3 * BIG, N=A + 4 * BIG, Q=None, S=None, **kw):
    d = dict(T=100, d=64, ldx=64, lda=64, ldh=64, ldn=64, dtype=1, q_group=0, eps=1e-5, flags=0)
    d.update(kw)
    desc = resbm.resbm_add_norm_desc(*[d[k] for k, _ in resbm.resbm_add_norm_desc._fields_])
    return lib.resbm_add_rmsnorm_fwd(ctypes.byref(desc), X, Am, gamma, H, N, Q, S, None)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(d=0), dict(d=1 << 30), dict(dtype=2), dict(flags=1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(X=None), dict(gamma=None), dict(N=None), dict(X=A + 1), dict(N=A + 4 * BIG + 1), dict(dtype=0, gamma=A + 2 * BIG + 2),
    dict(Q=A + 5 * BIG), dict(S=A + 5 * BIG), dict(Q=A + 5 * BIG, S=A + 6 * BIG + 2),
    dict(Q=A + 5 * BIG, S=A + 6 * BIG, q_group=16), dict(Q=A + 5 * BIG, S=A + 6 * BIG, q_group=96), dict(Q=A + 5 * BIG, S=A + 6 * BIG, q_group=-32),
    dict(ldx=63), dict(lda=-64), dict(ldh=0), dict(ldn=32), dict(ldn=1 << 60), dict(T=1 << 40, ldx=1 << 40),
    dict(N=A + 128), dict(H=A + 128), dict(N=A + 2 * BIG), dict(N=A + 3 * BIG), dict(H=A, ldh=128), dict(H=A + BIG + 64),
    dict(Q=A + 4 * BIG, S=A + 6 * BIG), dict(Q=A + 5 * BIG, S=A + 5 * BIG + 64), dict(Q=A + 64, S=A + 6 * BIG),
    dict(H=A, ldx=0, ldh=64),                                         # in place over one row read by every token
    dict(X=A, ldx=128, N=A + 64, ldn=128),                            # columns 32 .. 96 of a buffer whose 0 .. 64 are read
    dict(X=A + 128, ldx=128, N=A + 64, ldn=128),                      # the same from the other side
])
def test_add_norm_refuses(lib, bad):
    assert norm(lib, **bad) == INVALID


def test_add_norm_null_desc(lib):
    assert lib.resbm_add_rmsnorm_fwd(None, A, None, A + BIG, None, A + 2 * BIG, None, None, None) == INVALID


def tensors(n, count=1, **kw):
    t = (resbm.resbm_adamw_tensor * max(count, 1))()
    for i in range(count):
        for k, name in enumerate(("w", "g", "m", "v")):
            setattr(t[i], name, A + (8 * i + k) * BIG)
        t[i].n = n
    for k, v in kw.items():
        setattr(t[0], k, v)
    return t


def plan(lib, t, count=1, w=1, g=1, state=32, flags=0, plan_bytes=None):
    size = ctypes.c_size_t(0)
    assert lib.resbm_adamw_plan_bytes(count, ctypes.byref(size)) == resbm.RESBM_OK
    buf = (ctypes.c_uint64 * (size.value // 8 + 1))()
    st = lib.resbm_adamw_plan(ctypes.byref(resbm.resbm_adamw_desc(w, g, state, flags)), t, count, ctypes.addressof(buf),
                              size.value if plan_bytes is None else plan_bytes)
    return st, buf


def test_plan_accepts(lib):
    assert plan(lib, tensors(1000))[0] == resbm.RESBM_OK
    assert plan(lib, tensors(1000, 1000), 1000)[0] == resbm.RESBM_OK
    assert plan(lib, tensors(0, 3, w=None, g=None), 3)[0] == resbm.RESBM_OK          # empty tensors have no pointers
    assert plan(lib, tensors(5), 0)[0] == resbm.RESBM_OK
    assert plan(lib, tensors(1000, master=A + 6 * BIG))[0] == resbm.RESBM_OK
    assert plan(lib, tensors(1000, m_scale=A + 6 * BIG, v_scale=A + 7 * BIG), state=8)[0] == resbm.RESBM_OK
    shared = tensors(1000, 2)
    shared[1].g = shared[0].g                                                      # gradients may be shared
    assert plan(lib, shared, 2)[0] == resbm.RESBM_OK
    assert plan(lib, tensors(1000, w=None, m=None, v=None), state=0)[0] == resbm.RESBM_OK
    # neighbours touch without overlapping
    t = tensors(256, 2)
    t[1].w = t[0].w + 512
    assert plan(lib, t, 2)[0] == resbm.RESBM_OK


@pytest.mark.parametrize("bad", [
    dict(kw=dict(w=None)), dict(kw=dict(g=None)), dict(kw=dict(m=None)), dict(kw=dict(v=None)), dict(kw=dict(w=A + 1)), dict(kw=dict(m=A + 2 * BIG + 2)),
    dict(kw=dict(master=A + 6 * BIG + 2)), dict(n=-1), dict(w=2), dict(g=-1), dict(state=16), dict(flags=1),
    dict(kw=dict(master=A + 6 * BIG), w=0), dict(kw=dict(m_scale=A + 6 * BIG, v_scale=A + 7 * BIG)), dict(state=8),
    dict(state=8, kw=dict(m_scale=A + 6 * BIG)), dict(state=8, kw=dict(m_scale=A + 6 * BIG + 1, v_scale=A + 7 * BIG)),
    dict(kw=dict(m=A + 64)), dict(kw=dict(g=A + 2 * BIG + 64)), dict(kw=dict(v=A + 2 * BIG)),
    dict(state=8, kw=dict(m_scale=A + 6 * BIG, v_scale=A + 6 * BIG + 12)),         # 1000 elements: 4 blocks, 16 bytes of scales
    dict(count=2, second=dict(w=A)), dict(count=2, second=dict(m=A + 2 * BIG)), dict(count=2, second=dict(g=A)),
    dict(count=2, kw=dict(master=A + 6 * BIG)),                                    # one with a master copy, one without
])
def test_plan_refuses(lib, bad):
    count = bad.get("count", 1)
    t = tensors(bad.get("n", 1000), count, **bad.get("kw", {}))
    for k, v in bad.get("second", {}).items():
        setattr(t[1], k, v)
    st, buf = plan(lib, t, count, bad.get("w", 1), bad.get("g", 1), bad.get("state", 32), bad.get("flags", 0))
    assert st == INVALID
    # what was refused is no plan
    hyper = resbm.resbm_adamw_hyper(1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None)
    assert lib.resbm_adamw_step(ctypes.addressof(buf), ctypes.byref(hyper), None) == INVALID


def test_plan_sizes(lib):
    size = ctypes.c_size_t(0)
    assert lib.resbm_adamw_plan_bytes(-1, ctypes.byref(size)) == INVALID
    assert lib.resbm_adamw_plan_bytes(1, None) == INVALID
    assert plan(lib, tensors(10), plan_bytes=100)[0] == WORKSPACE
    assert plan(lib, tensors(1 << 41))[0] == UNSUPPORTED
    assert plan(lib, tensors((1 << 40) - 5, 2), 2)[0] in (UNSUPPORTED, INVALID)
    d = resbm.resbm_adamw_desc(1, 1, 32, 0)
    assert lib.resbm_adamw_plan(ctypes.byref(d), tensors(10), 1, None, 1 << 20) == INVALID
    assert lib.resbm_adamw_plan(None, tensors(10), 1, A, 1 << 20) == INVALID
    assert lib.resbm_adamw_plan(ctypes.byref(d), None, 1, A, 1 << 20) == INVALID


@pytest.mark.parametrize("bad", [dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta2=-0.1), dict(beta2=float("nan")),
                                 dict(eps=-1e-8), dict(weight_decay=-1.0), dict(step=0), dict(lr_dev=A + 2), dict(step_dev=A + 4), dict(grad_scale=A + 1)])
def test_step_refuses(lib, bad):
    st, buf = plan(lib, tensors(1000))
    assert st == resbm.RESBM_OK
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, lr_dev=None, step_dev=None, grad_scale=None)
    h.update(bad)
    hyper = resbm.resbm_adamw_hyper(*h.values())
    assert lib.resbm_adamw_step(ctypes.addressof(buf), ctypes.byref(hyper), None) == INVALID


def test_step_wants_a_plan_with_states(lib):
    hyper = resbm.resbm_adamw_hyper(1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None)
    zeros = (ctypes.c_uint64 * 1024)()
    assert lib.resbm_adamw_step(None, ctypes.byref(hyper), None) == INVALID
    assert lib.resbm_adamw_step(ctypes.addressof(zeros), ctypes.byref(hyper), None) == INVALID
    st, buf = plan(lib, tensors(1000), state=0)
    assert st == resbm.RESBM_OK
    assert lib.resbm_adamw_step(ctypes.addressof(buf), ctypes.byref(hyper), None) == INVALID
    assert lib.resbm_adamw_step(ctypes.addressof(plan(lib, tensors(1000))[1]), None, None) == INVALID


def test_grad_norm_refuses(lib):
    st, buf = plan(lib, tensors(1_000_000, 3), 3)
    assert st == resbm.RESBM_OK
    p = (ctypes.c_void_p * 1)(ctypes.addressof(buf))
    size = ctypes.c_size_t(0)
    assert lib.resbm_grad_norm_workspace_bytes(p, 1, ctypes.byref(size)) == resbm.RESBM_OK and size.value > 0
    need, out, ws = size.value, A, A + BIG
    zeros = (ctypes.c_uint64 * 1024)()
    none = (ctypes.c_void_p * 1)(ctypes.addressof(zeros))
    assert lib.resbm_grad_norm_workspace_bytes(none, 1, ctypes.byref(size)) == INVALID
    assert lib.resbm_grad_norm_workspace_bytes(p, 1, None) == INVALID
    fn = lib.resbm_grad_norm
    assert fn(none, 1, 1.0, out, ws, need, None) == INVALID
    assert fn(p, -1, 1.0, out, ws, need, None) == INVALID
    assert fn(None, 1, 1.0, out, ws, need, None) == INVALID
    for bad in (-1.0, float("nan"), float("inf")):
        assert fn(p, 1, bad, out, ws, need, None) == INVALID
    assert fn(p, 1, 1.0, None, ws, need, None) == INVALID
    assert fn(p, 1, 1.0, out + 2, ws, need, None) == INVALID
    assert fn(p, 1, 1.0, out, None, need, None) == WORKSPACE
    assert fn(p, 1, 1.0, out, ws, need - 1, None) == WORKSPACE
    assert fn(p, 1, 1.0, out, ws + 8, need, None) == INVALID
    assert fn(p, 1, 1.0, ws + 8, ws, need, None) == INVALID


def test_binding_refuses_host_tensors(lib):
    """The binding's own checks: tensors that are not on the device never reach the library."""
    if torch.cuda.is_available():
        pytest.skip("the checks of a host without a GPU")
    x, g = torch.zeros(4, 8), torch.ones(8)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        resbm.resbm_add_rmsnorm_fwd(x, None, g, 1e-5, None, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        resbm.resbm_add_rmsnorm_fwd(torch.zeros(8), None, g, 1e-5, None, torch.zeros(8))
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        resbm.AdamWPlan([x], [x], [x], [x])
