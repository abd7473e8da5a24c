"""The C ABI of include/resbm_vocab.h and its binding on the host, without a GPU: symbols, structures, refusals (fake, aligned, never
dereferenced device addresses), workspace sizes, and the binding's checks against a stand-in for the library."""
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


def test_exports_and_layout(lib):
    src = open(os.path.join(ROOT, "include", "resbm_vocab.h")).read()
    names = sorted(set(re.findall(r"RESBM_API\s+[\w\s\*]*?\b(resbm_\w+)\s*\(", src)))
    assert sorted(resbm.VOCAB_EXPORTS) == names
    for n in names:
        assert hasattr(lib, n), n
    for n, v in re.findall(r"\b(RESBM_VOCAB_\w+) = (\d+)", src):
        assert getattr(resbm, n) == int(v)
    assert ctypes.sizeof(resbm.resbm_vocab_desc) == 72 and ctypes.sizeof(resbm.resbm_embed_desc) == 64


def loss(lib, distill=False, bwd=False, **kw):
    d = dict(T=100, V=50, d=64, ldx=64, ldw=64, K=5, dtype=1, teacher_dtype=1, temperature=1.0, dloss_each=1, flags=0)
    a = dict(X=A, W=A + BIG, target=A + 2 * BIG, teacher=A + 3 * BIG, loss=A + 4 * BIG, lse=A + 5 * BIG, dloss=A + 6 * BIG, dX=A + 7 * BIG, dW=A + 8 * BIG,
             ws=A + 9 * BIG, ws_bytes=1 << 30)
    for k, v in kw.items():
        (d if k in d else a)[k] = v
    desc = resbm.resbm_vocab_desc(*[d[k] for k, _ in resbm.resbm_vocab_desc._fields_])
    f = getattr(lib, "resbm_%s_%s" % ("distill" if distill else "linear_ce", "bwd" if bwd else "fwd"))
    args = [a["X"], a["W"], a["target"]] + ([a["teacher"]] if distill else [])
    args += [a["lse"], a["dloss"], a["dX"], a["dW"]] if bwd else [a["loss"], a["lse"]]
    return f(ctypes.byref(desc), *args, a["ws"], a["ws_bytes"], None)


BAD = [dict(T=-1), dict(V=0), dict(d=0), dict(dtype=2), dict(flags=1), dict(ldx=63), dict(ldw=0), dict(ldx=1 << 60), dict(ldw=-64),
       dict(X=None), dict(W=None), dict(target=None), dict(X=A + 1), dict(target=A + 2 * BIG + 4), dict(ws=A + 9 * BIG + 128),
       dict(lse=None), dict(lse=A + 5 * BIG + 2)]


@pytest.mark.parametrize("distill", [False, True])
@pytest.mark.parametrize("bad", BAD + [dict(loss=None), dict(loss=A + 128), dict(lse=A + BIG), dict(lse=A + 4 * BIG + 64), dict(loss=A + 2 * BIG), dict(ws=A), dict(ws=A + 4 * BIG)])
def test_forward_refuses(lib, bad, distill):
    assert loss(lib, distill, False, **bad) == INVALID


@pytest.mark.parametrize("distill", [False, True])
@pytest.mark.parametrize("bad", BAD + [dict(dloss=None), dict(dloss_each=2), dict(dloss_each=-1), dict(dX=A + 256), dict(dW=A + BIG), dict(dW=A + 7 * BIG + 64), dict(dX=A + 5 * BIG),
                                       dict(dX=A + 7 * BIG + 1), dict(ws=A + 7 * BIG), dict(dW=A + 2 * BIG)])
def test_backward_refuses(lib, bad, distill):
    assert loss(lib, distill, True, **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(K=0), dict(K=1025), dict(K=-1), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
                                 dict(teacher=None), dict(teacher_dtype=3), dict(teacher=A + 3 * BIG + 1), dict(loss=A + 3 * BIG)])
def test_distillation_refuses(lib, bad):
    assert loss(lib, True, False, **bad) == INVALID


def test_limits_and_workspaces(lib):
    for bwd in (False, True):
        assert loss(lib, bwd=bwd, ws_bytes=1000) == WORKSPACE and loss(lib, bwd=bwd, ws=None) == WORKSPACE
        for big in (dict(T=1 << 29), dict(V=1 << 29), dict(d=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), dict(T=1 << 28, V=1 << 28),
                    dict(V=1 << 28, d=1 << 12, ldx=1 << 12, ldw=1 << 12), dict(T=1 << 28, d=1 << 12, ldx=1 << 12, ldw=1 << 12)):
            assert loss(lib, bwd=bwd, **big) == UNSUPPORTED
    out = ctypes.c_size_t(7)
    desc = resbm.resbm_vocab_desc(10, 10, 10, 10, 10, 0, 1, 1, 1.0, 0, 0)
    assert lib.resbm_vocab_workspace_bytes(ctypes.byref(desc), 5, ctypes.byref(out)) == INVALID
    assert lib.resbm_vocab_workspace_bytes(ctypes.byref(desc), -1, ctypes.byref(out)) == INVALID
    assert lib.resbm_vocab_workspace_bytes(ctypes.byref(desc), resbm.RESBM_VOCAB_DISTILL_FWD, ctypes.byref(out)) == INVALID   # (K = 0)
    assert lib.resbm_vocab_workspace_bytes(None, 0, ctypes.byref(out)) == INVALID
    assert lib.resbm_vocab_workspace_bytes(ctypes.byref(desc), 0, None) == INVALID


def test_the_workspace_does_not_hold_the_logits():
    """268 MB of a piece's dz at most (to 4096 words a piece), whatever the vocabulary"""
    size = resbm.resbm_vocab_workspace_bytes
    T, d = 16384, 2048
    rest = 3 * T * d * 4                                          # the packed rows of X, dX's sums and more
    for V in (32000, 131072, 1 << 20):
        assert size(resbm.RESBM_VOCAB_CE_BWD, T, V, d) <= (1 << 28) + rest
        # forward: 16 bytes a token and 256 words, of 512 in bf16
        assert size(resbm.RESBM_VOCAB_CE_FWD, T, V, d) <= 16 * T * (V / 256 + 2) + rest
    for op in range(4):
        for T in (0, 1, 7, 300):
            for V in (1, 1000):
                for dtype in ("bf16", "f32"):
                    assert size(op, T, V, 100, dtype, 5) > 0


def embed(lib, bwd=False, **kw):
    d = dict(T=100, V=50, d=64, ldt=64, ldo=64, padding=-1, dtype=1, scale=1.0, flags=0)
    a = dict(ids=A, table=A + BIG, out=A + 2 * BIG, ws=A + 3 * BIG, ws_bytes=1 << 30)
    for k, v in kw.items():
        (d if k in d else a)[k] = v
    desc = resbm.resbm_embed_desc(*[d[k] for k, _ in resbm.resbm_embed_desc._fields_])
    if bwd:   # table: dtable, out: dout
        return lib.resbm_embed_bwd(ctypes.byref(desc), a["ids"], a["out"], a["table"], a["ws"], a["ws_bytes"], None)
    return lib.resbm_embed_fwd(ctypes.byref(desc), a["ids"], a["table"], a["out"], None)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("bad", [dict(T=-1), dict(V=0), dict(d=0), dict(dtype=2), dict(flags=1), dict(scale=float("nan")), dict(scale=float("inf")), dict(ldo=63), dict(ids=None),
                                 dict(table=None), dict(out=None), dict(ids=A + 4), dict(table=A + BIG + 1), dict(out=A + BIG + 128), dict(table=A)])
def test_embed_refuses(lib, bad, bwd):
    if bad == dict(table=A) and not bwd:
        bad = dict(out=A)
    assert embed(lib, bwd, **bad) == INVALID


def test_embed_limits(lib):
    assert embed(lib, ldt=10) == INVALID and embed(lib, True, ws=A + 3 * BIG + 8) == INVALID and embed(lib, True, ws=A + BIG) == INVALID
    assert embed(lib, True, ws=None) == WORKSPACE and embed(lib, True, ws_bytes=100) == WORKSPACE
    for bwd in (False, True):
        assert embed(lib, bwd, T=1 << 29) == UNSUPPORTED and embed(lib, bwd, V=1 << 29) == UNSUPPORTED


# ---- the binding ------------------------------------------------------------------------------------------
class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or resbm.RESBM_OK


@pytest.fixture
def fake(monkeypatch):
    lib = Library()
    monkeypatch.setattr(resbm, "_lib", lib)
    monkeypatch.setattr(resbm, "_device", lambda: torch.zeros(1).get_device())
    return lib


def tensors(T=6, V=9, d=8, K=3):
    bf = torch.bfloat16
    return dict(X=torch.zeros(T, d, dtype=bf), W=torch.zeros(V, d, dtype=bf), labels=torch.zeros(T, dtype=torch.int64), index=torch.zeros(T, K, dtype=torch.int64),
                teacher=torch.zeros(T, K), loss=torch.zeros(T), lse=torch.zeros(T), dloss=torch.zeros(T), dX=torch.zeros(T, d, dtype=bf), dW=torch.zeros(V, d, dtype=bf),
                ws=torch.zeros(64, dtype=torch.uint8))


def calls(t):
    resbm.resbm_linear_ce_fwd(t["X"], t["W"], t["labels"], t["loss"], t["lse"], t["ws"], stream=0)
    resbm.resbm_linear_ce_bwd(t["X"], t["W"], t["labels"], t["lse"], t["dloss"], t["dX"], t["dW"], t["ws"], stream=0)
    resbm.resbm_distill_fwd(t["X"], t["W"], t["index"], t["teacher"], 2.0, t["loss"], t["lse"], t["ws"], stream=0)
    resbm.resbm_distill_bwd(t["X"], t["W"], t["index"], t["teacher"], 2.0, t["lse"], t["dloss"], t["dX"], t["dW"], t["ws"], stream=0)


def test_losses_reach_the_library(fake):
    t = tensors()
    calls(t)
    assert [n for n, _ in fake.calls] == ["resbm_linear_ce_fwd", "resbm_linear_ce_bwd", "resbm_distill_fwd", "resbm_distill_bwd"]
    d = fake.calls[3][1][0]
    assert (d.T, d.V, d.d, d.ldx, d.ldw, d.K, d.dtype, d.teacher_dtype, d.temperature, d.dloss_each) == (6, 9, 8, 8, 8, 3, 1, 0, 2.0, 1)
    for one in (torch.zeros(()), torch.zeros(1)):
        calls({**t, "dloss": one})
        assert fake.calls[-1][1][0].dloss_each == 0
    wide = torch.zeros(6, 20, dtype=torch.bfloat16)
    calls({**t, "X": wide[:, 4:12], "dX": None})
    assert fake.calls[-1][1][0].ldx == 20
    one = tensors(T=1)                               # one token: a gradient for each is the one gradient
    calls(one)
    assert fake.calls[-1][1][0].ldx == 8


@pytest.mark.parametrize("name,bad", [
    ("X", torch.zeros(6, 7, dtype=torch.bfloat16)), ("X", torch.zeros(6, 8)), ("X", torch.zeros(8, 6, dtype=torch.bfloat16).t()), ("X", torch.zeros(6, 8, dtype=torch.float16)),
    ("W", torch.zeros(9, 8)), ("W", torch.zeros(8, 9, dtype=torch.bfloat16).t()), ("W", torch.zeros(0, 8, dtype=torch.bfloat16)),
    ("loss", torch.zeros(5)), ("loss", torch.zeros(6, dtype=torch.float64)), ("lse", torch.zeros(12)[::2]), ("ws", torch.zeros(1, dtype=torch.uint8).expand(1 << 20))])
def test_binding_refuses_forward(fake, name, bad):
    t = {**tensors(), name: bad}
    with pytest.raises(ValueError):
        resbm.resbm_linear_ce_fwd(t["X"], t["W"], t["labels"], t["loss"], t["lse"], t["ws"], stream=0)
    with pytest.raises(ValueError):
        resbm.resbm_distill_fwd(t["X"], t["W"], t["index"], t["teacher"], 2.0, t["loss"], t["lse"], t["ws"], stream=0)
    assert not fake.calls


@pytest.mark.parametrize("name,bad", [
    ("labels", torch.zeros(6, dtype=torch.int32)), ("labels", torch.zeros(5, dtype=torch.int64)), ("labels", torch.zeros(12, dtype=torch.int64)[::2]), ("lse", torch.zeros(5)),
    ("dloss", torch.zeros(5)), ("dloss", torch.zeros(6, dtype=torch.bfloat16)), ("dloss", torch.zeros(1).expand(6)), ("dX", torch.zeros(6, 8)),
    ("dX", torch.zeros(6, 16, dtype=torch.bfloat16)[:, :8]), ("dW", torch.zeros(8, 8, dtype=torch.bfloat16))])
def test_binding_refuses_backward(fake, name, bad):
    t = {**tensors(), name: bad}
    with pytest.raises(ValueError):
        resbm.resbm_linear_ce_bwd(t["X"], t["W"], t["labels"], t["lse"], t["dloss"], t["dX"], t["dW"], t["ws"], stream=0)
    assert not fake.calls


@pytest.mark.parametrize("name,bad", [("index", torch.zeros(6, 3, dtype=torch.int32)), ("index", torch.zeros(6, 0, dtype=torch.int64)), ("index", torch.zeros(6, dtype=torch.int64)),
                                      ("index", torch.zeros(6, 1025, dtype=torch.int64)), ("teacher", torch.zeros(6, 4)), ("teacher", torch.zeros(6, 3, dtype=torch.float16))])
def test_binding_refuses_a_teacher(fake, name, bad):
    t = {**tensors(), name: bad}
    with pytest.raises(ValueError):
        resbm.resbm_distill_fwd(t["X"], t["W"], t["index"], t["teacher"], 2.0, t["loss"], t["lse"], t["ws"], stream=0)
    assert not fake.calls


def test_binding_of_the_embedding(fake):
    ids, table, out, ws = torch.zeros(6, dtype=torch.int64), torch.zeros(9, 8), torch.zeros(6, 8), torch.zeros(64, dtype=torch.uint8)
    resbm.resbm_embed_fwd(ids, torch.zeros(9, 20)[:, :8], 2.0, torch.zeros(6, 12)[:, :8], stream=0)
    d = fake.calls[0][1][0]
    assert (d.T, d.V, d.d, d.ldt, d.ldo, d.padding, d.dtype, d.scale) == (6, 9, 8, 20, 12, -1, 0, 2.0)
    resbm.resbm_embed_bwd(ids, out, 2.0, table, ws, padding=3, stream=0)
    assert fake.calls[1][1][0].padding == 3
    fake.calls.clear()
    for bad in (dict(ids=ids.int()), dict(ids=ids[:5]), dict(ids=ids.view(6, 1)), dict(table=table.bfloat16()), dict(table=torch.zeros(9, 7)), dict(out=torch.zeros(8, 6).t()),
                dict(out=out.half())):
        a = {**dict(ids=ids, table=table, out=out), **bad}
        with pytest.raises(ValueError):
            resbm.resbm_embed_fwd(a["ids"], a["table"], 1.0, a["out"], stream=0)
        with pytest.raises(ValueError):
            resbm.resbm_embed_bwd(a["ids"], a["out"], 1.0, a["table"], ws, stream=0)
    with pytest.raises(ValueError):
        resbm.resbm_embed_bwd(ids, out, 1.0, torch.zeros(9, 16)[:, :8], ws, stream=0)
    assert not fake.calls
