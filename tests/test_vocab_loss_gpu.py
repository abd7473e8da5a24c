"""resbm_linear_ce_* and resbm_distill_* against their formulas in 64 bits (tolerances: vocab_helpers)."""
import math

import pytest
import torch

import vocab_helpers as vh
from paper_2604_11947_gb300 import resbm

pytestmark = pytest.mark.gpu


def workspace(T, V, d, dtype, K=0):
    kinds = (resbm.RESBM_VOCAB_DISTILL_FWD, resbm.RESBM_VOCAB_DISTILL_BWD) if K else (resbm.RESBM_VOCAB_CE_FWD, resbm.RESBM_VOCAB_CE_BWD)
    n = max(resbm.resbm_vocab_workspace_bytes(k, T, V, d, dtype, K) for k in kinds)
    return torch.full((n + 512,), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN bytes: nothing is read before it is written)


def guarded(*shape, dtype=torch.float32, fill=7.0):
    """A dense tensor between two guards, and a check that the guards are as they were"""
    n = math.prod(shape)
    buf = torch.full((n + 512,), fill, dtype=dtype, device="cuda")

    def intact():
        assert bool((buf[:256] == fill).all()) and bool((buf[256 + n:] == fill).all())
    return buf[256:256 + n].view(shape), intact


def run(X, W, target, dloss, teacher=None, tau=1.0, dx=True, dw=True, ws=None):
    T, d = X.shape
    V = W.shape[0]
    dtype = "bf16" if X.dtype == torch.bfloat16 else "f32"
    ws = workspace(T, V, d, dtype, 0 if teacher is None else target.shape[1]) if ws is None else ws
    used = ws[:ws.numel() - 512]
    (loss, g1), (lse, g2) = guarded(T), guarded(T)
    (dX, g3), (dW, g4) = guarded(T, d, dtype=X.dtype), guarded(V, d, dtype=X.dtype)
    if teacher is None:
        resbm.resbm_linear_ce_fwd(X, W, target, loss, lse, used)
        resbm.resbm_linear_ce_bwd(X, W, target, lse, dloss, dX if dx else None, dW if dw else None, used)
    else:
        resbm.resbm_distill_fwd(X, W, target, teacher, tau, loss, lse, used)
        resbm.resbm_distill_bwd(X, W, target, teacher, tau, lse, dloss, dX if dx else None, dW if dw else None, used)
    torch.cuda.synchronize()
    for g in (g1, g2, g3, g4):
        g()
    assert bool((ws[-512:] == 0xFF).all())
    assert resbm.resbm_device_error() == 0
    return loss, lse, dX if dx else None, dW if dw else None


def each(T, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(T, generator=g, device="cuda")


SIZES = [(1, 1, 1), (1, 64, 64), (2, 300, 8), (3, 33, 40), (17, 1000, 100), (64, 257, 72), (255, 512, 256), (256, 511, 264), (257, 513, 1000),
         (300, 5000, 65), (600, 96, 200), (1000, 2049, 512), (130, 20011, 328), (4100, 300, 130), (1, 5003, 2056),
         # a handful of tokens, on and off the vectors, and both sides of where dz has two parts
         (1, 3001, 4096), (1, 700, 4104), (2, 1001, 1000), (4, 2000, 2048), (4, 999, 4095), (5, 1000, 2048), (7, 777, 2047), (8, 5000, 256), (8, 300, 3100),
         (8, 40, 4096), (9, 500, 512), (3, 200, 9000), (16, 9000, 520), (17, 9000, 520), (13, 32000, 1001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", SIZES)
def test_cross_entropy(T, V, d, dtype):
    X, W, labels = vh.inputs(T, V, d, dtype, seed=T + V + d)
    want = vh.ce(X, W, labels)
    loss, lse, dX, dW = run(X, W, labels, each(T))
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d,K,tau", [(1, 64, 64, 1, 1.0), (5, 40, 33, 40, 0.7), (200, 1000, 72, 7, 2.0), (300, 700, 128, 64, 1.0), (257, 3000, 100, 128, 3.0),
                                         (20, 2000, 64, 1024, 1.0), (40, 600, 56, 300, 2.0), (700, 90, 72, 33, 1.5)])
def test_distillation(T, V, d, K, tau, dtype):
    X, W, _ = vh.inputs(T, V, d, dtype, seed=K)
    index, teacher = vh.entries(T, V, K, dtype, seed=K)
    want = vh.distill(X, W, index, teacher, tau)
    loss, lse, dX, dW = run(X, W, index, each(T), teacher, tau)
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)
