"""resbm_embed_fwd and resbm_embed_bwd against their formulas in 64 bits.

The forward product is exact in fp32 up to its rounding (2^-24), and the output's (half a step of its type) on top. A word's
gradient is a sum of n rows in fp32: in its order, at most n + n / 32 additions, each off by 2^-24 of the terms' absolute sum, then the
product with the scale and the output's rounding."""
import pytest
import torch

from paper_2604_11947_gb300 import resbm

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def ids_of(T, V, kind, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "same":
        return torch.full((T,), V // 3, device="cuda")
    if kind == "few":
        return torch.randint(0, min(V, 5), (T,), generator=g, device="cuda")
    if kind == "runs":   # words that begin and end at and around the blocks' borders
        return torch.arange(T, device="cuda").div(31, rounding_mode="floor").flip(0) % V
    return torch.randint(0, V, (T,), generator=g, device="cuda")


def rows(T, d, dtype, pad=0, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(T, d + pad, generator=g, device="cuda").to(DT[dtype])[:, :d]


def backward(ids, dout, scale, V, padding=-1):
    T, d = dout.shape
    dtype = "bf16" if dout.dtype == torch.bfloat16 else "f32"
    n = resbm.resbm_vocab_workspace_bytes(resbm.RESBM_VOCAB_EMBED_BWD, T, V, d, dtype)
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    buf = torch.full((V * d + 512,), 7.0, dtype=dout.dtype, device="cuda")
    dtable = buf[256:256 + V * d].view(V, d)
    resbm.resbm_embed_bwd(ids, dout, scale, dtable, ws[:n], padding=padding)
    torch.cuda.synchronize()
    assert bool((buf[:256] == 7).all()) and bool((buf[256 + V * d:] == 7).all()) and bool((ws[n:] == 0xFF).all())
    return dtable


def check_backward(dtable, ids, dout, scale, V, padding=-1):
    keep = (ids != padding) & (ids >= 0) & (ids < V)
    d = dout.shape[1]
    g = torch.where(keep[:, None], dout.double(), 0.0)
    at = torch.where(keep, ids, 0)
    want = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, at, g) * scale
    mass = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, at, g.abs()) * abs(scale)
    n = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at, keep.double())[:, None]
    tol = mass * (n * 33 / 32 + 3) * U
    tol = tol + (want.abs() + tol) * torch.finfo(dout.dtype).eps / 2 + 1e-37
    off = (dtable.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    assert bool((dtable[n[:, 0] == 0] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (8, 100, 4096), (33, 7, 3), (1000, 257, 64), (777, 5000, 1003), (4097, 513, 100), (20, 50, 5000), (3, 4, 2056)])
def test_forward(T, V, d, dtype):
    for pad in (0, 8, 5):
        table, ids = rows(V, d, dtype, pad), ids_of(T, V, "any")
        for scale in (1.0, 31.67):
            out = torch.full((T + 1, d + pad), 7.0, dtype=DT[dtype], device="cuda")
            resbm.resbm_embed_fwd(ids, table, scale, out[:T, :d])
            assert torch.equal(out[:T, :d], (table[ids].float() * scale).to(DT[dtype]))   # one product in fp32, one rounding
            assert bool((out[T:] == 7).all()) and bool((out[:, d:] == 7).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["any", "same", "few", "runs"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (2, 100, 64), (31, 7, 8), (32, 40, 100), (33, 3, 33), (64, 1000, 256), (1000, 257, 72), (5000, 511, 40), (4096, 512, 1000),
                                   (9000, 40000, 24), (300, 70000, 2056), (100, 300000, 16), (20, 50, 5000)])
def test_backward(T, V, d, kind, dtype):
    ids, dout = ids_of(T, V, kind, T), rows(T, d, dtype)
    check_backward(backward(ids, dout, 2.5, V), ids, dout, 2.5, V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_backward_padding_strides_and_strangers(dtype):
    T, V, d = 3000, 400, 120
    for pad in (0, 8, 3):
        ids, dout = ids_of(T, V, "few"), rows(T, d, dtype, pad)
        ids[::7], ids[::11], ids[5], ids[6] = V, -3, 1 << 40, -(1 << 50)   # outside the table: nothing
        dout[::7] = float("nan")
        dout[::11] = float("inf")
        dout[5:7] = float("nan")
        ids[3::13] = 399
        dout[3::13] = float("nan")                                        # what padding tokens hold reaches nothing
        check_backward(backward(ids, torch.where((ids == 399)[:, None] | (ids < 0)[:, None] | (ids >= V)[:, None], dout, dout), 1.0, V, 399),
                       torch.where(ids == 399, -1, ids), torch.nan_to_num(dout, nan=0.0, posinf=0.0), 1.0, V)


def test_backward_padding_only_and_empty():
    dout = rows(100, 64, "bf16")
    ids = torch.full((100,), 9, device="cuda")
    assert bool((backward(ids, dout, 1.0, 50, padding=9) == 0).all())
    assert bool((backward(ids[:0], dout[:0], 1.0, 50) == 0).all())


def test_forward_strangers_and_empty():
    table = rows(10, 64, "bf16")
    ids = torch.tensor([3, -1, 10, 1 << 40, 9], device="cuda")
    out = torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda")
    resbm.resbm_embed_fwd(ids, table, 1.0, out)
    assert torch.isnan(out).all(dim=1).tolist() == [False, True, True, True, False]
    assert torch.equal(out[0], table[3]) and torch.equal(out[4], table[9])
    resbm.resbm_embed_fwd(ids[:0], table, 1.0, out[:0])


def test_backward_is_reproducible():
    ids, dout = ids_of(20000, 300, "any"), rows(20000, 136, "bf16")
    first = backward(ids, dout, 1.0, 300)
    for _ in range(3):
        assert torch.equal(backward(ids, dout, 1.0, 300), first)


def test_large_sort():
    """Several rounds a warp in the sort"""
    ids, dout = ids_of(200000, 260000, "any"), rows(200000, 8, "f32")
    check_backward(backward(ids, dout, 1.0, 260000), ids, dout, 1.0, 260000)
