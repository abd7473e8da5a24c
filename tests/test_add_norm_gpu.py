"""resbm_add_rmsnorm_fwd against its definition in 64 bits.

Tolerances, from the arithmetic. H is one fp32 addition rounded once: exactly torch's. The norm is taken of H as stored,
so N, Q and S are compared with n = h s gamma of that H in 64 bits. The sum of squares has positive terms only, added in
fp32 by a thread (at most 64 of them in the register kernels, no more than 13 one after the other, for which 32 stands;
d / 1024 in the long one), then over 5 shuffles and at most 32 warps: its relative error is at most (terms + 37) 2^-24, half of that in the root; mean, eps, root, reciprocal and
the two products add six roundings. N's own rounding is half a step (2^-8 of the value for bf16, 2^-24 for fp32). A code is
off by half a step of e4m3: 2^-4 of the value, or 2^-10 of the scale below 2^-6 of it."""
import pytest
import torch

from paper_2604_11947_gb300 import resbm

pytestmark = pytest.mark.gpu
EPS = 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn


def rows(T, d, dtype, seed, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, d + pad, generator=g, device="cuda") * scale * torch.exp(torch.randn(T, 1, generator=g, device="cuda"))
    return x.to(DT[dtype])[:, :d]


def gamma_of(d, dtype, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(DT[dtype])


def call_error(d):
    """Relative error of n before its rounding"""
    return ((max(32, -(-d // 1024)) + 37) / 2 + 6) * 2.0 ** -24


def outputs(T, d, dtype, out, group, pad=0, fill=None):
    dt = DT[dtype]
    wide = lambda: torch.full((T + 2, d + pad), float("nan") if fill is None else fill, dtype=dt, device="cuda")
    o = {}
    if "h" in out:
        o["H"] = wide()
    if "n" in out:
        o["N"] = wide()
    if "q" in out:
        o["Q"] = torch.full((T + 2, d), 0x55, dtype=torch.uint8, device="cuda")
        o["S"] = torch.full((T + 2, -(-d // group) if group else 1), -7.0, device="cuda")
    return o


def check(X, A, gamma, eps, o, T, d, group):
    """The outputs (with two more rows behind them, left as they were) against 64 bits"""
    h = X if A is None else (X.float() + A.float()).to(X.dtype)
    if "H" in o:
        assert torch.equal(o["H"][:T, :d], h)
    hd = h.double()
    n = hd / (hd.square().mean(dim=1, keepdim=True) + eps).sqrt() * gamma.double()
    err = call_error(d)
    if "N" in o:
        tol = n.abs() * (torch.finfo(X.dtype).eps / 2 * (1 + 2 * err) + err) + 1e-37
        off = (o["N"][:T, :d].double() - n).abs()
        assert bool((off <= tol).all()), float((off / tol).max())
    if "Q" in o:
        g = group or d
        padded = torch.nn.functional.pad(n, (0, -d % g)).view(T, -(-d // g), g)
        S = padded.abs().amax(dim=2).clamp_min(2.0 ** -100) / 448
        assert bool(((o["S"][:T].double() - S).abs() <= S * (err + 2 * 2.0 ** -24)).all())
        per = S.repeat_interleave(g, dim=1)[:, :d]
        back = o["Q"][:T].view(E4M3).double() * o["S"][:T].double().repeat_interleave(g, dim=1)[:, :d]
        tol = torch.maximum(n.abs() * 2.0 ** -4, per * 2.0 ** -10) * (1 + 2.0 ** -10) + n.abs() * (3 * err)
        off = (back - n).abs()
        assert bool((off <= tol).all()), float((off / tol).max())
    for k, t in o.items():   # nothing behind the last row or column
        if k in ("H", "N"):
            assert bool(torch.isnan(t[T:]).all()) and bool(torch.isnan(t[:T, d:]).all()), k
    if "Q" in o:
        assert bool((o["Q"][T:] == 0x55).all()) and bool((o["S"][T:] == -7.0).all())


def run(X, A, gamma, o, T, d, group, eps=EPS):
    cut = lambda k: o[k][:T, :d] if k in o else None
    resbm.resbm_add_rmsnorm_fwd(X, A, gamma, eps, cut("H"), cut("N"), o["Q"][:T] if "Q" in o else None, o["S"][:T] if "S" in o else None,
                                group if "Q" in o else 0)


# every register form (a warp a row with 1 to 4 vectors of 16 bytes a lane, up to 512 threads a row with 3, 4 or 8 each) on
# both sides of its border, and the long one; realigned rows of 8 vectors a thread are test_add_norm_widest_gpu's
WIDTHS = [1, 2, 7, 8, 31, 32, 33, 64, 127, 128, 129, 250, 256, 264, 500, 512, 520, 1000, 1001, 1024, 1032, 2048, 2049, 2056, 4095, 4096,
          4104, 5001, 8192, 8200, 12288, 16384, 16392, 32768, 32776, 40001]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, dtype):
    T = 37 if d <= 4096 else 5
    X, A, gamma = rows(T, d, dtype, 1), rows(T, d, dtype, 2, scale=0.5), gamma_of(d, dtype)
    for group in (0, 32, 128, 1024):
        o = outputs(T, d, dtype, "hnq", group)
        run(X, A, gamma, o, T, d, group)
        check(X, A, gamma, EPS, o, T, d, group)
    assert resbm.resbm_device_error() == 0


@pytest.mark.parametrize("group", [0, 32, 64, 128, 256, 512, 2048, 1 << 20])
@pytest.mark.parametrize("dtype,d", [("bf16", 4096), ("f32", 4096), ("bf16", 1024), ("f32", 500), ("bf16", 3001), ("bf16", 200), ("f32", 33000)])
def test_groups(dtype, d, group):
    T = 19
    X, gamma = rows(T, d, dtype, 5), gamma_of(d, dtype)
    o = outputs(T, d, dtype, "q", group)
    run(X, None, gamma, o, T, d, group)
    check(X, None, gamma, EPS, o, T, d, group)


@pytest.mark.parametrize("T", [0, 1, 2, 3, 8, 9, 1000, 20011])
@pytest.mark.parametrize("out", ["hn", "n", "q", "hq", "hnq"])
def test_rows_and_outputs(T, out):
    d = 768
    X, A, gamma = rows(T, d, "bf16", 1), rows(T, d, "bf16", 2), gamma_of(d, "bf16")
    for a in (A, None):
        o = outputs(T, d, "bf16", out, 128)
        run(X, a, gamma, o, T, d, 128)
        check(X, a, gamma, EPS, o, T, d, 128)


@pytest.mark.parametrize("dtype,d,pad", [("bf16", 256, 8), ("bf16", 256, 5), ("f32", 100, 4), ("f32", 100, 3), ("bf16", 40, 1), ("bf16", 33000, 8), ("f32", 33000, 3)])
def test_strides(dtype, d, pad):
    """Rows that are slices of wider buffers, on and off the vector's alignment; nothing between the rows is written."""
    T = 21
    X, A, gamma = rows(T, d, dtype, 1, pad), rows(T, d, dtype, 2, 2 * pad), gamma_of(d, dtype)
    o = outputs(T, d, dtype, "hnq", 32, pad)
    run(X, A, gamma, o, T, d, 32)
    check(X, A, gamma, EPS, o, T, d, 32)
    # X, H and N as columns of one buffer
    buf = torch.full((T, 3 * d + pad), 9.0, dtype=DT[dtype], device="cuda")
    buf[:, :d] = X
    resbm.resbm_add_rmsnorm_fwd(buf[:, :d], A, gamma, EPS, buf[:, d:2 * d], buf[:, 2 * d:3 * d])
    assert torch.equal(buf[:, :d], X) and torch.equal(buf[:, d:2 * d], o["H"][:T, :d]) and torch.equal(buf[:, 2 * d:3 * d], o["N"][:T, :d])
    assert bool((buf[:, 3 * d:] == 9.0).all())


@pytest.mark.parametrize("dtype,d", [("bf16", 1), ("bf16", 64), ("bf16", 65), ("bf16", 300), ("bf16", 1999), ("bf16", 2048), ("bf16", 5001), ("f32", 3), ("f32", 64),
                                     ("f32", 333), ("f32", 2500)])
def test_every_alignment(dtype, d):
    """Each tensor off the vectors' alignment by its own number of elements, in rows that follow each other without a gap:
    what lies before the first row and behind the last stays."""
    T, n = 13, 8
    X, A, gamma = rows(T, d, dtype, 1), rows(T, d, dtype, 2), gamma_of(d, dtype)
    want = outputs(T, d, dtype, "hnq", 32)
    run(X, A, gamma, want, T, d, 32)
    check(X, A, gamma, EPS, want, T, d, 32)

    def at(offset, src, dt, fill):
        buf = torch.full((offset + src.numel() + 16,), fill, dtype=dt, device="cuda")
        view = buf[offset:offset + src.numel()].view(src.shape)
        view.copy_(src)
        return buf, view

    dt = DT[dtype]
    for k in range(n):
        (_, x), (_, a), (_, g) = at(k, X, dt, 3.0), at((3 * k + 1) % n, A, dt, 3.0), at((5 * k) % n, gamma, dt, 3.0)
        hb, h = at((k + 2) % n, X, dt, 5.0)
        nb, y = at((2 * k) % n, X, dt, 5.0)
        qb, q = at(k + 8, torch.zeros(T, d, dtype=torch.uint8, device="cuda"), torch.uint8, 99)
        S = torch.empty(T, -(-d // 32), device="cuda")
        resbm.resbm_add_rmsnorm_fwd(x, a, g, EPS, h, y, q, S, 32)
        assert torch.equal(h, want["H"][:T]) and torch.equal(y, want["N"][:T]) and torch.equal(q, want["Q"][:T]) and torch.equal(S, want["S"][:T])
        for buf, view, fill in ((hb, h, 5.0), (nb, y, 5.0), (qb, q, 99)):
            o = view.storage_offset()
            assert bool((buf[:o] == fill).all()) and bool((buf[o + T * d:] == fill).all())
        resbm.resbm_add_rmsnorm_fwd(x, a, g, EPS, x, None, q, S, 32)      # in place
        assert torch.equal(x, want["H"][:T])


@pytest.mark.parametrize("dtype,d", [("bf16", 512), ("f32", 77), ("bf16", 4096), ("bf16", 34000)])
def test_in_place_and_broadcast(dtype, d):
    T = 50
    X, A, gamma = rows(T, d, dtype, 1), rows(T, d, dtype, 2), gamma_of(d, dtype)
    o = outputs(T, d, dtype, "hnq", 0)
    run(X, A, gamma, o, T, d, 0)
    for which in ("X", "A"):
        x, a = X.clone(), A.clone()
        o2 = outputs(T, d, dtype, "nq", 0)
        resbm.resbm_add_rmsnorm_fwd(x, a, gamma, EPS, x if which == "X" else a, o2["N"][:T], o2["Q"][:T], o2["S"][:T], 0)
        assert torch.equal(x if which == "X" else a, o["H"][:T]) and torch.equal(a if which == "X" else x, A if which == "X" else X)
        assert torch.equal(o2["N"][:T], o["N"][:T]) and torch.equal(o2["Q"], o["Q"]) and torch.equal(o2["S"], o["S"])
    both = X.clone()   # x + x, in place of both
    n = torch.empty_like(both)
    resbm.resbm_add_rmsnorm_fwd(both, both, gamma, EPS, both, n)
    assert torch.equal(both, (X.float() * 2).to(X.dtype))
    one = A[:1].expand(T, d)   # one row for all tokens
    o3 = outputs(T, d, dtype, "hn", 0)
    run(X, one, gamma, o3, T, d, 0)
    check(X, one, gamma, EPS, o3, T, d, 0)


def test_rows_of_zeros_and_extremes():
    d = 512
    X = torch.zeros(6, d, dtype=torch.bfloat16, device="cuda")
    X[1] = 1e-30
    X[2] = 1e18          # squares reach 1e36: within fp32
    X[3, ::2] = -3.0
    X[4, 7] = float("inf")
    X[5, 9] = float("nan")
    gamma = gamma_of(d, "bf16")
    o = outputs(6, d, "bf16", "nq", 128)
    run(X, None, gamma, o, 6, d, 128)
    check(X[:4], None, gamma, EPS, {"N": torch.cat((o["N"][:4], o["N"][6:])), "Q": torch.cat((o["Q"][:4], o["Q"][6:])),
                                    "S": torch.cat((o["S"][:4], o["S"][6:]))}, 4, d, 128)
    assert bool((o["N"][0] == 0).all()) and bool((o["Q"][0] & 0x7F == 0).all()) and bool((o["S"][0] > 0).all())
    # an infinity: 1 / rms = 0, so 0 but for the infinity's own NaN; the group that holds it reads back as NaN
    n = o["N"][4].float()
    assert bool(torch.isnan(n[7])) and bool((n[torch.arange(d, device="cuda") != 7] == 0).all())
    back = o["Q"][4].view(E4M3).float() * o["S"][4].repeat_interleave(128)
    assert bool(torch.isnan(back[:128]).all()) and bool((back[128:] == 0).all())
    assert bool(torch.isnan(o["N"][5].float()).all()) and bool(torch.isnan(o["Q"][5].view(E4M3).float() * o["S"][5].repeat_interleave(128)).all())
    # eps = 0 and a row of zeros: 0 / 0
    resbm.resbm_add_rmsnorm_fwd(X[:1], None, gamma, 0.0, None, o["N"][:1])
    assert bool(torch.isnan(o["N"][0].float()).all())


def test_stream_graph_and_repeat():
    """On a stream of its own, captured and replayed with other inputs, and bit for bit the same again."""
    T, d = 300, 1536
    X, A, gamma = rows(T, d, "bf16", 1), rows(T, d, "bf16", 2), gamma_of(d, "bf16")
    o = outputs(T, d, "bf16", "hnq", 128)
    run(X, A, gamma, o, T, d, 128)
    want = {k: v.clone() for k, v in o.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2 = outputs(T, d, "bf16", "hnq", 128)
    with torch.cuda.stream(side):
        run(X, A, gamma, o2, T, d, 128)
    side.synchronize()
    x, a = torch.zeros_like(X), torch.zeros_like(A)
    o3 = outputs(T, d, "bf16", "hnq", 128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(x, a, gamma, o3, T, d, 128)
    x.copy_(X)
    a.copy_(A)
    graph.replay()
    torch.cuda.synchronize()
    for got in (o2, o3):
        for k in want:
            assert torch.equal(got[k][:T].view(torch.uint8), want[k][:T].view(torch.uint8)), k


def test_binding_refusals():
    X, gamma = rows(4, 64, "bf16", 1), gamma_of(64, "bf16")
    N = torch.empty_like(X)
    S, Q = torch.empty(4, 1, device="cuda"), torch.empty(4, 64, dtype=E4M3, device="cuda")
    fn = resbm.resbm_add_rmsnorm_fwd
    for args in ((X[0], None, gamma, EPS, None, N), (X, X[:3], gamma, EPS, None, N), (X, None, gamma[:32], EPS, None, N), (X, None, gamma, EPS, None, N.float()),
                 (X, None, gamma.float(), EPS, None, N), (X.half(), None, gamma.half(), EPS, None, N.half()), (X, None, gamma, EPS, None, None, Q, None),
                 (X, None, gamma, EPS, None, None, Q, S, 32), (X, None, gamma, EPS, None, None, Q[:, :32], S), (X, None, gamma, EPS, None, None, N, S),
                 (X.cpu(), None, gamma, EPS, None, N), (X, None, gamma, EPS, None, N.cpu()), (X.t(), None, gamma[:4], EPS, None, N.t())):
        with pytest.raises(ValueError):
            fn(*args)
    for args in ((X, None, gamma, -1.0, None, N), (X, None, gamma, EPS, X, None), (X, None, gamma, EPS, None, X), (X, None, gamma, EPS, N, N),
                 (X, None, gamma, EPS, None, None, Q, torch.empty(4, 4, device="cuda"), 16)):
        with pytest.raises((resbm.ResbmError, ValueError)):
            fn(*args)


@pytest.mark.parametrize("d", [4096, 4097])
def test_offsets_past_32_bits(d):
    """Over 2^31 elements: the first and the last rows."""
    T = (1 << 31) // d + 777
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB")
    X, A = (torch.zeros(T, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    spots = (slice(0, 50), slice(T - 800, T))
    for i, at in enumerate(spots):
        k = X[at].shape[0]
        X[at], A[at] = rows(k, d, "bf16", i), rows(k, d, "bf16", 5 + i)
    gamma = gamma_of(d, "bf16")
    o = {"H": torch.empty_like(X), "N": torch.empty_like(X), "Q": torch.empty(T, d, dtype=torch.uint8, device="cuda"), "S": torch.empty(T, -(-d // 128), device="cuda")}
    resbm.resbm_add_rmsnorm_fwd(X, A, gamma, EPS, o["H"], o["N"], o["Q"], o["S"], 128)
    pad = {"H": float("nan"), "N": float("nan"), "Q": 0x55, "S": -7.0}   # (check() looks at two rows behind as well)
    for at in spots:
        k = X[at].shape[0]
        part = {n: torch.cat((t[at], torch.full((2, t.shape[1]), pad[n], device="cuda").to(t.dtype))) for n, t in o.items()}
        check(X[at], A[at], gamma, EPS, part, k, d, 128)
