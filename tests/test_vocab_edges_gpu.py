"""The losses over the vocabulary off the plain case: tokens without targets, what masked places hold, strides and alignment, large logits,
pieces of the vocabulary, offsets past 32 bits, streams and graphs, and their gradients against differences."""
import pytest
import torch

import vocab_helpers as vh
from paper_2604_11947_gb300 import resbm
from test_vocab_loss_gpu import each, run, workspace

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def same(a, b):
    return all(x is None or y is None or torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 40, 600])
def test_no_token_has_a_target(T, dtype):
    X, W, labels = vh.inputs(T, 300, 72, dtype)
    X = torch.full_like(X, float("nan"))
    loss, lse, dX, dW = run(X, W, torch.full_like(labels, -1), each(T))
    assert all(bool((t == 0).all()) for t in (loss, lse, dX, dW))
    index, teacher = vh.entries(T, 300, 5, dtype, empty=1.1)
    loss, lse, dX, dW = run(X, W, index, each(T), teacher, 2.0)
    assert all(bool((t == 0).all()) for t in (loss, lse, dX, dW))


def test_no_tokens():
    X, W, labels = vh.inputs(0, 300, 72)
    _, _, dX, dW = run(X, W, labels, torch.zeros(1, device="cuda"))
    assert dX.shape == (0, 72) and bool((dW == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [9, 300])
def test_what_tokens_without_a_target_hold(T, dtype):
    """NaN and infinities there reach nothing: the same bits as with zeros."""
    X, W, labels = vh.inputs(T, 500, 136, dtype, ignored=0.4)
    labels[0], labels[1] = 3, -1
    clean = torch.where((labels >= 0)[:, None], X, 0.0)
    for bad in (float("nan"), float("inf"), -float("inf")):
        dirty = torch.where((labels >= 0)[:, None], X, bad)
        assert same(run(dirty, W, labels, each(T)), run(clean, W, labels, each(T)))
    index, teacher = vh.entries(T, 500, 7, dtype, empty=0.4)
    has = (index >= 0).any(dim=1)
    dirty = torch.where(has[:, None], X, float("nan"))
    dirty_teacher = torch.where(index >= 0, teacher, float("nan"))
    assert same(run(dirty, W, index, each(T), dirty_teacher), run(torch.where(has[:, None], X, 0.0), W, index, each(T), teacher))


def test_a_nan_stays_in_its_row():
    X, W, labels = vh.inputs(400, 300, 72, ignored=0.0)
    X[5, 3] = float("nan")
    loss, lse, dX, dW = run(X, W, labels, each(400))
    others = torch.arange(400, device="cuda") != 5
    assert bool(torch.isnan(loss[5])) and bool(torch.isfinite(loss[others]).all()) and bool(torch.isfinite(dX[others]).all())
    assert bool(torch.isnan(dX[5]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_targets_past_the_vocabulary(dtype):
    X, W, labels = vh.inputs(300, 257, 72, dtype, ignored=0.0)
    for far in (257, 300, 511, 1 << 31, 1 << 40):
        labels[7] = far
        loss, lse, dX, dW = run(X, W, labels, each(300))
        others = torch.arange(300, device="cuda") != 7
        assert bool(torch.isnan(loss[7])) and bool(torch.isfinite(loss[others]).all()) and bool(torch.isfinite(lse).all())
        assert bool(torch.isnan(dX[7]).all()) and bool(torch.isfinite(dX[others]).all()) and bool(torch.isnan(dW).all())
        index, teacher = vh.entries(300, 257, 4, dtype, missing=0, empty=0)
        index[7, 2] = far
        loss, lse, dX, _ = run(X, W, index, each(300), teacher)
        assert bool(torch.isnan(loss[7])) and bool(torch.isfinite(loss[others]).all()) and bool(torch.isnan(dX[7]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,wpad", [(8, 0), (5, 0), (0, 8), (0, 3), (3, 5), (24, 40)])
def test_strides(pad, wpad, dtype):
    for T, V, d in ((33, 700, 64), (700, 300, 136), (5, 999, 200)):
        X, W, labels = vh.inputs(T, V, d, dtype, pad=pad, wpad=wpad)
        got = run(X, W, labels, each(T))
        vh.ce(X, W, labels).check_fwd(*got[:2])
        vh.ce(X, W, labels).check_bwd(each(T), *got[2:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_addresses_off_the_vectors(dtype):
    """Tensors that begin one element into an allocation"""
    T, V, d = 300, 700, 72
    shift = lambda t: torch.cat((t.new_zeros(1), t.reshape(-1)))[1:].view(t.shape)
    X, W, labels = vh.inputs(T, V, d, dtype)
    want = vh.ce(X, W, labels)
    X, W = shift(X), shift(W)
    loss, lse = shift(torch.empty(T, device="cuda")), shift(torch.empty(T, device="cuda"))
    dX, dW = shift(torch.empty_like(X)), shift(torch.empty_like(W))
    ws = workspace(T, V, d, dtype)[:-512]
    resbm.resbm_linear_ce_fwd(X, W, labels, loss, lse, ws)
    resbm.resbm_linear_ce_bwd(X, W, labels, lse, each(T), dX, dW, ws)
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)


@pytest.mark.parametrize("T,V", [(1, 300), (40, 1)])
def test_the_stride_of_a_single_row(T, V):
    """Whatever it is, it is not used."""
    X, W, labels = vh.inputs(T, V, 72, ignored=0.0)
    X, W = X.contiguous(), W.contiguous()
    want, lib = run(X, W, labels, each(T)), resbm.load()
    ws = workspace(T, V, 72, "bf16")[:-512]
    for ld in (0, 1, -5, 73, 1 << 50):
        loss, lse, dX, dW, g = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(X), torch.empty_like(W), each(T)
        desc = resbm.resbm_vocab_desc(T, V, 72, ld if T == 1 else 72, ld if V == 1 else 72, 0, 1, 0, 1.0, 1, 0)
        p, s = (lambda t: t.data_ptr()), torch.cuda.current_stream().cuda_stream
        assert lib.resbm_linear_ce_fwd(desc, p(X), p(W), p(labels), p(loss), p(lse), p(ws), ws.numel(), s) == 0
        assert lib.resbm_linear_ce_bwd(desc, p(X), p(W), p(labels), p(lse), p(g), p(dX), p(dW), p(ws), ws.numel(), s) == 0
        torch.cuda.synchronize()
        assert same((loss, lse, dX, dW), want)


def test_one_gradient_for_all_losses():
    X, W, labels = vh.inputs(300, 700, 72)
    for one in (torch.tensor(0.37, device="cuda"), torch.tensor([0.37], device="cuda")):
        assert same(run(X, W, labels, one), run(X, W, labels, torch.full((300,), 0.37, device="cuda")))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", [(300, 700, 72), (20, 5000, 256), (2000, 256, 512)])
def test_one_of_the_gradients(T, V, d, dtype):
    """Either alone: the same values (fp32 sums may be cut at other places), within the same tolerance"""
    X, W, labels = vh.inputs(T, V, d, dtype)
    want = vh.ce(X, W, labels)
    both = run(X, W, labels, each(T))
    for dx, dw in ((True, False), (False, True)):
        got = run(X, W, labels, each(T), dx=dx, dw=dw)
        want.check_bwd(each(T), *got[2:])
        assert same(got, both)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_bits_every_time(dtype):
    X, W, labels = vh.inputs(1500, 3000, 200, dtype)
    first = run(X, W, labels, each(1500))
    for fill in (0, 0x7F):
        ws = workspace(1500, 3000, 200, dtype)
        ws[:-512] = fill
        assert same(run(X, W, labels, each(1500), ws=ws), first)
    index, teacher = vh.entries(1500, 3000, 9, dtype)
    assert same(run(X, W, index, each(1500), teacher, 2.0), run(X, W, index, each(1500), teacher, 2.0))


@pytest.mark.parametrize("T,V,d", [(300, 20011, 1000), (300, 20011, 1001), (2000, 6000, 520), (5, 30000, 264)])
def test_units_of_both_gradients_in_one_warp(T, V, d):
    """The same bits, and right ones, many times over: a warp stores units of dX (fp32) and of dW after one another."""
    X, W, labels = vh.inputs(T, V, d)
    want = vh.ce(X, W, labels)
    first = run(X, W, labels, each(T))
    want.check_bwd(each(T), *first[2:])
    for _ in range(25):
        assert same(run(X, W, labels, each(T)), first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(dtype):
    """Logits of thousands: the maximum is taken out before the exponentials."""
    X, W, labels = vh.inputs(200, 600, 128, dtype)
    X = (X.float() * 500).to(X.dtype)
    want = vh.ce(X, W, labels)
    assert float(want.z.abs().max()) > 2000
    got = run(X, W, labels, each(200))
    want.check_fwd(*got[:2])
    assert all(bool(torch.isfinite(t).all()) for t in got)
    index, teacher = vh.entries(200, 600, 5, dtype)
    want = vh.distill(X, W, index, teacher, 0.05)
    want.check_fwd(*run(X, W, index, each(200), teacher, 0.05)[:2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_of_the_vocabulary(dtype):
    """More than one piece: dX is added up over them, in the last one the words end."""
    T, V, d = 20000, 13001, 64
    X, W, labels = vh.inputs(T, V, d, dtype)
    labels[:4] = torch.tensor([0, V - 1, V // 2, 8191], device="cuda")
    got = run(X, W, labels, each(T))
    want = vh.ce(X, W, labels)
    want.check_fwd(*got[:2])
    want.check_bwd(each(T), *got[2:])


def test_pieces_of_a_head_off_the_vectors():
    X, W, labels = vh.inputs(500, 9001, 64, wpad=3)
    got = run(X, W, labels, each(500))
    want = vh.ce(X, W, labels)
    want.check_fwd(*got[:2])
    want.check_bwd(each(500), *got[2:])


def test_offsets_past_32_bits():
    """600000 tokens: a piece's dz has 2.46e9 elements."""
    T, V, d = 600_000, 4100, 64
    X, W, labels = vh.inputs(T, V, d, ignored=0.01)
    dloss = torch.full((1,), 1.0 / T, device="cuda")
    ws = torch.empty(max(resbm.resbm_vocab_workspace_bytes(k, T, V, d) for k in (0, 1)), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    resbm.resbm_linear_ce_fwd(X, W, labels, loss, lse, ws)
    resbm.resbm_linear_ce_bwd(X, W, labels, lse, dloss, dX, dW, ws)
    want, tol = torch.zeros(V, d, dtype=torch.float64, device="cuda"), torch.zeros(V, d, dtype=torch.float64, device="cuda")
    for t in range(0, T, 20000):
        part = slice(t, t + 20000)
        ref = vh.ce(X[part], W, labels[part])
        ref.check_fwd(loss[part], lse[part])
        ref.check_bwd(dloss, dX[part], None)
        dz, err = ref.grads(dloss)
        want += dz.t() @ ref.X
        tol += (err + vh._acc(T, False) * (dz.abs() + err)).t() @ ref.X.abs()
    tol = (tol + 2.0 ** -8 * (want.abs() + tol)) * 1.001
    assert bool(((dW.double() - want).abs() <= tol).all())
    assert resbm.resbm_device_error() == 0


def test_teachers():
    T, V, d, K = 300, 500, 72, 6
    X, W, labels = vh.inputs(T, V, d, ignored=0.0)
    index, teacher = vh.entries(T, V, K, "f32")                   # a teacher in another type than the student
    got = run(X, W, index, each(T), teacher, 2.0)
    want = vh.distill(X, W, index, teacher, 2.0)
    want.check_fwd(*got[:2])
    want.check_bwd(each(T), *got[2:])
    index[:, 3] = index[:, 1]                                     # the same word twice counts twice
    teacher[:, 4] = float("-inf")                                 # an entry of no weight
    teacher[:, 0] = 5.0                                           # (and one of some)
    index[:, 0] = torch.randint(0, V, (T,), device="cuda")
    got = run(X, W, index, each(T), teacher, 1.0)
    want = vh.distill(X, W, index, teacher, 1.0)
    want.check_fwd(*got[:2])
    want.check_bwd(each(T), *got[2:])
    # one entry at temperature 1 is a label
    one, logit = labels[:, None].contiguous(), torch.full((T, 1), 3.0, device="cuda")
    a, b = run(X, W, one, each(T), logit, 1.0), run(X, W, labels, each(T))
    assert same(a[1:], b[1:])
    assert bool(((a[0] - b[0]).abs() <= 8 * U * (b[1].abs() + 20)).all())   # (sums of the same terms in another order)


@pytest.mark.parametrize("which", ["ce", "distill"])
def test_gradients_against_differences(which):
    """The change of the kernel's own losses along a direction. Allowed: the losses' errors over the step, what the central difference
    leaves out (from the formula in 64 bits) and the gradient's own error, all from vocab_helpers."""
    T, V, d, h = 40, 200, 48, 2.0 ** -6
    X, W, labels = vh.inputs(T, V, d, "f32")
    index, teacher = vh.entries(T, V, 5, "f32")
    ref = (lambda x, w: vh.ce(x, w, labels)) if which == "ce" else (lambda x, w: vh.distill(x, w, index, teacher, 2.0))
    call = (lambda x, w: run(x, w, labels, g)) if which == "ce" else (lambda x, w: run(x, w, index, g, teacher, 2.0))
    g = each(T)
    _, _, dX, dW = call(X, W)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for k in range(4):
        A = torch.randn(T, d, generator=gen, device="cuda").sign() if k % 2 == 0 else torch.zeros(T, d, device="cuda")
        B = torch.randn(V, d, generator=gen, device="cuda").sign() / 8 if k % 2 else torch.zeros(V, d, device="cuda")
        up, down = (X + h * A, W + h * B), (X - h * A, W - h * B)
        ru, rd = ref(*up), ref(*down)
        w64 = lambda l: float((l.double() * g.double()).sum())
        change = (w64(call(*up)[0]) - w64(call(*down)[0])) / (2 * h)
        slope = float((dX.double() * A.double()).sum() + (dW.double() * B.double()).sum())
        base = ref(X, W)
        dz, err = base.grads(g)
        true = float(((dz @ base.W) * A.double()).sum() + ((dz.t() @ base.X) * B.double()).sum())
        losses = float((g.double().abs() * torch.where(base.has, ru.loss_err + rd.loss_err, 0.0)).sum()) / (2 * h)
        left_out = abs((w64(ru.loss) - w64(rd.loss)) / (2 * h) - true)
        total = dz.abs() + err
        own = float((((err + vh._acc(V, True) * total) @ base.W.abs()) * A.double().abs()).sum()
                    + (((err + vh._acc(T, True) * total).t() @ base.X.abs()) * B.double().abs()).sum()) * 1.01
        assert abs(change - slope) <= losses + left_out + own, (change, slope, losses, left_out, own)


def test_another_stream_and_two_at_once():
    X, W, labels = vh.inputs(700, 3000, 136)
    want = run(X, W, labels, each(700))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            loss, lse = torch.empty(700, device="cuda"), torch.empty(700, device="cuda")
            dX, dW, ws = torch.empty_like(X), torch.empty_like(W), workspace(700, 3000, 136, "bf16")[:-512]
            for _ in range(3):
                resbm.resbm_linear_ce_fwd(X, W, labels, loss, lse, ws)
                resbm.resbm_linear_ce_bwd(X, W, labels, lse, each(700), dX, dW, ws)
            outs.append((loss, lse, dX, dW))
    torch.cuda.synchronize()
    assert all(same(o, want) for o in outs)


def test_two_graphs_that_share_a_workspace():
    """Captured calls, replayed one after the other with other inputs and another number of tokens in use"""
    T, V, d = 600, 2000, 136
    ws = workspace(T, V, d, "bf16")[:-512]
    made, g = [], each(T)   # (g: one for both graphs, alive as long as they are)
    for seed in (1, 2):
        X, W, labels = (t.contiguous() for t in vh.inputs(T, V, d, seed=seed))
        loss, lse, dX, dW = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(X), torch.empty_like(W)
        call = lambda: (resbm.resbm_linear_ce_fwd(X, W, labels, loss, lse, ws), resbm.resbm_linear_ce_bwd(X, W, labels, lse, g, dX, dW, ws))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call()
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        made.append((graph, X, W, labels, (loss, lse, dX, dW)))
    for seed, ignored in ((3, 0.1), (4, 0.9), (5, 0.0)):
        for graph, X, W, labels, out in made:
            for dst, src in zip((X, W, labels), vh.inputs(T, V, d, seed=seed, ignored=ignored)):
                dst.copy_(src)
            graph.replay()
        torch.cuda.synchronize()
        for graph, X, W, labels, out in made:
            assert same(out, run(X, W, labels, each(T)))
