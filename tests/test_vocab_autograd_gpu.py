"""pipeline.embed, linear_cross_entropy and distillation as autograd functions, and the model that uses them."""
import pytest
import torch
import torch.nn.functional as Fn

import vocab_helpers as vh
from paper_2604_11947_gb300 import pipeline, resbm

pytestmark = pytest.mark.gpu
CFG = pipeline.PipelineConfig(layers=4, d=256, heads=4, ffn=512, vocab=1000, stages=2, r=16, m=16, batch=3, seq=40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_cross_entropy_and_its_gradients(dtype, reduction):
    X, W, labels = vh.inputs(60, 300, 72, dtype)
    x, w = X.clone().view(3, 20, 72).requires_grad_(), W.clone().requires_grad_()
    loss = pipeline.linear_cross_entropy(x, w, labels.view(3, 20), reduction)
    up = torch.randn(loss.shape, device="cuda")
    loss.backward(up)
    want = vh.ce(X, W, labels)
    n = int((labels >= 0).sum())
    if reduction == "none":
        want.check_fwd(loss.detach().view(-1), want.lse)
        g = up.view(-1)
    else:
        k = n if reduction == "mean" else 1
        assert abs(float(loss) - float(want.loss.sum()) / k) <= float(torch.where(want.has, want.loss_err, 0.0).sum()) / k + 60 * vh.U * float(want.loss.abs().sum()) / k
        g = (up / k).expand(60)
    want.check_bwd(g.contiguous(), x.grad.view(60, 72), w.grad)


def test_distillation_and_its_gradients():
    X, W, _ = vh.inputs(60, 300, 72)
    index, teacher = vh.entries(60, 300, 6)
    x, w = X.clone().view(3, 20, 72).requires_grad_(), W.clone().requires_grad_()
    loss = pipeline.distillation(x, w, index.view(3, 20, 6), teacher.view(3, 20, 6), 2.0, "none")
    loss.backward(torch.ones_like(loss))
    want = vh.distill(X, W, index, teacher, 2.0)
    want.check_fwd(loss.detach().view(-1), want.lse)
    want.check_bwd(torch.ones(60, device="cuda"), x.grad.view(60, 72), w.grad)


def test_inputs_out_of_the_ordinary():
    X, W, labels = vh.inputs(60, 300, 72)
    for frozen in range(2):   # one of the two needs no gradient; a strided input; twice the same backward
        x, w = X.clone().requires_grad_(frozen == 0), W.clone().requires_grad_(frozen == 1)
        loss = pipeline.linear_cross_entropy(x, w, labels)
        loss.backward(retain_graph=True)
        first = (x if frozen == 0 else w).grad.clone()
        loss.backward()
        assert torch.equal((x if frozen == 0 else w).grad, first + first)
        assert (w if frozen == 0 else x).grad is None
    wide = torch.randn(3, 20, 150, device="cuda", dtype=torch.bfloat16)
    a = pipeline.linear_cross_entropy(wide[..., 10:82], W, labels.view(3, 20), "none")
    b = pipeline.linear_cross_entropy(wide[..., 10:82].contiguous(), W, labels.view(3, 20), "none")
    assert torch.equal(a, b)
    t = wide[0, :, :72].t().contiguous().t()          # columns before rows
    assert torch.equal(pipeline.linear_cross_entropy(t, W, labels[:20], "none"), pipeline.linear_cross_entropy(t.contiguous(), W, labels[:20], "none"))
    row = X[:1].clone().requires_grad_()              # one row for all tokens: its gradient is the rows' sum
    pipeline.linear_cross_entropy(row.expand(60, 72), W, labels, "sum").backward()
    each = X[:1].expand(60, 72).contiguous().requires_grad_()
    pipeline.linear_cross_entropy(each, W, labels, "sum").backward()
    off = (row.grad.double() - each.grad.double().sum(dim=0)).abs()
    assert bool((off <= each.grad.double().abs().sum(dim=0) * 60 * 2.0 ** -8).all())   # (60 additions, rounded to bf16 at worst each)
    table = torch.randn(9, 72, device="cuda").requires_grad_()
    ids = torch.arange(12, device="cuda") % 9
    pipeline.embed(ids, table).backward(torch.ones(72, device="cuda").expand(12, 72))   # a gradient of one row for all tokens
    assert torch.equal(table.grad, torch.where(torch.arange(9, device="cuda") < 3, 2.0, 1.0)[:, None].expand(9, 72))
    empty = pipeline.linear_cross_entropy(X[:0].clone().requires_grad_(), W, labels[:0])
    empty.backward()
    assert float(empty) == 0.0
    none = pipeline.linear_cross_entropy(X, W, torch.full_like(labels, -100))
    assert float(none) == 0.0
    with pytest.raises(ValueError):
        pipeline.linear_cross_entropy(X, W, labels[:30])
    with pytest.raises(ValueError):
        pipeline.linear_cross_entropy(X, W, labels, "median")
    with pytest.raises(ValueError):
        pipeline.distillation(X, W, labels[:, None], torch.zeros(60, 2, device="cuda"))
    with pytest.raises(ValueError):
        pipeline.linear_cross_entropy(X, W.float(), labels)


def test_inputs_that_change_before_the_backward():
    X, W, labels = vh.inputs(60, 300, 72)
    x, w = X.clone().requires_grad_(), W.clone().requires_grad_()
    loss = pipeline.linear_cross_entropy(x, w, labels)
    with torch.no_grad():
        w.mul_(2.0)
    with pytest.raises(RuntimeError):
        loss.backward()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_embed(dtype):
    table = torch.randn(50, 72, device="cuda").to(dtype).requires_grad_()
    ids = torch.randint(0, 50, (4, 30), device="cuda")
    out = pipeline.embed(ids, table, 3.0, padding=7)
    assert torch.equal(out, (table.detach()[ids].float() * 3.0).to(dtype))
    up = torch.randn_like(out)
    out.backward(up)
    keep = (ids != 7).reshape(-1, 1)
    terms = torch.where(keep, up.reshape(-1, 72).double(), 0.0)
    want = torch.zeros(50, 72, dtype=torch.float64, device="cuda").index_add_(0, ids.reshape(-1), terms) * 3
    mass = torch.zeros(50, 72, dtype=torch.float64, device="cuda").index_add_(0, ids.reshape(-1), terms.abs()) * 3
    tol = mass * 127 * vh.U + want.abs() * vh.half_step(dtype) * 1.01 + mass * 127 * vh.U * vh.half_step(dtype)
    assert bool(((table.grad.double() - want).abs() <= tol).all())


def _losses(cfg, tokens):
    model = pipeline.PipelineModel(cfg)
    loss = pipeline.train_step(model, tokens)
    return model, loss.detach()


@pytest.mark.parametrize("cfg", [CFG, CFG.with_(fuse_add_norm=True), CFG.with_(stages=1)])
def test_the_model_with_its_ends_in_the_library(cfg):
    """The hidden states are the same bits with either embedding; the fused loss is the formula's on them, and its gradients are
    the formula's."""
    tokens = pipeline.synthetic_tokens(cfg)
    model, loss = _losses(cfg.with_(fuse_vocab=True), tokens)
    plain, _ = _losses(cfg, tokens)
    with torch.no_grad():
        last = model.hidden(tokens)
        assert torch.equal(last, plain.hidden(tokens))
    labels = pipeline.next_tokens(tokens).reshape(-1)
    want = vh.ce(last.reshape(-1, cfg.d), model.head.detach(), labels)
    n = int((labels >= 0).sum())
    assert n == cfg.batch * (cfg.seq - 1)
    assert abs(float(loss) - float(want.loss.sum()) / n) <= float(want.loss_err.max()) + 8 * vh.U * float(want.loss.max())
    g = torch.full((cfg.tokens,), 1.0 / n, device="cuda")
    want.check_bwd(g, None, model.head.grad)
    for p in model.parameters():
        assert p.grad is not None and bool(torch.isfinite(p.grad.float()).all())
    assert resbm.resbm_device_error() == 0


def test_distillation_of_a_model_from_another():
    """The student's loss is the formula's on its hidden states and the teacher's top logits; a teacher teaches itself nothing:
    all of its own logits at any temperature leave a loss of the logits' rounding (bf16: half a step of 2^-8)."""
    tokens = pipeline.synthetic_tokens(CFG)
    teacher, student = pipeline.PipelineModel(CFG.with_(stages=1, seed=3)), pipeline.PipelineModel(CFG)
    index, top = teacher.top_logits(tokens, 8, rows=50)
    with torch.no_grad():
        logits = Fn.linear(teacher.hidden(tokens), teacher.head)
    assert index.shape == (3, 40, 8) and torch.equal(top, logits.gather(2, index)) and torch.equal(top[..., 0], logits.amax(dim=-1))
    loss = student.distill(tokens, index, top, 2.0)
    loss.backward()
    with torch.no_grad():
        last = student.hidden(tokens).reshape(-1, CFG.d)
    want = vh.distill(last, student.head.detach(), index.view(-1, 8), top.view(-1, 8), 2.0)
    assert abs(float(loss) - float(want.loss.mean())) <= float(want.loss_err.max()) + 8 * vh.U * float(want.loss.max())
    want.check_bwd(torch.full((CFG.tokens,), 1.0 / CFG.tokens, device="cuda"), None, student.head.grad)
    assert all(p.grad is not None for n, p in student.named_parameters())


def test_a_captured_step():
    """The forward and backward of the ends in a graph, replayed with other tokens"""
    V, d = 500, 136
    table = (torch.randn(V, d, device="cuda") / 8).bfloat16()
    ids, labels = torch.randint(0, V, (200,), device="cuda"), torch.randint(0, V, (200,), device="cuda")

    def step(t):
        x = pipeline.embed(ids, t, 2.0)
        loss = pipeline.linear_cross_entropy(x, t, labels)      # tied: the table is the head too
        return loss, *torch.autograd.grad(loss, t)

    leaf = table.clone().requires_grad_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(leaf)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(leaf)
    for seed in range(3):
        torch.manual_seed(seed)
        ids.copy_(torch.randint(0, V, (200,)))
        labels.copy_(torch.randint(-2, V, (200,)))
        graph.replay()
        want = step(table.clone().requires_grad_())
        assert all(torch.equal(a, b) for a, b in zip(out, want))
