"""Batches of which few tokens have a target: their gradients are those of these tokens alone, as exact as in a call of their own
(tolerances: vocab_helpers, of a call over these tokens)."""
import pytest
import torch

import vocab_helpers as vh
from test_vocab_loss_gpu import each, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n,V,d", [(17, 1, 1000, 264), (40, 3, 500, 65), (121, 16, 2000, 520), (300, 2, 3000, 1024), (600, 16, 1001, 2056), (5000, 1, 9000, 136), (4096, 2, 32000, 2048),
                                     (300, 17, 3000, 264), (20000, 5, 13001, 64)])
def test_few_labels(T, n, V, d, dtype):
    X, W, labels = vh.inputs(T, V, d, dtype, seed=n, ignored=0.0)
    used = torch.randperm(T, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")[:n].sort().values
    some = torch.full_like(labels, -100)
    some[used] = labels[used]
    X = torch.where((some >= 0)[:, None], X, float("nan"))
    want, g = vh.ce(X[used], W, labels[used]), each(T)
    loss, lse, dX, dW = run(X, W, some, g)
    want.check_fwd(loss[used], lse[used])
    want.check_bwd(g[used], dX[used], dW)
    others = some < 0
    assert bool((loss[others] == 0).all()) and bool((dX[others] == 0).all())
    for dx, dw in ((True, False), (False, True)):
        _, _, one, two = run(X, W, some, g, dx=dx, dw=dw)
        assert torch.equal(one, dX) if dx else torch.equal(two, dW)


@pytest.mark.parametrize("T,n,V,d,K", [(300, 2, 3000, 264, 7), (5000, 11, 700, 1100, 5)])
def test_few_targets_of_a_teacher(T, n, V, d, K):
    X, W, _ = vh.inputs(T, V, d, seed=n, ignored=0.0)
    index, teacher = vh.entries(T, V, K, empty=0.0, missing=0.0)
    used = torch.arange(n, device="cuda") * (T // n) + 3
    some = torch.full_like(index, -1)
    some[used] = index[used]
    want, g = vh.distill(X[used], W, index[used], teacher[used], 2.0), each(T)
    loss, lse, dX, dW = run(X, W, some, g, teacher, 2.0)
    want.check_fwd(loss[used], lse[used])
    want.check_bwd(g[used], dX[used], dW)
    assert int((dX != 0).any(dim=1).sum()) == n
