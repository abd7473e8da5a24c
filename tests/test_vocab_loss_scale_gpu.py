"""Losses' gradients that tokens have in common: not rounded with dz (tolerances: vocab_helpers, but for the means derived here)."""
import pytest
import torch

import vocab_helpers as vh
from paper_2604_11947_gb300 import pipeline
from test_vocab_loss_gpu import each, run

pytestmark = pytest.mark.gpu


def uncertain(T, V, d, seed=1):
    """Hidden states that know nothing of the label: p of about 1 / V"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    X = (torch.randn(T, d, generator=g, device="cuda") / 8).bfloat16()
    W = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).bfloat16()
    return X, W, torch.randint(0, V, (T,), generator=g, device="cuda")


def check_means(X, W, labels, g, dX, dW):
    """Rounding errors have no sign over the elements: the part of the exact gradient that is missing or too much,
    <off, want> / <want, want>, has as allowed error
      the outputs' rounding: 2^-8 of an element, independent: 2^-8 / sqrt(tokens d) at one standard deviation and below, five of them allowed
      the label's dz, 1 - p of it: rounded it is off by p at most where p is under 2^-9, with one sign
      the other words' dz, in sum as large as the label's in absolute value, but in norm sqrt(V) less: 2^-8 / sqrt(V tokens), five of them
      the logits and the exponentials: 2^-14"""
    want = vh.ce(X, W, labels)
    dz, _ = want.grads(g)
    n, d, V = int(want.has.sum()), X.shape[1], W.shape[0]
    p = float(want.p[want.has].max())
    assert p < 2.0 ** -9
    bound = 5 * 2.0 ** -8 / (n * d) ** 0.5 + p + 5 * 2.0 ** -8 / (n * V) ** 0.5 + 2.0 ** -14
    for got, exact in ((dX, dz @ want.W), (dW, dz.t() @ want.X)):
        share = float(((got.double() - exact) * exact).sum() / (exact * exact).sum())
        assert abs(share) <= bound, (share, bound)
    assert bound < 2.0 ** -10   # (the rounding of 1 / 24, 1 / 200 and 0.083 to bf16 is off by 2^-9 and more of them)


@pytest.mark.parametrize("T,V,d,g", [(24, 24141, 1240, 1 / 24), (200, 5000, 264, 1 / 200), (300, 3000, 1000, 0.083), (9000, 2500, 136, -1 / 24), (300, 9001, 65, 1 / 24)])
def test_one_factor_of_all_losses(T, V, d, g):
    X, W, labels = uncertain(T, V, d)
    _, _, dX, dW = run(X, W, labels, torch.full((1,), g, device="cuda"))
    check_means(X, W, labels, torch.full((T,), g, device="cuda"), dX, dW)
    vh.ce(X, W, labels).check_bwd(torch.full((T,), g, device="cuda"), dX, dW)
    # the same number for each, and other ones where there is no label
    other = torch.randperm(T, device="cuda")[:T // 5]
    some, each_of = labels.clone(), torch.full((T,), g, device="cuda")
    some[other], each_of[other] = -100, 1e30
    _, _, dX, dW = run(X, W, some, each_of)
    check_means(X, W, some, torch.where(some >= 0, g, 0.0), dX, dW)


def test_the_mean_of_the_pipelines_loss():
    X, W, labels = uncertain(120, 4000, 520)
    labels[::6] = -1
    x, w = X.clone().requires_grad_(), W.clone().requires_grad_()
    pipeline.linear_cross_entropy(x, w, labels).backward()
    check_means(X, W, labels, torch.full((120,), 1 / 100, device="cuda"), x.grad, w.grad)


@pytest.mark.parametrize("T", [60, 5000])
def test_gradients_out_of_the_ordinary(T):
    """Zeros, infinities and NaN among the losses' gradients: a token's row of dX is its own affair."""
    X, W, labels = vh.inputs(T, 300, 72, ignored=0.2)
    labels[:6] = 5
    plain = each(T)
    for scale in (0.0, 1e-30, 1e30):
        g = plain * scale
        _, _, dX, dW = run(X, W, labels, g)
        vh.ce(X, W, labels).check_bwd(g, dX, dW)
    g = plain.clone()
    g[2], g[3], g[4] = torch.nan, torch.inf, 0.0
    g[labels < 0] = torch.nan
    _, _, dX, dW = run(X, W, labels, g)
    rows = torch.arange(T, device="cuda")
    fine = (labels >= 0) & (rows != 2) & (rows != 3)
    vh.ce(X[fine], W, labels[fine]).check_bwd(g[fine], dX[fine], None)
    assert bool(torch.isnan(dX[2]).all()) and not bool(torch.isfinite(dX[3]).any()) and bool((dX[4] == 0).all()) and bool((dX[labels < 0] == 0).all())
    for one in (torch.inf, torch.nan):   # (what 1 / n is without a label)
        _, _, dX, dW = run(X, W, torch.full_like(labels, -1), torch.full((1,), one, device="cuda"))
        assert bool((dX == 0).all()) and bool((dW == 0).all())
        assert all(bool((t == 0).all()) for t in run(X, W, torch.full_like(labels, -1), torch.full((T,), one, device="cuda"))[2:])
