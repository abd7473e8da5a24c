"""The log-sum-exp of large logits in fp32, and the probabilities that the backward forms with it, to their own rounding."""
import pytest
import torch

from test_vocab_loss_gpu import each, run

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def exact_logits(T, V, most):
    """X (T, 2), W (V, 2) whose products are exact in fp32 (8 bits a factor): logits up to `most`; the second column of W is one, X's zero."""
    g = torch.Generator(device="cuda").manual_seed(3)
    X, W = torch.zeros(T, 2, device="cuda"), torch.ones(V, 2, device="cuda")
    X[:, 0] = (most * (0.5 + 0.5 * torch.rand(T, generator=g, device="cuda"))).bfloat16().float()
    W[:, 0] = (1 - torch.rand(V, generator=g, device="cuda") / 16).bfloat16().float()
    return X, W, torch.randint(0, V, (T,), generator=g, device="cuda")


@pytest.mark.parametrize("tau", [None, 2.0])
@pytest.mark.parametrize("most", [20.0, 100.0, 1000.0])
def test_lse_and_probabilities(most, tau):
    """lse: its rounding (U of it), and 2^-20 for the exponentials and the sum. The sum of dz over the words, which the gradient's second column
    is: with the lse given, exp(z - lse) has an argument of a rounding of U |z - lse| and a product's, an exponential of 2^-22, and the sum 2^-20."""
    T, V = 3000, 400
    X, W, labels = exact_logits(T, V, most)
    g = each(T)
    if tau is None:
        loss, lse, dX, _ = run(X, W, labels, g)
    else:
        loss, lse, dX, _ = run(X, W, labels[:, None].contiguous(), g, torch.zeros(T, 1, device="cuda"), tau)
    z = X.double() @ W.double().t() / (tau or 1.0)
    want = torch.logsumexp(z, dim=1)
    assert bool(((lse.double() - want).abs() <= U * want * 1.01 + 2.0 ** -20).all()), float(((lse.double() - want).abs() / want).max() / U)
    p = torch.exp(z - lse.double()[:, None])
    total = (p.sum(dim=1) - 1) * g.double() * (tau or 1.0)
    tol = g.double().abs() * (tau or 1.0) * ((p * (z - lse.double()[:, None]).abs()).sum(dim=1) * 2 * U + 2.0 ** -20)
    off = (dX[:, 1].double() - total).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("T", [6, 120, 256])
def test_a_few_tokens_probabilities_sum_to_one(T):
    """Forward and backward form the same logits, whatever the tensor cores cut off: with the forward's lse the probabilities' sum is off by
    lse's rounding (U of it), 2^-20 for either side's exponentials and sum, and the second product's error: 2^-18 (17 MMAs' truncation,
    2 * 2^-23 each) of the sum of |dz|, 2 at most. Sums of 64 terms of about 1000 and then of nearly as much with the other sign leave
    logits of about one with an error of their own."""
    V, d = 545, 1216
    g = torch.Generator(device="cuda").manual_seed(4)
    x = 0.5 + torch.rand(T, 9, 1, 64, generator=g, device="cuda")
    w = (0.9 + 0.2 * torch.rand(V, 9, 1, 64, generator=g, device="cuda")) * (1000 / 64)
    rest = torch.randn(V, 9, 1, 64, generator=g, device="cuda") / 24
    X, W = torch.zeros(T, d, device="cuda"), torch.ones(V, d, device="cuda")
    X[:, :1152], W[:, :1152] = torch.cat((x, x), dim=2).view(T, 1152), torch.cat((w, rest - w), dim=2).view(V, 1152)
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    up = each(T)
    _, lse, dX, _ = run(X, W, labels, up)
    assert float(lse.abs().max()) < 16
    off = dX[:, -1].double().abs() / up.double().abs()
    tol = U * 16 * 1.01 + 2 * 2.0 ** -20 + 2 * 17 * 2.0 ** -22 + 4 * U
    assert bool((off <= tol).all()), float((off / tol).max())
