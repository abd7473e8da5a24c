"""resbm_add_rmsnorm_fwd over the range that the header names (a row's mean square under 1e37), and its backward over its own (1e25):
single elements whose squares leave fp32 although the row's mean does not, and rows whose sums do. The checks and tolerances
are test_add_norm_gpu's."""
import pytest
import torch

from paper_2604_11947_gb300 import pipeline, resbm
from test_add_norm_gpu import DT, check, gamma_of, outputs, run

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def outliers(T, d, dtype, size):
    """Rows of N(0, 1) with one element of `size` each, at the ends and in between"""
    gen = torch.Generator(device="cuda").manual_seed(d)
    X = torch.randn(T, d, generator=gen, device="cuda")
    for t in range(T):
        X[t, (t * (d - 1)) // max(T - 1, 1)] = size * (-1) ** t
    return X.to(DT[dtype])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 300), ("bf16", 1001), ("bf16", 4096), ("bf16", 4100), ("bf16", 32768), ("bf16", 40000),
                                     ("f32", 64), ("f32", 301), ("f32", 4096), ("f32", 16384), ("f32", 20000)])
@pytest.mark.parametrize("group", [0, 32])
def test_one_large_element(dtype, d, group):
    """|h| up to sqrt(1e37 d): 2.5e19 at d = 64"""
    T = 7
    for size in (2e19, 0.99 * (1e37 * d) ** 0.5):
        X, gamma = outliers(T, d, dtype, size), gamma_of(d, dtype)
        o = outputs(T, d, dtype, "nq", group)
        run(X, None, gamma, o, T, d, group)
        check(X, None, gamma, 1e-5, o, T, d, group)


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("bf16", 2048), ("bf16", 4097), ("bf16", 32768), ("bf16", 40000), ("f32", 1000), ("f32", 16384), ("f32", 20000)])
def test_rows_of_large_elements(dtype, d):
    T = 5
    X = torch.full((T, d), 2.9e18, device="cuda").to(DT[dtype])
    X[:, ::2] *= -1
    gamma = gamma_of(d, dtype)
    o = outputs(T, d, dtype, "hnq", 128)
    run(X, torch.zeros_like(X), gamma, o, T, d, 128)
    check(X, torch.zeros_like(X), gamma, 1e-5, o, T, d, 128)


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("bf16", 1001), ("f32", 4096), ("f32", 12001)])
def test_rows_of_small_elements(dtype, d):
    """eps = 0: mean squares down to 1e-33"""
    T = 5
    gen = torch.Generator(device="cuda").manual_seed(d)
    X = (3.3e-17 * (1 + torch.rand(T, d, generator=gen, device="cuda"))).to(DT[dtype])
    gamma = gamma_of(d, dtype)
    o = outputs(T, d, dtype, "nq", 0)
    run(X, None, gamma, o, T, d, 0, eps=0.0)
    check(X, None, gamma, 0.0, o, T, d, 0)


@pytest.mark.parametrize("d", [64, 1001, 4096, 16384])
def test_backward_of_large_rows(d):
    """fp32 rows of a mean square of 1e24 through pipeline.add_norm. The gradient is s g - h s^3 mean(g h) with g = dN gamma and
    s = 1e-12. A row's sums are chains of d / 256 terms and 13 more: L roundings, relative to the sum of the magnitudes; half of
    that and three more in s, 1.5 L + 11 in its cube, L + 2 in the other sum, and five along the way: 2.5 L + 18 of the terms'
    sizes. dgamma: L / 2 + 3 from s, two products, and the sum over the rows."""
    T, L = 6, -(-d // 256) + 13
    gen = torch.Generator(device="cuda").manual_seed(d)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, gamma, dn = (1e12 * rnd(T, d)).requires_grad_(), (1 + 0.3 * rnd(d)).requires_grad_(), rnd(T, d)
    n = pipeline.add_norm(x, None, gamma)[1]
    n.backward(dn)
    h, g = x.detach().double(), dn.double() * gamma.detach().double()
    s = (h.square().mean(dim=1, keepdim=True) + pipeline.NORM_EPS).rsqrt()
    c = s ** 3 * (g * h).mean(dim=1, keepdim=True)
    size = s * g.abs() + h.abs() * s ** 3 * (g * h).abs().mean(dim=1, keepdim=True)
    assert bool(((x.grad.double() - (s * g - h * c)).abs() <= (2.5 * L + 18) * U * size).all())
    dg = dn.double() * h * s
    assert bool(((gamma.grad.double() - dg.sum(dim=0)).abs() <= (L / 2 + T + 12) * U * dg.abs().sum(dim=0)).all())
