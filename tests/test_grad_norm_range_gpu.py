"""resbm_grad_norm at the ends of fp32's squares, as the header states them."""
import pytest
import torch

from paper_2604_11947_gb300 import resbm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def norm(grads):
    plan = resbm.AdamWPlan(None, grads)
    out = torch.full((2,), -1.0, device="cuda")
    resbm.resbm_grad_norm(plan, 1.0, out, resbm.grad_norm_workspace(plan))
    return out.tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 7, 5000, 100_001])
def test_small_gradients(dtype, n):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = 1 + torch.rand(n, generator=gen, device="cuda")
    for size, tol in ((2e-19, 20 * U),              # squares are normal numbers
                      (1e-20, 2.0 ** -17),          # of 1e-40 and more, off by half a denormal (2^-150) each: 2^-17
                      (1e-24, None)):               # under half the smallest denormal
        g = (size * x).to(dtype)
        want = float(g.double().square().sum().sqrt())
        got, coef = norm([g])
        assert coef == 1.0
        if tol is None:
            assert got == 0.0
        else:
            assert abs(got - want) <= (tol + 20 * U) * want, (size, got, want)
    # beside others they are what they are to the sum: nothing
    both = norm([(1e-24 * x).to(dtype), torch.ones(3, device="cuda", dtype=dtype)])[0]
    assert abs(both - 3 ** 0.5) <= 4 * U * 3 ** 0.5


def test_large_gradients():
    for size, finite in ((1.8e19, True), (1.9e19, False)):
        got, coef = norm([torch.full((1,), size, device="cuda")])
        assert (abs(got - size) <= 4 * U * size and abs(coef * size - 1) < 1e-5) if finite else (got == float("inf") and coef != coef)
