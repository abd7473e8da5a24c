"""pipeline.add_norm where its inputs are out of the ordinary: no tokens, one input twice, one row, strided and broadcast inputs,
gradients that arrive strided."""
import pytest
import torch

from paper_2604_11947_gb300 import pipeline
from test_optim_gpu import reference

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def leaves(*shapes, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(7)
    return [torch.randn(*s, generator=gen, device="cuda").to(dtype).requires_grad_() for s in shapes]


def tolerance(d, wd, dn, gamma):
    """test_add_norm_gradients': fp32 sums of at most d / 32 + 80 operations, relative to the terms' size"""
    return U * wd.abs() + (d / 32 + 80) * U * (wd.abs().amax() + 4 * dn.abs().amax() * gamma.abs().amax())


@pytest.mark.parametrize("shape", [(0, 64), (0, 7, 33), (2, 0, 64)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_tokens(shape, dtype):
    x, a, gamma = leaves(shape, shape, shape[-1:], dtype=dtype)
    h, n = pipeline.add_norm(x, a, gamma)
    assert h.shape == n.shape == shape
    (h.sum() + n.sum()).backward()
    assert x.grad.shape == a.grad.shape == shape and bool((gamma.grad == 0).all())


def test_one_input_twice():
    T, d = 9, 200
    x, gamma, dh, dn = leaves((T, d), (d,), (T, d), (T, d))
    h, n = pipeline.add_norm(x, x, gamma)
    torch.autograd.backward((h, n), (dh.detach(), dn.detach()))
    _, _, wd, _ = reference(x.detach(), x.detach(), gamma.detach(), dh.detach(), dn.detach())
    assert bool(((x.grad.double() - 2 * wd).abs() <= 2 * tolerance(d, wd, dn.detach(), gamma.detach())).all())


def test_the_two_gradients_are_apart():
    """x and a get equal gradients in memory of their own: scaling one leaves the other."""
    x, a, gamma = leaves((5, 64), (5, 64), (64,))
    h, n = pipeline.add_norm(x, a, gamma)
    (h.sum() + (n * n).sum()).backward()
    want = x.grad.clone()
    x.grad.mul_(3.0)
    assert torch.equal(a.grad, want)


@pytest.mark.parametrize("shape", [(64,), (1, 64), (3, 4, 65)])
def test_shapes(shape):
    d = shape[-1]
    x, a, gamma, dh, dn = leaves(shape, shape, (d,), shape, shape)
    h, n = pipeline.add_norm(x, a, gamma)
    torch.autograd.backward((h, n), (dh.detach(), dn.detach()))
    flat = lambda t: t.detach().reshape(-1, d)
    wh, wn, wd, _ = reference(*[flat(t) for t in (x, a)], gamma.detach(), flat(dh), flat(dn))
    assert h.shape == n.shape == shape and torch.equal(flat(h).double(), wh)
    assert bool(((flat(n).double() - wn).abs() <= (d / 32 + 80) * U * (wn.abs() + 1)).all())
    assert bool(((flat(x.grad).double() - wd).abs() <= tolerance(d, wd, dn.detach(), gamma.detach())).all()) and torch.equal(x.grad, a.grad)


def test_strided_inputs_and_gradients():
    """x and a as columns of wider buffers and transposed, gradients that are expanded or transposed"""
    T, d = 12, 48
    wide, turned, gamma = leaves((T, 2 * d + 5), (d, T), (d,))
    x, a = wide[:, 3:3 + d], turned.t()
    h, n = pipeline.add_norm(x, a, gamma)
    row, col = (t.detach() for t in leaves((1, d), (d, T)))
    torch.autograd.backward((h, n), (row.expand(T, d), col.t()))
    _, _, wd, _ = reference(x.detach(), a.detach(), gamma.detach(), row.expand(T, d), col.t())
    tol = tolerance(d, wd, col, gamma.detach())
    assert bool(((wide.grad[:, 3:3 + d].double() - wd).abs() <= tol).all()) and bool((wide.grad[:, :3] == 0).all())
    assert bool(((turned.grad.t().double() - wd).abs() <= tol).all())


def test_gradients_add_up_over_microbatches():
    """Two backward passes into the same leaves: each leaf has the sum of its own."""
    x, a, gamma = leaves((5, 64), (5, 64), (64,))
    each = []
    for k in (1.0, 2.0):
        y, b, g = (t.detach().clone().requires_grad_() for t in (x, a, gamma))
        for leaf in ((x, a, gamma), (y, b, g)):
            h, n = pipeline.add_norm(*leaf)
            (k * (h * h).sum() + n.sum()).backward()
        each.append((y.grad, b.grad, g.grad))
    for t, first, second in zip((x, a, gamma), *each):
        assert torch.equal(t.grad, first + second)


def test_rows_in_two_shapes():
    x, a, gamma = leaves((2, 3, 64), (6, 64), (64,))
    for which in (0, 1):
        for t in (x, a, gamma):
            t.grad = None
        out = pipeline.add_norm(x, a, gamma)
        assert out[0].shape == out[1].shape == x.shape
        (out[which] * out[which]).sum().backward()
        assert a.grad.shape == a.shape and torch.equal(x.grad.view(6, 64), a.grad)
        x.grad.zero_()
        assert bool((a.grad != 0).any())
