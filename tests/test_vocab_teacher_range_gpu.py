"""Teachers' logits at the ends of their type, and temperatures far from one (tolerances: vocab_helpers)."""
import pytest
import torch

import vocab_helpers as vh
from test_vocab_loss_gpu import each, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [0.25, 0.7, 1.0, 3.0])
def test_the_types_lowest_and_highest_values(tau, dtype):
    T, V, d, K = 60, 300, 72, 6
    X, W, _ = vh.inputs(T, V, d, dtype, ignored=0.0)
    index, teacher = vh.entries(T, V, K, dtype, missing=0.0, empty=0.0)
    end = torch.finfo(teacher.dtype)
    teacher[:20] = end.min            # masked everywhere: alike
    teacher[20:40, ::2] = end.min     # masked in places
    teacher[40:50] = end.max
    teacher[50, :3], teacher[51, 1:] = end.max, end.min
    want = vh.distill(X, W, index, teacher, tau)
    assert bool(torch.isfinite(want.loss).all())
    loss, lse, dX, dW = run(X, W, index, each(T), teacher, tau)
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [0.01, 100.0, 1e4])
def test_temperatures_far_from_one(tau, dtype):
    T, V, d, K = 60, 300, 72, 6
    X, W, _ = vh.inputs(T, V, d, dtype, ignored=0.0)
    index, teacher = vh.entries(T, V, K, dtype, empty=0.1)
    want = vh.distill(X, W, index, teacher, tau)
    loss, lse, dX, dW = run(X, W, index, each(T), teacher, tau)
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)


def test_entries_without_weight():
    """-infinity: none; everywhere: no distribution, a loss of NaN for that token alone"""
    T, V, d, K = 60, 300, 72, 6
    X, W, _ = vh.inputs(T, V, d, ignored=0.0)
    index, teacher = vh.entries(T, V, K, missing=0.0, empty=0.0)
    teacher[:, 1::2] = -torch.inf
    teacher[7] = -torch.inf
    loss, lse, dX, _ = run(X, W, index, each(T), teacher, 0.7)
    nan = torch.isnan(loss)
    assert int(nan.sum()) == 1 and bool(nan[7]) and bool(torch.isfinite(lse).all())
    assert bool(torch.isnan(dX[7]).all()) and bool(torch.isfinite(dX[~nan]).all())
