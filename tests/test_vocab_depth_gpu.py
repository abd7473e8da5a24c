"""The losses over the vocabulary at widths and lengths where an error that grows with the number of additions shows (tolerances:
vocab_helpers, but for the errors of a logit, which are derived here)."""
import math

import pytest
import torch

import vocab_helpers as vh
from paper_2604_11947_gb300 import resbm
from test_vocab_loss_gpu import each, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [4, 40])
def test_certain_tokens_of_a_wide_model(T):
    """Positive terms, so that what the tensor cores cut off as they add has one sign; one word has all the probability, so that p - 1 is
    next to nothing and the gradients are the error of the logits alone. A logit of terms whose absolute sum is S, in pieces of 32 MMAs
    in the forward and 64 in the backward, each of which cuts off at most 2 * 2^-23 of the piece: (32 and 64) 2^-22 S in all,
    and u S for each piece that is added in fp32."""
    V, d = 64, 131072
    g = torch.Generator(device="cuda").manual_seed(1)
    X = (0.5 + torch.rand(T, d, generator=g, device="cuda")).bfloat16()
    W = torch.randn(V, d, generator=g, device="cuda") * (0.01 / d ** 0.5)
    W[0] = (0.5 + torch.rand(d, generator=g, device="cuda")) * (256 / d)
    W, labels = W.bfloat16(), torch.zeros(T, dtype=torch.int64, device="cuda")
    want = vh.ce(X, W, labels)
    S = want.X.abs() @ want.W.abs().t()
    lse_err = (32 * 2.0 ** -22 + (d / 512 + 1) * vh.U) * S.amax(dim=1)
    want.lse_err = lse_err + 2.0 ** -17 + 8 * vh.U * 2 * want.lse.abs()
    want.loss_err = 2 * want.lse_err + 2.0 ** -20 * want.lse.abs()
    want.dz_err = (64 * 2.0 ** -22 + (d / 1024 + 1) * vh.U) * S
    assert float(want.z.max()) > 250 and float(want.loss.max()) < 1e-30
    loss, lse, dX, dW = run(X, W, labels, each(T))
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)


def test_a_gradient_of_a_million_tokens():
    """Terms of one sign in dW, which the tensor cores' truncation makes smaller, in as many units as there are CTA pairs (so that
    none is split for their sake). A head of zeros: dz of every word but the label is 2^-32 exactly. 65536 products in an accumulator
    are 4096 MMAs that cut off at most 2 * 2^-23 of it each, 2^-10 in all, and the 16 accumulators are added in fp32. The rounding to bf16,
    2^-8 of a value, has no sign over columns of other sizes: the mean of its 4864 is under 2^-8 / 4864^0.5 * 4."""
    T, V, d = 1 << 20, 4096, 4864
    g = torch.Generator(device="cuda").manual_seed(1)
    X, total, size = torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda"), 1 << 16
    for t in range(0, T, size):
        X[t:t + size] = ((0.5 + torch.rand(size, d, generator=g, device="cuda")) * (1 + torch.arange(d, device="cuda") / d)).bfloat16()
        total += X[t:t + size].sum(dim=0, dtype=torch.float64)
    W, labels = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")
    lse, dW = torch.full((T,), math.log(V), device="cuda"), torch.empty_like(W)
    ws = resbm.vocab_workspace(resbm.RESBM_VOCAB_CE_BWD, T, V, d)
    resbm.resbm_linear_ce_bwd(X, W, labels, lse, torch.full((1,), 1.0 / T, device="cuda"), None, dW, ws)
    want = total / T / V
    off = (dW[1:].double() - want) / want
    bound = 2.0 ** -10 + 16 * vh.U
    assert float(off.mean().abs()) <= bound + 4 * 2.0 ** -8 / d ** 0.5, float(off.mean())
    assert float(off.abs().max()) <= (bound + 2.0 ** -8) * 1.01
