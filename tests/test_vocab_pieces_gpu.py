"""The losses over a vocabulary that goes in several pieces, whose ends lie inside a unit's columns: targets at, before and behind
every border (tolerances: vocab_helpers)."""
import pytest
import torch

import vocab_helpers as vh
from test_vocab_loss_gpu import each, run

pytestmark = pytest.mark.gpu


def every_word(T, V, K, seed=0):
    """K entries a token that name every word of the vocabulary at least once (T K >= V), in no order, none twice for a token"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    words = torch.cat([torch.randperm(V, generator=g, device="cuda") for _ in range(-(-T * K // V))])[:T * K]
    index = words.view(T, K)
    if K > 1:   # (a token whose entries lie over the end of a permutation may have a word twice: once is enough)
        index = index.sort(dim=1).values
        index[:, 1:][index[:, 1:] == index[:, :-1].clone()] = -1
    return index.contiguous(), 2 * torch.randn(T, K, generator=g, device="cuda")


# pieces of 2816 words and units of 96 columns; 4096 and 224; fp32 11008 and 160, 64256 and 224
@pytest.mark.parametrize("T,V,d,K,wpad,dtype", [(300, 8193, 64, 64, 3, "bf16"), (777, 8000, 512, 20, 1, "bf16"), (40, 33000, 4096, 1024, 0, "f32"),
                                                (126, 128256, 768, 1024, 0, "f32")])
def test_distillation_from_every_word(T, V, d, K, wpad, dtype):
    X, W, _ = vh.inputs(T, V, d, dtype, ignored=0.0, wpad=wpad)
    index, teacher = every_word(T, V, K)
    assert bool((torch.bincount(index[index >= 0], minlength=V) > 0).all())
    for logits in (teacher, torch.where(torch.arange(K, device="cuda") % 3 == 1, -torch.inf, teacher)):   # (entries of no weight, too)
        want = vh.distill(X, W, index, logits, 2.0)
        loss, lse, dX, dW = run(X, W, index, each(T), logits, 2.0)
        want.check_fwd(loss, lse)
        want.check_bwd(each(T), dX, dW)


@pytest.mark.parametrize("V,d,wpad,dtype", [(8193, 64, 3, "bf16"), (33000, 4096, 0, "f32")])
def test_labels_around_every_multiple_of_256(V, d, wpad, dtype):
    """Pieces are of whole 256 words."""
    labels = torch.stack([torch.arange(0, V, 256, device="cuda") + i for i in (-1, 0, 1, 31, 32)]).clamp(0, V - 1).view(-1)
    T = labels.numel()
    X, W, _ = vh.inputs(T, V, d, dtype, ignored=0.0, wpad=wpad)
    want = vh.ce(X, W, labels)
    loss, lse, dX, dW = run(X, W, labels, each(T))
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)
