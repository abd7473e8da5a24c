"""Heads that are slices of padded rows, with a guard behind the workspace that the query asks for (tolerances: vocab_helpers)."""
import pytest
import torch

import vocab_helpers as vh
from test_embed_gpu import backward, check_backward, ids_of, rows
from test_vocab_loss_gpu import each, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,d,wpad", [(512, 200000, 1004, 4), (300, 150000, 1021, 3), (2, 131072, 2044, 4)])
def test_a_head_of_padded_rows(T, V, d, wpad):
    """Rows of no whole 16 bytes, whole 16 bytes apart: W is used as it lies (run() checks what lies behind the workspace)."""
    X, W, labels = vh.inputs(T, V, d, wpad=wpad)
    assert W.stride(0) % 8 == 0 and W.data_ptr() % 16 == 0 and d % 8
    want = vh.ce(X, W, labels)
    loss, lse, dX, dW = run(X, W, labels, each(T))
    want.check_fwd(loss, lse)
    want.check_bwd(each(T), dX, dW)
    dense = run(X, W.contiguous(), labels, each(T))
    want.check_fwd(*dense[:2])
    want.check_bwd(each(T), *dense[2:])


def test_an_embedding_of_more_tokens_times_words_than_a_loss_may_have():
    T, V, d = 1 << 22, 1 << 21, 8
    ids, dout = ids_of(T, V, "any"), rows(T, d, "bf16")
    check_backward(backward(ids, dout, 0.5, V), ids, dout, 0.5, V)
