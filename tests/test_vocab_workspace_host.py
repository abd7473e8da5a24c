"""Workspace sizes of include/resbm_vocab.h, without a GPU."""
import pytest

from paper_2604_11947_gb300 import build, resbm


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


SHAPES = [(4096, 32000, 2052), (1024, 131072, 4100), (512, 250002, 2044), (1, 131072, 2044), (512, 200000, 1004), (300, 150000, 2043), (9, 113457, 6916)]


@pytest.mark.parametrize("T,V,d", SHAPES)
def test_a_head_of_padded_rows_has_room(T, V, d):
    """A head of d columns (no whole 16 bytes) whose rows lie whole 16 bytes apart is used as it lies, in the pieces, slots and
    packed rows of X that d rounded up to eight columns has. That width's size covers this form, so this width's has to be no smaller."""
    wide = -(-d // 8) * 8
    assert wide > d and (wide - 1) // 64 == (d - 1) // 64
    for op in (resbm.RESBM_VOCAB_CE_FWD, resbm.RESBM_VOCAB_CE_BWD, resbm.RESBM_VOCAB_DISTILL_FWD, resbm.RESBM_VOCAB_DISTILL_BWD):
        size = lambda n: resbm.resbm_vocab_workspace_bytes(op, T, V, n, "bf16", 5)
        assert size(d) >= size(wide)


@pytest.mark.parametrize("T,V,d", [(1 << 22, 1 << 21, 8), ((1 << 29) - 1, (1 << 29) - 1, 64), (1 << 20, 1000, 1 << 20), (1, 1, 1), (0, 1, 1 << 20)])
def test_the_embedding_has_limits_of_its_own(T, V, d):
    """Every size that resbm_embed_bwd takes has a workspace size: 4 numbers a token and 2 rows of fp32 a block of 32 tokens."""
    size = resbm.resbm_vocab_workspace_bytes(resbm.RESBM_VOCAB_EMBED_BWD, T, V, d)
    blocks = (T + 31) // 32
    assert 16 * T + 8 * blocks * d <= size <= 16 * T + 8 * blocks * d + 3 * 256


@pytest.mark.parametrize("T,V,d,status", [(1 << 29, 1, 1, resbm.RESBM_ERR_UNSUPPORTED), (1, 1 << 29, 1, resbm.RESBM_ERR_UNSUPPORTED), (1, 1, (1 << 20) + 1, resbm.RESBM_ERR_UNSUPPORTED),
                                          (-1, 1, 1, resbm.RESBM_ERR_INVALID_ARG), (1, 0, 1, resbm.RESBM_ERR_INVALID_ARG), (1, 1, 0, resbm.RESBM_ERR_INVALID_ARG)])
def test_sizes_that_the_embedding_refuses(T, V, d, status):
    with pytest.raises(resbm.ResbmError) as e:
        resbm.resbm_vocab_workspace_bytes(resbm.RESBM_VOCAB_EMBED_BWD, T, V, d)
    assert e.value.status == status
