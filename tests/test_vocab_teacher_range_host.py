"""Temperatures at both ends of their range, on the host."""
import pytest

from paper_2604_11947_gb300 import resbm
from test_vocab_host import lib, loss   # noqa: F401  (lib: its fixture)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("temperature", [1e-19, 1e-38, 1e-45, 1e19, 3e38])
def test_temperatures_whose_square_or_reciprocal_is_no_float(lib, temperature, bwd):   # noqa: F811
    assert loss(lib, True, bwd, temperature=temperature) == resbm.RESBM_ERR_INVALID_ARG
