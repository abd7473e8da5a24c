"""resbm_add_rmsnorm_fwd in rows of eight vectors a thread (2049 to 4096 vectors: bf16 d = 16385 to 32768, fp32 8193 to 16384) off
the vectors' alignment, by width, by address and by stride. The checks and their tolerances are test_add_norm_gpu's: a thread adds
4 pairs a vector and then 8 vectors, 13 sums one after the other, within its 32."""
import pytest
import torch

import test_add_norm_gpu as base
from paper_2604_11947_gb300 import resbm

pytestmark = pytest.mark.gpu
WIDTHS = [("bf16", 16385), ("bf16", 20001), ("bf16", 24583), ("bf16", 32767), ("f32", 8193), ("f32", 12001), ("f32", 16383)]


@pytest.mark.parametrize("dtype,d", WIDTHS)
@pytest.mark.parametrize("group", [0, 32, 128, 1024, 8192])
def test_widths(dtype, d, group):
    for T in (1, 5, 400):      # (more rows than CTAs run at once)
        X, A, gamma = base.rows(T, d, dtype, 1), base.rows(T, d, dtype, 2, scale=0.5), base.gamma_of(d, dtype)
        o = base.outputs(T, d, dtype, "hnq", group)
        base.run(X, A, gamma, o, T, d, group)
        base.check(X, A, gamma, base.EPS, o, T, d, group)
    assert resbm.resbm_device_error() == 0


@pytest.mark.parametrize("dtype,d", [("bf16", 16385), ("bf16", 20001), ("bf16", 32768), ("f32", 8193), ("f32", 12001), ("f32", 16384)])
def test_every_alignment_in_place_and_around(dtype, d):
    base.test_every_alignment(dtype, d)


@pytest.mark.parametrize("dtype,d,pad", [("bf16", 20000, 5), ("bf16", 32767, 1), ("f32", 12000, 3), ("f32", 16383, 1)])
def test_strides(dtype, d, pad):
    base.test_strides(dtype, d, pad)


@pytest.mark.parametrize("dtype,d", [("bf16", 20001), ("f32", 12001)])
def test_in_place_and_broadcast(dtype, d):
    base.test_in_place_and_broadcast(dtype, d)
