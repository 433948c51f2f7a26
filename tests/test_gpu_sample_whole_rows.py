"""Sampling where one bin holds a whole row of the largest vocabulary, 2^20 entries: rows of one value, and
temperatures beside which all values are alike. Tokens and counts are the definition's (u W of equal weights
is exact), log probabilities within the bound of test_gpu_sample.py."""

import pytest
import torch

from test_gpu_sample import BF16, F32, check, logits, uniform

pytestmark = pytest.mark.gpu

VOCAB = 2 ** 20
U = [0.0, 0.25, 1 - 2.0 ** -21, 1.0]


@pytest.mark.parametrize("dtype,value", [(F32, 0.0), (F32, -1.5), (F32, 3e38), (BF16, -1.5), (BF16, 2048.0), (BF16, 2.0 ** -40)])
def test_a_row_of_one_value(dtype, value):
    """bf16 rows of 2048 and 2^-40 have no bins of their own values."""
    x = torch.full((4, len(U), VOCAB), value).to(dtype)
    check(x, torch.tensor([U] * 4), [(1.0, 0, 1.0, 0.0), (1.0, 1000, 1.0, 0.0), (0.5, 0, 0.5, 0.0), (2.0, 2 ** 19, 0.75, 1.0)])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_values_alike_beside_the_temperature(dtype):
    """All weights are 1 to the last bit: the k-th share of u is drawn in the values' order."""
    x = logits(40, 1, 3, VOCAB, dtype=dtype)
    if dtype == BF16:
        x[..., 5] = 1100.0                                  # the general way
    check(x, torch.tensor([[0.0, 0.3, 0.8]]), [(1e30, 0, 1.0, 0.0)])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_half_of_a_row_at_one_value(dtype):
    x = logits(41, 1, 2, VOCAB, dtype=dtype)
    x[..., ::2] = 16.0
    if dtype == BF16:
        x[..., 5] = -1100.0
    check(x, uniform(42, 1, 2), [(1.0, 0, 0.9, 0.0)])
