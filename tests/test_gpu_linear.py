"""moe_quant_linear: single rows, and sums held to what independent roundings leave."""
import math

import pytest
import torch

from test_gpu_block import BF16, FP16, FP32, E32, P, gen, linear_bound, packed, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("words", [32, 35, 40])
def test_one_row_of_any_length(T, words):
    """A matrix of one row has no row stride that could be out of line."""
    K = 256
    codes, sz, w, mag = packed(1, K, 64, 3, pad=16)
    x = torch.randn(T, K, device="cuda", generator=gen(T)).to(BF16)
    y = torch.empty(T, 1, device="cuda")
    P().moe_quant_linear(x, codes[:, :words], sz, y)
    want = x.double() @ w.t()
    within(y, want, linear_bound(x, mag, K, FP32, want), "one row")
