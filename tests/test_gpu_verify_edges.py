"""Verification of drafts: temperatures of greedy sequences."""
import math

import pytest
import torch

from test_gpu_block import BF16, FP32
from test_gpu_verify import check, drafts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,V,dt", [("chain", 300, FP32), ("wide", 5000, BF16), ("tree", 70000, FP32)])
def test_greedy_sequences_whose_temperature_is_none(kind, V, dt):
    """A negative or not finite temperature is no temperature, with random numbers or without."""
    heat = torch.tensor([1.0, -1.0, math.nan, 0.0, math.inf, -math.inf, 0.5, -1e-30], device="cuda")
    s = drafts([5] * 8, V, kind, 3, dt, noise=0.2)
    v, (_, n, nxt) = check(s, 5, heat=heat, greedy=True)
    assert v.status_value() == -6      # MOE_ERR_RANGE
    for b in range(8):
        assert (nxt[b] == -1 and n[b] == 1) if b in (1, 2, 4, 5, 7) else nxt[b] >= 0
    fine = torch.tensor([1.0, 0.0, 1e-30, 0.5, 3e38, 2.0, 0.0, 1.0], device="cuda")
    v, got = check(s, 5, heat=fine, greedy=True)
    assert v.status_value() == 0 and got == check(s, 5, greedy=True)[1]      # they change nothing
