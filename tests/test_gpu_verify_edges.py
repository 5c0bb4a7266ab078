"""Verification of drafts: temperatures of greedy sequences, and how far a row's sum may be off."""
import math

import numpy as np
import pytest
import torch

from test_gpu_block import BF16, FP32, P
from test_gpu_verify import check, drafts, i32

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


def test_a_sum_of_equal_terms_is_held_in_64_bits():
    """A largest logit in every 256, over equal ones: its probability is 1 / (512 + 130560 e), e an fp32
    exponential, off by a unit in the last place (2^-23 of itself at most, as e is over 1/2) and by its
    argument's three roundings (2^-24 |log2 e| each, |log2 e| < 0.1).  In all less than 1.35e-7 of
    itself, so that random numbers 1.6e-7 away from it are told from it; terms that are added up in 32 bits,
    where every partial sum of equal ones is rounded, are off by up to 5e-7."""
    B, V = 64, 131072
    gap = np.linspace(0.05, 0.065, B).astype(np.float32)
    logits = torch.from_numpy(-gap).cuda()[:, None].expand(B, V).repeat_interleave(2, 0).contiguous()
    logits[::2, ::256] = 0.0
    p = 1 / (V / 256 + V / 256 * 255 * np.exp(-gap.astype(np.float64)))
    tokens, off = i32([0, 512] * B), i32(list(range(0, 2 * B + 1, 2)))
    for sign, count in ((-1, 2), (1, 1)):
        u = (p * (1 + sign * 1.6e-7)).astype(np.float32)
        near = np.nextafter(u, np.float32(sign), dtype=np.float32)      # rounded away from p
        u = np.where((u.astype(np.float64) - p) * sign < 1.6e-7 * p, near, u)
        rows = torch.zeros(2 * B, device="cuda")
        rows[1::2] = torch.from_numpy(u).cuda()
        _, n, _ = P().DraftVerifier()(logits, tokens, off, 2, u=rows, u_next=torch.zeros(B, device="cuda"))
        assert n.tolist() == [count] * B, sign
