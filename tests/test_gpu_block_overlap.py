"""The overlaps of inputs and outputs that the decoder block's entry points promise to take."""
import pytest
import torch

from test_gpu_block import BF16, P, norm_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 6])
@pytest.mark.parametrize("d", [64, 1000, 2048, 20000])
def test_norm_in_place_of_any_input(T, d):
    """r_out and h over r, y and a gate per element, in every order, give the same bits."""
    s = norm_case(T, d, BF16, BF16, BF16, True, "element", d)
    w = dict(w_post=s["w_post"], w_pre=s["w_pre"])
    P().moe_block_norm(s["r"], s["h"], y=s["y"], gate=s["gate"], r_out=s["r_out"], **w)
    names = ("r", "y", "gate")
    for over_r in names + (None,):
        for over_h in names + (None,):
            if over_r == over_h and over_r is not None:
                continue
            t = {n: s[n].clone() for n in names}
            r_out = t[over_r] if over_r else torch.empty_like(t["r"])
            h = t[over_h] if over_h else torch.empty_like(t["r"])
            P().moe_block_norm(t["r"], h, y=t["y"], gate=t["gate"], r_out=r_out, **w)
            assert torch.equal(r_out, s["r_out"]) and torch.equal(h, s["h"]), (over_r, over_h)
