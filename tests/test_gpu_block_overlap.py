"""The overlaps of inputs and outputs that the decoder block's entry points promise to take."""
import pytest
import torch

from test_gpu_block import BF16, P, batch, gen, norm_case

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


@pytest.mark.parametrize("ctx,new", [(0, 1), (90, 7), (4000, 40)])
def test_attention_between_rows(ctx, new):
    """Queries and outputs as parts of the same rows."""
    cache, off = batch([ctx], [new], 32, 2, 64, BF16, 5)
    q = torch.randn(new, 4, 64, device="cuda", generator=gen(6)).to(BF16)
    want = cache.attend(q, off, new, ctx + new)
    for q_at, o_at in ((0, 4), (4, 0), (5, 1)):
        rows = torch.full((new, 10, 64), 3.0, device="cuda").to(BF16)
        rows[:, q_at:q_at + 4] = q
        before = rows.clone()
        cache.attend(rows[:, q_at:q_at + 4], off, new, ctx + new, out=rows[:, o_at:o_at + 4])
        assert torch.equal(rows[:, o_at:o_at + 4], want)
        rows[:, o_at:o_at + 4] = before[:, o_at:o_at + 4]
        assert torch.equal(rows, before)
    rows = torch.zeros(2 * new + 2, 4, 64, device="cuda", dtype=BF16)   # one after the other in an allocation
    rows[new:2 * new] = q
    cache.attend(rows[new:2 * new], off, new, ctx + new, out=rows[:new])
    assert torch.equal(rows[:new], want)


@pytest.mark.parametrize("q_out", ["in place", "beside"])
def test_append_between_rows(q_out):
    """Queries, keys, values and rotated queries as parts of the same rows."""
    new, Hq, Hkv, D = [5, 70], 4, 2, 64
    cache, off = batch([33, 0], new, 32, Hkv, D, BF16, 7)
    rows = torch.randn(75, 2 * Hq + 2 * Hkv, D, device="cuda", generator=gen(8)).to(BF16)
    ang = torch.rand(200, D // 2, device="cuda", generator=gen(9)) * 6.28
    rot = dict(cos=ang.cos(), sin=ang.sin())
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:Hq + 2 * Hkv]
    want = cache.append(q, k, v, off, 70, **rot)
    kept = cache.k.clone(), cache.v.clone()
    cache.k.zero_(), cache.v.zero_()
    cache.append(q, k, v, off, 70, q_out=q if q_out == "in place" else rows[:, Hq + 2 * Hkv:], **rot)
    assert torch.equal(q if q_out == "in place" else rows[:, Hq + 2 * Hkv:], want)
    for b in range(2):
        for a, w in zip((cache.k, cache.v), kept):
            n = [33, 0][b]
            for slot in range(n, n + new[b]):
                pg, o = int(cache.table[b, slot // 32]), slot % 32
                at = (pg, slice(None), o) if a is cache.k else (pg, slice(None), slice(None), o)
                assert torch.equal(a[at], w[at])
