"""moe_tree_attention with values that are not finite among the cached tokens, on every way
that rows and keys are laid over waves (rows per key head and head size choose it)."""
import math

import pytest
import torch

from test_gpu_block import BF16, FP16, batch, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,new,Hq,dt", [
    (64, 4, 4, BF16), (64, 12, 2, FP16), (64, 16, 3, BF16), (64, 30, 4, FP16), (64, 64, 3, BF16),
    (128, 3, 2, FP16), (128, 12, 4, BF16), (128, 31, 4, FP16), (128, 50, 4, BF16),
    (256, 4, 4, BF16), (256, 9, 4, FP16), (256, 40, 4, BF16)])
def test_cached_values_that_are_not_finite_reach_every_row(D, new, Hq, dt):
    """Every token sees every cached slot, so an infinite or NaN value there leaves nothing
    finite in its channel, whichever tile of keys it is in, and changes no other channel."""
    ctx, page = 500, 32
    cache, off = batch([ctx], [new], page, 1, D, dt, 17)
    q = torch.randn(new, Hq, D, device="cuda", generator=gen(18)).to(dt)
    rest = [c for c in range(D) if c != 2]
    for guess in (ctx + new, 0):      # keys in parts, and in one
        clean = cache.attend(q, off, new, guess)
        assert torch.isfinite(clean).all()
        for tile in range(4, (ctx + page - 1) // page):
            slot, val = tile * 32 + 7, math.nan if tile % 2 else math.inf
            at = (int(cache.table[0, slot // page]), 0, 2, slot % page)
            was = cache.v[at].clone()
            cache.v[at] = val
            out = cache.attend(q, off, new, guess)
            cache.v[at] = was
            assert not torch.isfinite(out[:, :, 2]).any(), "value %s in tile %d was lost" % (val, tile)
            assert torch.equal(out[:, :, rest], clean[:, :, rest]), tile
