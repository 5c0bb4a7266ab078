"""moe_tree_attention where values or weights are extreme: values that are not finite among the
cached tokens, and weights that are far below the largest, on every way
that rows and keys are laid over waves (rows per key head and head size choose it)."""
import math

import pytest
import torch

from test_gpu_block import BF16, E32, FP16, P, TINY, U, batch, gen, rows_of, within

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


@pytest.mark.parametrize("D,new", [(64, 1), (64, 30), (64, 40), (128, 1), (128, 20), (128, 70), (256, 3), (256, 40)])
def test_many_small_weights_count(D, new):
    """2^20 fp16 keys of 2^-26.5 of the largest weight each, beside 8 of the largest (one in each
    of the first tiles, so that every wave has seen it).  A weight below fp16's normal range
    is off by up to 2^-25 where the largest is stored as 2^7, so the sum by up to N 2^-32 of the
    largest; the fp32 sum of weights by up to 2^-11 of itself (8192 steps of half a unit in the
    last place of 2^7)."""
    N, page, tops = 1 << 20, 1024, 8
    k = torch.zeros(N // page + 1, 1, page, D, dtype=FP16, device="cuda")
    v = torch.ones(N // page + 1, 1, D, page, dtype=FP16, device="cuda")
    at = 32 * torch.arange(tops, device="cuda")
    k[0, 0, at, 0] = 16
    v[0, 0, :, at] = 0
    k[N // page, 0, :new, 0] = -1000       # the new tokens' own keys weigh nothing
    table = torch.arange(N // page + 1, dtype=torch.int32, device="cuda")[None]
    cache = P().PagedCache(k, v, table, torch.tensor([N], dtype=torch.int32, device="cuda"))
    q = torch.zeros(new, 1, D, dtype=FP16, device="cuda")
    q[:, 0, 0] = 1.0
    off = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    small = (N - tops) * 2.0 ** -26.5
    want = torch.full((new, 1, D), small / (tops + small), dtype=torch.float64, device="cuda")
    bound = N * 2.0 ** -32 / tops + (2 * 2.0 ** -11 + 2.0 ** -14) * want
    for guess in (0, N + new):             # the keys in one part, and in many
        out = cache.attend(q, off, new, guess, scale=26.5 * math.log(2) / 16)
        within(out, want, bound, "small weights")


@pytest.mark.parametrize("lens,new,Hq,Hkv,D,dt", [
    ([100], [1], 4, 2, 64, BF16), ([700, 33], [3, 1], 8, 2, 64, FP16), ([2500], [4], 16, 2, 64, BF16),
    ([0, 31], [8, 2], 4, 1, 128, BF16), ([3000, 5], [1, 1], 8, 2, 128, BF16), ([900], [32], 2, 2, 128, FP16),
    ([64], [1], 16, 1, 256, BF16), ([1200, 7], [4, 3], 4, 1, 256, FP16)])
def test_few_rows_keep_more_of_their_weights(lens, new, Hq, Hkv, D, dt):
    """Up to 32 rows per key head (16 at head_dim 256) a weight, and so their sum, is off by 2^-15
    of itself, its exponential's error included, or by 2^-32 of the largest where fp16 cannot
    hold its rest; scores as in attention_want.  The output's rounding is the largest error then."""
    cache, off = batch(lens, new, 32, Hkv, D, dt, 23)
    q = torch.randn(sum(new), Hq, D, device="cuda", generator=gen(24)).to(dt)
    out = cache.attend(q, off, max(new), max(a + n for a, n in zip(lens, new)))
    scale, n0 = D ** -0.5, 0
    for b, (a, n) in enumerate(zip(lens, new)):
        for i in range(n):
            seen = a + i + 1
            k, v = (x.double() for x in rows_of(cache, b, range(seen)))
            qi = q[n0 + i].double().view(Hkv, -1, D)
            k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
            w = torch.softmax(torch.matmul(qi, k) * scale, 2)
            e = (D + 8) * E32 * scale * torch.matmul(qi.abs(), k.abs()).amax(2, keepdim=True)
            want, size = torch.matmul(w, v), torch.matmul(w, v.abs())
            rel = 4 * e + 2 * 2.0 ** -15 + (seen / 16 + 64) * E32
            bound = rel * size + (2 * 2.0 ** -32 * v.abs().sum(1, keepdim=True) if dt == FP16 else 0)
            bound = bound + U[dt] * 1.01 * want.abs() + TINY[dt]
            within(out[n0 + i].view(Hkv, -1, D), want, bound, "sequence %d, token %d" % (b, i))
        n0 += n


@pytest.mark.parametrize("D,new,Hq,dt", [
    (64, 1, 4, BF16), (64, 7, 4, FP16), (64, 40, 4, BF16), (128, 3, 4, FP16), (128, 8, 4, BF16), (128, 60, 4, FP16),
    (256, 2, 4, BF16), (256, 3, 5, FP16), (256, 40, 4, BF16)])
@pytest.mark.parametrize("val", [math.inf, -math.inf])
def test_infinite_cached_values_keep_their_sign(D, new, Hq, dt, val):
    """Weights are positive (scores here are a few units apart), so one infinite value makes
    its channel infinite for everybody, and two of opposite sign make it NaN."""
    ctx, page = 500, 32
    cache, off = batch([ctx], [new], page, 1, D, dt, 27)
    q = torch.randn(new, Hq, D, device="cuda", generator=gen(28)).to(dt)
    clean = cache.attend(q, off, new, ctx + new)
    rest = [c for c in range(D) if c not in (3, 5)]
    for tile in range(0, (ctx + page - 1) // page):
        saved = cache.v.clone()
        slot = tile * 32 + tile % 20
        pg, o = int(cache.table[0, slot // page]), slot % page
        cache.v[pg, 0, 3, o] = val
        cache.v[pg, 0, 5, o] = val
        far = (slot + 200) % ctx
        cache.v[int(cache.table[0, far // page]), 0, 5, far % page] = -val
        out = cache.attend(q, off, new, ctx + new)
        cache.v.copy_(saved)
        assert (out[:, :, 3] == val).all(), tile
        assert torch.isnan(out[:, :, 5]).all(), tile
        assert torch.equal(out[:, :, rest], clean[:, :, rest]), tile
