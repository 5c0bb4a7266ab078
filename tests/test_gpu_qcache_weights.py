"""moe_qcache_attention where weights or scales are extreme: many weights far below the largest, how
much of each weight counts, and scales of zero, on every way that rows and keys are laid
over waves (rows per key head and head size choose it)."""
import math

import pytest
import torch

from test_gpu_block import BF16, E32, FP16, P, TINY, U, chain_sees, gen, within
from test_gpu_qcache import attention_want, fill, qbatch, qrows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,new,dt", [(64, 1, FP16), (64, 30, BF16), (64, 40, FP16), (64, 140, BF16), (128, 1, BF16), (128, 20, FP16),
                                      (128, 70, FP16), (128, 130, BF16), (256, 3, FP16), (256, 40, BF16), (256, 70, FP16)])
def test_many_small_weights_count(D, new, dt):
    """2^20 keys of 2^-26.5 of the largest weight each, beside 8 of the largest (one in each of the first
    tiles, so that every wave has seen it).  A weight below fp16's normal range is off by up to 2^-25
    where the largest is stored as 2^7, so the values' sum by up to N 2^-32 of the largest, and by
    its own additions: 2^15 products one after the other into a sum that grows evenly, each rounded twice, by 2^-23 of the sum
    so far at most.  In the sum of weights all small ones of a lane that holds a largest may be lost, those of
    a quarter of the slots."""
    N, page, tops = 1 << 20, 1024, 8
    k = torch.zeros(N // page + 1, 1, page, D, dtype=torch.int8, device="cuda")
    v = torch.ones(N // page + 1, 1, D, page, dtype=torch.int8, device="cuda")
    scales = [torch.ones(N // page + 1, 1, page, device="cuda") for _ in "kv"]
    at = 64 * torch.arange(tops, device="cuda")
    k[0, 0, at, 0] = 16
    v[0, 0, :, at] = 0
    k[N // page, 0, :new, 0] = -127       # the new tokens' own keys weigh nothing
    scales[0][N // page] = 8
    table = torch.arange(N // page + 1, dtype=torch.int32, device="cuda")[None]
    cache = P().QuantPagedCache(k, v, *scales, table, torch.tensor([N], dtype=torch.int32, device="cuda"), dtype=dt)
    q = torch.zeros(new, 1, D, dtype=dt, device="cuda")
    q[:, 0, 0] = 1.0
    off = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    small = (N - tops) * 2.0 ** -26.5
    want = torch.full((new, 1, D), small / (tops + small), dtype=torch.float64, device="cuda")
    bound = N * 2.0 ** -32 / tops + (2.0 ** -8 + small / 4 / tops + 1.01 * U[dt]) * want + TINY[dt]
    assert bound.max() < 0.05 * want.max()
    for guess in (0, N + new):             # the keys in one part, and in many
        out = cache.attend(q, off, new, guess, scale=26.5 * math.log(2) / 16)
        assert cache.status_value() == 0
        within(out, want, bound, "small weights")


def tight(cache, lens, new, q, scale, dt, rel, parts=1):
    """A chain's attention in 64 bits, and a bound: a weight off by `rel` of itself, once in the values' sum and
    once in the weights', or, in the values' sum, by 2^-32 of the row's largest product of weight and value scale;
    scores as in attention_want; sums by (keys / 16 + 64) E32; the output's rounding."""
    outs, bounds, n0 = [], [], 0
    Hq, D = q.shape[1:]
    for b, (a, n) in enumerate(zip(lens, new)):
        kc, ks, vc, vs = (x.double() for x in qrows(cache, b, range(a + n)))
        for i in range(n):
            seen = a + i + 1
            k = (kc[:seen] * ks[:seen, :, None]).permute(1, 2, 0).contiguous()
            codes, s = vc[:seen].transpose(0, 1).contiguous(), vs[:seen].t().contiguous()
            qi = q[n0 + i].double().view(kc.shape[1], -1, D)
            w = torch.softmax(torch.matmul(qi, k) * scale, 2)
            e = (D + 8) * E32 * scale * torch.matmul(qi.abs(), k.abs()).amax(2, keepdim=True)
            ws = w * s[:, None]
            want, size = torch.matmul(ws, codes), torch.matmul(ws, codes.abs())
            bound = (4 * e + 2 * rel + (seen / 16 + 64) * E32) * size
            bound = bound + 2.0 ** -32 * ws.amax(2, keepdim=True) * codes.abs().sum(1, keepdim=True)
            outs.append(want.reshape(Hq, D))
            bounds.append((bound + U[dt] * 1.01 * (want.abs() + bound) + TINY[dt]).reshape(Hq, D))
        n0 += n
    return torch.stack(outs), torch.stack(bounds)


@pytest.mark.parametrize("lens,new,Hq,Hkv,D", [
    ([100], [1], 4, 2, 64), ([700, 33], [3, 1], 8, 2, 64), ([6], [16], 2, 1, 64), ([3, 9, 20], [1, 7, 16], 4, 2, 64),
    ([5], [1], 64, 2, 64), ([2500], [4], 16, 2, 128), ([0, 31], [8, 2], 4, 1, 128), ([9], [1], 16, 1, 128), ([2, 70], [32, 5], 2, 2, 128),
    ([3000, 5], [1, 1], 8, 2, 128), ([64], [1], 16, 1, 256), ([4], [8], 2, 1, 256), ([1200, 7], [4, 3], 4, 1, 256)])
def test_few_fp16_rows_keep_more_of_their_weights(lens, new, Hq, Hkv, D):
    """Up to 32 rows per key head (16 at head_dim 256) a weight of an fp16 row enters as its
    fp16 rounding and the rounded rest: off by 2^-22.  Its exponent, of scores below 2^4 and value scales between
    2^-8 and 1, is off by 2^-19 (the score's products with its scale and log2 s', their logarithm, the maximum
    taken off: 2^-21 to 2^-20 each, times ln 2), its power by 2^-23: 2^-17 covers them.  The output's
    rounding is the largest error then."""
    cache, off = qbatch(lens, new, 64, Hkv, D, FP16, 23, junk=True)
    tot, g = sum(lens) + sum(new), gen(25)
    v = torch.randn(tot, Hkv, D, device="cuda", generator=g)
    top = 2.0 ** -(8 * torch.rand(tot, Hkv, 1, device="cuda", generator=g))
    fill(cache, lens, new, torch.randn(tot, Hkv, D, device="cuda", generator=g), v / v.abs().amax(-1, keepdim=True) * 127 * top)
    q = 0.7 * torch.randn(sum(new), Hq, D, device="cuda", generator=g)
    q[:, ::2] *= 0.05     # scores that are hardly off themselves
    q = q.to(FP16)
    want, bound = tight(cache, lens, new, q, D ** -0.5, FP16, 2.0 ** -17)
    for guess in (0, max(a + n for a, n in zip(lens, new)), 30000):
        within(cache.attend(q, off, max(new), guess), want, bound, "split for %d" % guess)


@pytest.mark.parametrize("D,new,Hq,dt", [(64, 2, 3, BF16), (64, 20, 2, FP16), (64, 12, 4, BF16), (64, 70, 4, FP16), (128, 3, 4, FP16), (128, 40, 4, BF16),
                                         (128, 70, 4, FP16), (256, 3, 4, BF16), (256, 30, 2, FP16), (256, 70, 2, BF16)])
def test_weights_count_down_to_2_32_of_the_largest(D, new, Hq, dt):
    """Values of scales from 2^-24 to 1, where the large ones' weights are small: a weight times its
    value's scale counts to half a unit of fp16 or 2^-32 of the row's largest (exponents of up to 2^6 are
    off by 2^-16 in all)."""
    ctx = 230
    cache, off = qbatch([ctx], [new], 64, 1, D, dt, 43, junk=True)
    tot, g = ctx + new, gen(5)
    level = torch.rand(tot, 1, 1, device="cuda", generator=g)
    v = torch.randn(tot, 1, D, device="cuda", generator=g) * 2.0 ** (-24 * (1 - level))
    k = torch.randn(tot, 1, D, device="cuda", generator=g)
    k[..., 0] = 4 - 34 * level[..., 0]
    fill(cache, [ctx], [new], k, v)
    q = torch.randn(new, Hq, D, device="cuda", generator=g).to(dt)
    q[..., 0] = 1 + torch.rand(new, Hq, device="cuda", generator=g).to(dt)
    want, bound = tight(cache, [ctx], [new], q, 0.6, dt, 1.01 * U[FP16] + 2.0 ** -15)
    for guess in (0, tot):
        within(cache.attend(q, off, new, guess, scale=0.6), want, bound, "split for %d" % guess)


@pytest.mark.parametrize("D,new,Hq", [(64, 1, 2), (64, 20, 2), (64, 50, 2), (64, 130, 2), (128, 2, 4), (128, 40, 4), (128, 70, 4), (256, 3, 4), (256, 70, 4)])
@pytest.mark.parametrize("dt", [BF16, FP16])
def test_value_scales_of_zero(D, new, Hq, dt):
    """A caller's own rows of zeros may have a scale of zero: they take their share of the softmax.  Codes
    of such a row may count as if it were 2^-64: by 9 x 2^-64 at most with the codes here, which the
    weight's rounding (2^-11, its exponent 2^-15) and then the output's (2^-8) may raise by less than
    2^-7 of itself."""
    ctx = 300
    cache, off = qbatch([ctx], [new], 64, 2, D, dt, 44)
    q = torch.randn(new, Hq, D, device="cuda", generator=gen(1)).to(dt)
    for slot in list(range(0, ctx, 3)) + list(range(ctx, ctx + new, 2)):      # cached ones and drafts
        pg, o = int(cache.table[0, slot // 64]), slot % 64
        cache.v[pg, :, :, o] = 0 if slot % 2 else 9
        cache.v_scale[pg, :, o] = 0
        cache.k_scale[pg, :, o] *= slot % 7 != 0
    want, bound = attention_want(cache, [ctx], [new], q, chain_sees([new]), 0.3, dt)
    for guess in (0, ctx + new):
        within(cache.attend(q, off, new, guess, scale=0.3), want, bound + 9 * 2.0 ** -64 * (1 + 2.0 ** -7))
    cache.v_scale.zero_()
    out = cache.attend(q, off, new, ctx + new, scale=0.3)
    assert out.abs().max().item() <= 127 * 2.0 ** -64 * 1.01
    cache.v.zero_()
    assert (cache.attend(q, off, new, ctx + new, scale=0.3) == 0).all()
    cache.v_scale[int(cache.table[0, 0]), :, 0] = math.nan      # none is a number still
    assert cache.attend(q, off, new, ctx + new, scale=0.3).isnan().all()
