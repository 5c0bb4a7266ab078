"""Normed heads and the paged cache in 8 bits against their definitions in 64 bits.

Bounds are worked out before any run from the arithmetic the header promises: U is a type's
unit roundoff, a chain of n fp32 operations on terms whose absolute values add up to A is off
by at most about n 2^-24 A, and a code stands for its value to half a step.
"""
import math

import pytest
import torch

from test_gpu_block import (BF16, E32, FP16, TINY, U, P, batch, chain_sees, gen, rows_of, tree, tree_sees,
                            within)

pytestmark = pytest.mark.gpu
HALF = 0.5 + 2.0 ** -16     # of a step: what a code may be off by


def qbatch(lens, new, page, Hkv, D, dt, seed, spare=3, junk=False):
    """A cache in 8 bits with pages in random order.  junk: slots that no token was written to hold
    NaN scales; else random rows everywhere."""
    plain, off = batch(lens, new, page, Hkv, D, dt, seed, spare)
    g, shape = gen(seed + 2), plain.k.shape
    k = torch.randint(-128, 128, shape, device="cuda", generator=g).to(torch.int8)
    v = torch.randint(-128, 128, plain.v.shape, device="cuda", generator=g).to(torch.int8)
    ks, vs = (torch.full(shape[:3], math.nan, device="cuda") for _ in "kv")
    if not junk:
        k, v = k.clamp(min=-127), v.clamp(min=-127)
        ks, vs = (0.02 * torch.randn(shape[:3], device="cuda", generator=g).exp() for _ in "kv")
    return P().QuantPagedCache(k, v, ks, vs, plain.table, plain.lens, dtype=dt), off


def qrows(cache, b, slots):
    """Codes [slots][Hkv][D] and scales [slots][Hkv] of keys and values."""
    page = cache.k.shape[2]
    slots = torch.as_tensor(slots, device="cuda")
    pg, o = cache.table[b].long()[slots // page], slots % page
    return cache.k[pg, :, o], cache.k_scale[pg, :, o], cache.v[pg, :, :, o], cache.v_scale[pg, :, o]


def fill(cache, lens, new, k, v):
    """Write rows' values, quantised here, into the cache: k, v [tokens of all sequences][Hkv][D]."""
    page, n = cache.k.shape[2], 0
    for b, (a, m) in enumerate(zip(lens, new)):
        sl = torch.arange(a + m, device="cuda")
        pg, o = cache.table[b].long()[sl // page], sl % page
        for x, codes, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
            x = x[n:n + a + m].float()
            s = (x.abs().amax(-1) / 127).clamp(2.0 ** -64, 2.0 ** 64)
            q = (x / s[..., None]).round().clamp(-127, 127).to(torch.int8)
            scale[pg, :, o] = s
            if codes is cache.k:
                codes[pg, :, o] = q
            else:
                codes[pg, :, :, o] = q
        n += a + m


def heads_want(x, w, eps, cos, sin, pos, rot, inter):
    """Normed and rotated heads in 64 bits, and how far fp32 may be off before the last rounding:
    a sum of D squares over lanes ((D / 16 + 24) roundings and a root of half of that, a quotient,
    two products), two products and a sum of the rotation."""
    x = x.double()
    D = x.shape[-1]
    e = x.abs() * 0
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
        e = (D / 16 + 32) * E32 * x.abs()
    if not rot:
        return x, e
    c, s = cos[pos].double()[:, None], sin[pos].double()[:, None]
    at = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b, y, f = x[..., at[0]], x[..., at[1]], x.clone(), e.clone()
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    ea, eb = e[..., at[0]], e[..., at[1]]
    f[..., at[0]] = ea * c.abs() + eb * s.abs() + 4 * E32 * ((a * c).abs() + (b * s).abs())
    f[..., at[1]] = ea * s.abs() + eb * c.abs() + 4 * E32 * ((a * s).abs() + (b * c).abs())
    return y, f


APPEND = [
    # lens, new, page, Hq, Hkv, D, type, rot, interleaved, norm
    ([0], [1], 64, 4, 2, 64, BF16, 64, False, "qk"), ([31, 0, 100], [3, 0, 70], 64, 6, 2, 128, FP16, 128, False, "qk"),
    ([5, 64, 63, 1], [1, 64, 2, 33], 64, 8, 8, 128, BF16, 64, True, "k"), ([1000], [129], 128, 3, 1, 256, FP16, 256, True, "q"),
    ([7, 9], [40, 1], 1024, 2, 1, 64, BF16, 0, False, "qk"), ([33], [700], 64, 4, 4, 64, BF16, 32, False, ""),
    ([50, 127], [16, 17], 128, 10, 2, 256, BF16, 256, False, "qk"), ([60], [20], 64, 1, 1, 128, FP16, 16, True, "qk")]


@pytest.mark.parametrize("lens,new,page,Hq,Hkv,D,dt,rot,inter,norm", APPEND)
@pytest.mark.parametrize("bits", [16, 8])
def test_append(bits, lens, new, page, Hq, Hkv, D, dt, rot, inter, norm):
    cache, off = (batch if bits == 16 else qbatch)(lens, new, page, Hkv, D, dt, 21)
    N, g = sum(new), gen(2)
    qkv = torch.randn(N, Hq + 2 * Hkv, D, device="cuda", generator=g).to(dt)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    pos = torch.randint(0, 500, (N,), device="cuda", generator=g).int() if rot != 32 else None
    ang = torch.rand(max(500, max(a + n for a, n in zip(lens, new))), max(rot // 2, 1), device="cuda", generator=g) * 6.28
    cos, sin = (ang.cos(), ang.sin()) if rot else (None, None)
    w_q, w_k = (1 + 0.2 * torch.randn(D, device="cuda", generator=g) if x in norm else None for x in "qk")
    kw = dict(positions=pos, cos=cos, sin=sin, interleaved=inter, w_q=w_q, w_k=w_k, eps=1e-5)
    names = ("k", "v") if bits == 16 else ("k", "v", "k_scale", "v_scale")
    was, before = [getattr(cache, x).clone() for x in names], qkv.clone()
    out = cache.append(q, k, v, off, max(new), **kw)
    assert cache.status_value() == 0 and torch.equal(qkv, before)
    n = 0
    for b in range(len(lens)):
        if new[b] == 0:
            continue
        p = pos[n:n + new[b]].long() if pos is not None else torch.arange(lens[b], lens[b] + new[b], device="cuda")
        sl, slots = slice(n, n + new[b]), torch.arange(lens[b], lens[b] + new[b], device="cuda")
        want, e = heads_want(q[sl], w_q, 1e-5, cos, sin, p, rot, inter)
        within(out[sl], want, e + (U[dt] * 1.001 * want.abs() + TINY[dt]) * ((e > 0) | (want != q[sl].double())), "queries")
        want, e = heads_want(k[sl], w_k, 1e-5, cos, sin, p, rot, inter)
        pg, o = cache.table[b].long()[slots // page], slots % page
        if bits == 16:
            ks, vs = rows_of(cache, b, slots)
            within(ks, want, e + (U[dt] * 1.001 * want.abs() + TINY[dt]) * ((e > 0) | (want != k[sl].double())), "keys")
            assert torch.equal(vs, v[sl])
        else:
            kc, ks, vc, vs = qrows(cache, b, slots)
            for codes, s, x, ex in ((kc, ks, want, e), (vc, vs, v[sl].double(), 0 * e)):
                step, top = s.double()[..., None], x.abs().amax(-1, keepdim=True)
                within(step, top / 127, ex.amax(-1, keepdim=True) / 127 + 2 * E32 * top / 127, "scale")
                within(codes.double() * step, x, HALF * step + ex + 130 * E32 * top, "codes")
                assert codes.abs().max() == 127 and (codes.abs().amax(-1) >= 126).all()
            was[2][pg, :, o], was[3][pg, :, o] = ks, vs
            ks, vs = kc, vc
        was[0][pg, :, o], was[1][pg, :, :, o] = ks, vs
        n += new[b]
    for x, y in zip(names, was):       # everything else in the cache is untouched
        assert torch.equal(getattr(cache, x).view(torch.int8), y.view(torch.int8)), x
    # in place, and keys alone
    q2 = q.contiguous()
    cache.append(q2, k, v, off, max(new), q_out=q2, **kw)
    assert torch.equal(q2, out)
    cache.append(None, k, v, off, max(new) + 5, **kw)
    for x, y in zip(names, was):
        assert torch.equal(getattr(cache, x).view(torch.int8), y.view(torch.int8)), x


@pytest.mark.parametrize("D,rot,inter", [(64, 64, False), (128, 64, True), (256, 0, False)])
def test_append_norm_without_weights_is_the_plain_append(D, rot, inter):
    lens, new = [3, 70], [5, 90]
    a, off = batch(lens, new, 32, 2, D, BF16, 5)
    b, _ = batch(lens, new, 32, 2, D, BF16, 5)
    qkv = torch.randn(95, 8, D, device="cuda", generator=gen(1)).to(BF16)
    ang = torch.rand(200, max(rot // 2, 1), device="cuda", generator=gen(2))
    cos, sin = (ang.cos(), ang.sin()) if rot else (None, None)
    out = a.append(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], off, 90, cos=cos, sin=sin, interleaved=inter)
    other = torch.empty_like(out)
    P().moe_cache_append_norm(b.desc, b.table, b.lens, off, 90, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], other, None, None,
                              cos=cos, sin=sin, interleaved=inter)
    assert torch.equal(out, other) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_skips_what_is_out_of_range(bits):
    cache, off = (batch if bits == 16 else qbatch)([10, 20], [2, 3], 64, 2, 64, BF16, 4)
    names = ("k", "v") if bits == 16 else ("k", "v", "k_scale", "v_scale")
    was = {x: getattr(cache, x).clone() for x in names}
    kv = torch.randn(5, 2, 64, device="cuda").to(BF16)
    cos, w = torch.ones(50, 32, device="cuda"), torch.ones(64, device="cuda")
    q_out = torch.full((5, 2, 64), 9.0, device="cuda").to(BF16)
    pos = torch.tensor([-1, 0, 50, 1, 2], dtype=torch.int32, device="cuda")
    cache.append(kv, kv, kv, off, 3, positions=pos, cos=cos, sin=0 * cos, q_out=q_out, w_q=w, w_k=w)
    assert cache.status_value() == -5
    assert (q_out[[0, 2]] == 9).all() and (q_out[[1, 3, 4]] != 9).any(2).all()
    for b, slots in ((0, [10]), (1, [20])):    # the tokens whose position is out of range
        page = cache.k.shape[2]
        pg, o = int(cache.table[b, slots[0] // page]), slots[0] % page
        assert torch.equal(cache.k[pg, :, o], was["k"][pg, :, o]) and torch.equal(cache.v[pg, :, :, o], was["v"][pg, :, :, o])
        if bits == 8:
            assert torch.equal(cache.k_scale[pg, :, o], was["k_scale"][pg, :, o])
            assert torch.equal(cache.v_scale[pg, :, o], was["v_scale"][pg, :, o])
    for x in names:
        getattr(cache, x).copy_(was[x])
    for bad in (cache.k.shape[0], -1):   # a page that does not exist, then a length that cannot be
        cache.status.zero_()
        cache.table[1, 0] = bad
        cache.lens[0] = -5
        cache.append(None, kv, kv, off, 3, w_k=w)
        assert cache.status_value() == -5
        assert all(torch.equal(getattr(cache, x), was[x]) for x in names)


def test_rows_that_scales_cannot_follow():
    """Zeros, values below the least scale, beyond the largest, and rows that are not finite."""
    D = 64
    cache, off = qbatch([0], [6], 64, 1, D, BF16, 7)
    x = torch.randn(6, 1, D, device="cuda", generator=gen(3))
    x[0] = 0
    x[1] *= 1e-21
    x[2, 0, 5], x[2, 0, 9] = 1e30, -2e28
    x[3, 0, 1] = math.inf
    x[4, 0, 2] = math.nan
    x = x.to(BF16)
    cache.append(None, x, x, off, 6)
    assert cache.status_value() == 0
    k, v = cache.read(cache.lens, off, 6, rows=6)
    assert torch.equal(k.isnan(), v.isnan()) and torch.equal(k[[0, 1, 2, 5]], v[[0, 1, 2, 5]])
    assert (k[:2] == 0).all()
    assert k[2, 0, 5].item() == float(torch.tensor(127 * 2.0 ** 64).to(BF16)) and k[2, 0, 9].item() == -k[2, 0, 5].item()
    assert (k[2, 0, [i for i in range(D) if i not in (5, 9)]] == 0).all()
    assert k[3:5].isnan().all()
    within(k[5], x[5].double(), (HALF / 127 + 2 * U[BF16]) * x[5].double().abs().amax())


@pytest.mark.parametrize("lens,new,page,Hkv,D,dt", [
    ([0], [1], 64, 2, 64, BF16), ([31, 0, 100], [3, 0, 170], 64, 3, 128, FP16), ([5, 64, 63], [1, 64, 2], 128, 1, 256, BF16),
    ([1000], [700], 1024, 2, 128, BF16)])
def test_read(lens, new, page, Hkv, D, dt):
    cache, off = qbatch(lens, new, page, Hkv, D, dt, 9)
    N = sum(new)
    room = torch.full((2, N + 2, Hkv + 1, D), 5.0, device="cuda").to(dt)
    k, v = cache.read(cache.lens, off, max(new), k_out=room[0, :N, :Hkv], v_out=room[1, :N, 1:])
    assert cache.status_value() == 0
    n = 0
    for b in range(len(lens)):
        if new[b]:
            kc, ks, vc, vs = qrows(cache, b, range(lens[b], lens[b] + new[b]))
            assert torch.equal(k[n:n + new[b]], (kc.float() * ks[..., None]).to(dt))
            assert torch.equal(v[n:n + new[b]], (vc.float() * vs[..., None]).to(dt))
        n += new[b]
    assert (room[:, N:] == 5).all() and (room[0, :N, Hkv] == 5).all() and (room[1, :N, 0] == 5).all()
    # one of the two alone, new tensors, and the whole text from its start
    k1, v1 = torch.empty_like(k.contiguous()), torch.empty_like(v.contiguous())
    assert cache.read(cache.lens, off, max(new), k_out=k1)[1] is None and torch.equal(k1, k)
    cache.read(cache.lens, off, max(new) + 100, v_out=v1)
    assert torch.equal(v1, v)
    total = [a + n for a, n in zip(lens, new)]
    ends = torch.tensor([sum(total[:b]) for b in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    k2, v2 = cache.read(0 * cache.lens, ends, max(total), rows=sum(total))
    n = 0
    for b in range(len(lens)):
        at = int(ends[b]) + lens[b]
        assert torch.equal(k2[at:at + new[b]], k[n:n + new[b]]) and torch.equal(v2[at:at + new[b]], v[n:n + new[b]])
        n += new[b]
    # a page out of range is not followed
    cache.table[0, 0] = cache.k.shape[0]
    k3 = torch.full_like(k2, 3.0)
    cache.read(0 * cache.lens, ends, max(total), k_out=k3)
    assert cache.status_value() == -5
    first = min(page, total[0])
    assert (k3[:first] == 3).all() and torch.equal(k3[total[0]:], k2[total[0]:])


# ------------------------------------------------------------------ attention
def attention_want(cache, lens, new, q, sees, scale, dt):
    """The definition in 64 bits over the values the rows stand for, and its bound.  Scores are off
    by (D + 8) E32 of their absolute sums (e, times scale), and by the rounding of an exponent
    of up to 2^8 (2^-16); a weight is rounded to fp16 in the values' sum (U[FP16]), or, where weight
    times value scale is 2^-12 of the row's largest or less, may be off by 2^-22 of that largest;
    sums by (keys / 16 + 64) E32."""
    outs, bounds, n0 = [], [], 0
    Hq, D = q.shape[1], q.shape[2]
    for b in range(len(lens)):
        n, tot = new[b], lens[b] + new[b]
        if n == 0:
            continue
        kc, ks, vc, vs = (x.double() for x in qrows(cache, b, range(tot)))
        G = Hq // kc.shape[1]
        for i in range(n):
            see = torch.tensor([j for j in range(tot) if j < lens[b] or sees[b][i][j - lens[b]]], dtype=torch.long, device="cuda")
            qi = q[n0 + i].double().view(-1, G, D)
            if len(see) == 0:
                outs.append(torch.zeros(Hq, D, dtype=torch.float64, device="cuda"))
                bounds.append(outs[-1])
                continue
            kk = (kc[see] * ks[see][..., None]).permute(1, 2, 0).contiguous()
            vv, s = (vc[see] * vs[see][..., None]).transpose(0, 1).contiguous(), vs[see].t()[:, None]
            sc = torch.matmul(qi, kk) * scale
            e = (D + 8) * E32 * abs(scale) * torch.matmul(qi.abs(), kk.abs()).amax(2, keepdim=True)
            w = torch.softmax(sc, 2)
            o, mag = torch.matmul(w, vv), torch.matmul(w, vv.abs())
            most = (w * s).amax(2, keepdim=True)
            lost = torch.minimum(most * 2.0 ** -22, w * s) * (w * s < most * 2.0 ** -12)
            rel = 4 * e + 2.0 ** -15 + 1.01 * U[FP16] + (len(see) / 16 + 64) * E32
            bd = rel * mag + torch.matmul(lost, vc[see].abs().transpose(0, 1).contiguous())
            outs.append(o.reshape(Hq, D))
            bounds.append((bd + U[dt] * 1.01 * (o.abs() + bd) + TINY[dt]).reshape(Hq, D))
        n0 += n
    return torch.stack(outs), torch.stack(bounds)


ATTEND = [
    # lens, new, page, Hq, Hkv, D, type, chain
    ([0], [1], 64, 1, 1, 64, BF16, True), ([1], [1], 64, 4, 2, 64, FP16, True), ([63, 64, 65], [1, 1, 1], 64, 8, 2, 128, BF16, True),
    ([100, 0, 7, 64], [5, 3, 1, 16], 64, 6, 2, 64, BF16, False), ([63, 200], [17, 2], 64, 8, 8, 128, FP16, False),
    ([500], [64], 128, 12, 4, 64, BF16, False), ([1000, 3], [9, 40], 64, 16, 2, 128, BF16, False),
    ([77], [3], 1024, 5, 1, 256, FP16, False), ([300, 5], [20, 33], 64, 24, 8, 256, BF16, False),
    ([0, 0], [130, 66], 64, 2, 1, 64, FP16, True), ([0], [70], 64, 16, 1, 128, BF16, False), ([5000], [1], 64, 8, 1, 128, BF16, True),
    ([3000, 10, 4097], [4, 2, 1], 256, 4, 4, 64, FP16, False), ([2500], [11], 64, 64, 1, 128, FP16, False),
    ([40] * 9, [1, 2, 0, 4, 5, 0, 7, 8, 2], 64, 10, 2, 64, BF16, False), ([6000], [40], 64, 4, 1, 256, BF16, False),
    ([128], [8], 64, 3, 3, 128, BF16, True), ([700], [40], 64, 4, 1, 128, FP16, False)]


@pytest.mark.parametrize("lens,new,page,Hq,Hkv,D,dt,chain", ATTEND)
def test_attend(lens, new, page, Hq, Hkv, D, dt, chain):
    cache, off = qbatch(lens, new, page, Hkv, D, dt, 31, junk=True)
    g, tot = gen(8), sum(lens) + sum(new)
    fill(cache, lens, new, torch.randn(tot, Hkv, D, device="cuda", generator=g),
         torch.randn(tot, Hkv, D, device="cuda", generator=g) * torch.randn(tot, Hkv, 1, device="cuda", generator=g).exp())
    N = sum(new)
    wide = torch.randn(N, Hq + 3, D, device="cuda", generator=g).to(dt)
    q = wide[:, 1:1 + Hq]
    parents = [tree(n, 3 + b) for b, n in enumerate(new)]
    mask = None if chain else P().tree_mask(parents)
    sees = chain_sees(new) if chain else tree_sees(parents)
    scale = D ** -0.5
    most = max(a + n for a, n in zip(lens, new))
    out = cache.attend(q, off, max(new), most, mask=mask, scale=scale)
    assert cache.status_value() == 0
    want, bound = attention_want(cache, lens, new, q, sees, scale, dt)
    within(out, want, bound, "attend")
    assert torch.equal(cache.attend(q, off, max(new), most, mask=mask, scale=scale), out)
    # the host's idea of the longest sequence changes the split, not the result's meaning
    for guess in (0, 40000):
        within(cache.attend(q, off, max(new), guess, mask=mask, scale=scale), want, bound, "attend, another split")
    room = torch.full((N, Hq + 1, D), 5.0, device="cuda").to(dt)
    cache.attend(q, off, max(new), most, mask=mask, scale=scale, out=room[:, :Hq])
    assert torch.equal(room[:, :Hq], out) and (room[:, Hq] == 5).all()
    within(cache.attend(q, off, max(new) + 3, most, mask=mask, scale=scale), want, bound, "attend, another max_new")


@pytest.mark.parametrize("big", [0.0, 30.0, -30.0])
def test_attend_large_scores_and_scales(big):
    cache, off = qbatch([700], [6], 64, 2, 64, BF16, 41)
    q = 4 * torch.randn(6, 4, 64, device="cuda", generator=gen(1)).to(BF16)
    k = torch.randn(706, 2, 64, device="cuda", generator=gen(2))
    k[..., 0] += big
    fill(cache, [700], [6], k, torch.randn(706, 2, 64, device="cuda", generator=gen(3)))
    for scale in (1.0, -0.7, 0.0):
        out = cache.attend(q, off, 6, 706, scale=scale)
        want, bound = attention_want(cache, [700], [6], q, chain_sees([6]), scale, BF16)
        within(out, want, bound, "scale %g" % scale)


@pytest.mark.parametrize("D,new", [(64, 2), (128, 40), (256, 3)])
def test_attend_values_of_any_scale(D, new):
    """Tokens whose values are zeros take their share of the softmax, and large values of tokens
    that hardly count, or that a row does not see, leave the others' as they are."""
    ctx = 300
    cache, off = qbatch([ctx], [new], 64, 1, D, BF16, 43)
    tot = ctx + new
    k = torch.randn(tot, 1, D, device="cuda", generator=gen(2))
    v = torch.randn(tot, 1, D, device="cuda", generator=gen(3))
    v[::3] = 0
    v[1::3] *= (torch.rand(v[1::3].shape[0], 1, 1, device="cuda", generator=gen(4)) * 60 - 45).exp2()
    k[::3] *= 2
    v[ctx + new - 1] *= 2.0 ** 50
    fill(cache, [ctx], [new], k, v)
    q = torch.randn(new, 4, D, device="cuda", generator=gen(1)).to(BF16)
    out = cache.attend(q, off, new, tot, scale=0.3)
    want, bound = attention_want(cache, [ctx], [new], q, chain_sees([new]), 0.3, BF16)
    within(out, want, bound)
    # all values zero: zeros
    cache.v_scale.fill_(2.0 ** -64)
    cache.v.zero_()
    assert (cache.attend(q, off, new, tot, scale=0.3) == 0).all()


@pytest.mark.parametrize("D,Hq", [(64, 2), (128, 8), (256, 4)])
@pytest.mark.parametrize("ctx", [0, 5, 90, 3000])
def test_attend_masked_places_may_hold_anything(D, Hq, ctx):
    """Drafts that a token does not see do not reach it, whatever they hold."""
    new = [12, 70]
    cache, off = qbatch([ctx, ctx + 9], new, 64, 2, D, BF16, 51)
    q = torch.randn(82, Hq, D, device="cuda", generator=gen(3)).to(BF16)
    parents = [tree(12, 1, fan=4), tree(70, 2, fan=30)]
    mask, sees = P().tree_mask(parents), tree_sees(parents)
    clean = cache.attend(q, off, 70, ctx + 79, mask=mask)
    bad = {0: [(3, "k_scale"), (5, "v_scale")], 1: [(10, "v_scale"), (65, "k_scale")]}
    for b, items in bad.items():
        for i, what in items:
            slot = [ctx, ctx + 9][b] + i
            getattr(cache, what)[int(cache.table[b, slot // 64]), :, slot % 64] = math.nan
    out = cache.attend(q, off, 70, ctx + 79, mask=mask)
    n = 0
    for b in range(2):
        for i in range(new[b]):
            if any(sees[b][i][j] for j, _ in bad[b]):
                assert out[n + i].isnan().all()
            else:
                assert torch.equal(out[n + i], clean[n + i]), (b, i)
        n += new[b]


def test_attend_empty_rows_and_mask_words():
    cache, off = qbatch([0, 40], [3, 3], 64, 2, 64, FP16, 61)
    q = torch.randn(6, 4, 64, device="cuda", generator=gen(3)).to(FP16)
    mask = torch.zeros(6, 2, dtype=torch.int64, device="cuda")
    mask[1, 0] = 0b10
    out = cache.attend(q, off, 3, 43, mask=mask)
    assert (out[[0, 2]] == 0).all()
    kc, ks, vc, vs = qrows(cache, 0, [1])
    one = (vc.double() * vs.double()[..., None])[0].repeat_interleave(2, 0)
    within(out[1], one, (U[FP16] + 8 * E32) * one.abs() + TINY[FP16])
    more = mask.clone()
    more[:, 0] |= -8          # bits 3 .. 63: no such drafts
    more[:, 1] = -1
    assert torch.equal(cache.attend(q, off, 3, 43, mask=more), out)
    want, bound = attention_want(cache, [0, 40], [3, 3], q, [[[False] * 3] * 3] * 2, 64 ** -0.5, FP16)
    within(out[3:], want[3:], bound[3:])
    none, kept = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.full_like(q, 2.0)
    cache.attend(q, none, 3, 43, mask=mask, out=kept)
    assert (kept == 2).all()


@pytest.mark.parametrize("new", [2, 20])
def test_attend_skips_pages_out_of_range(new):
    cache, off = qbatch([200, 50], [new, new], 64, 1, 64, BF16, 71)
    q = torch.randn(2 * new, 4, 64, device="cuda", generator=gen(3)).to(BF16)
    good = cache.attend(q, off, new, 200 + new)
    saved = cache.table.clone()
    for bad in (-1, cache.k.shape[0], 1 << 30):
        cache.status.zero_()
        cache.table[0, 1] = bad
        out = cache.attend(q, off, new, 200 + new)
        assert cache.status_value() == -5
        assert torch.equal(out[new:], good[new:])
        # slots 64 .. 127 are not followed: the same as attention without them
        cache.table.copy_(saved)
        left = [j for j in range(200 + new) if j < 64 or j >= 128]
        kc, ks, vc, vs = (x.double() for x in qrows(cache, 0, left))
        sc = (q[new - 1].double() @ (kc * ks[..., None])[:, 0].t()) / 8
        want = torch.softmax(sc, 1) @ (vc * vs[..., None])[:, 0]
        assert (out[new - 1].double() - want).abs().max().item() < 4 * U[BF16] * (vc * vs[..., None]).abs().max().item()
    cache.status.zero_()
    cache.lens[0] = -3
    kept = torch.full_like(q, 2.0)
    cache.attend(q, off, new, 200 + new, out=kept)
    assert cache.status_value() == -5 and (kept[:new] == 2).all() and torch.equal(kept[new:], good[new:])


def test_cache_past_32_bits():
    """Pages whose codes lie past 2^31 from the start of k and v."""
    page, Hkv, D = 64, 8, 128
    n_pages = (1 << 31) // (page * Hkv * D) + 6
    k = torch.empty(n_pages, Hkv, page, D, dtype=torch.int8, device="cuda")
    v = torch.empty(n_pages, Hkv, D, page, dtype=torch.int8, device="cuda")
    ks, vs = (torch.empty(n_pages, Hkv, page, device="cuda") for _ in "kv")
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, n_pages - 3]], dtype=torch.int32, device="cuda")
    cache = P().QuantPagedCache(k, v, ks, vs, table, torch.tensor([0], dtype=torch.int32, device="cuda"))
    kv = torch.randn(200, 2 * Hkv, D, device="cuda", generator=gen(1)).to(BF16)
    off = torch.tensor([0, 200], dtype=torch.int32, device="cuda")
    cache.append(None, kv[:, :Hkv], kv[:, Hkv:], off, 200)
    got = cache.read(cache.lens, off, 200, rows=200)
    for x, y in zip(got, (kv[:, :Hkv], kv[:, Hkv:])):
        top = y.double().abs().amax(-1, keepdim=True)
        within(x, y, (HALF / 127 + U[BF16]) * top)
    q = torch.randn(200, Hkv, D, device="cuda", generator=gen(2)).to(BF16)
    out = cache.attend(q, off, 200, 200)
    want, bound = attention_want(cache, [0], [200], q, chain_sees([200]), D ** -0.5, BF16)
    within(out, want, bound)
    cache.lens.fill_(100)
    one = torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    cache.keep(one, torch.tensor([[5, 60, 99]], dtype=torch.int32, device="cuda"),
               torch.tensor([3], dtype=torch.int32, device="cuda"))
    three = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    now = cache.read(cache.lens, three, 3, rows=3)
    assert all(torch.equal(x, y[[105, 160, 199]]) for x, y in zip(now, got))


@pytest.mark.parametrize("page,Hkv,D", [(64, 2, 64), (64, 8, 128), (128, 1, 256)])
def test_keep(page, Hkv, D):
    lens, new = [0, 30, 64, 127, 500, 9], [40, 40, 70, 70, 5, 3]
    paths = [[0, 1, 2], [3, 9, 39], list(range(0, 70, 2)), [69], [], [0, 2]]
    cache, off = qbatch(lens, new, page, Hkv, D, BF16, 81)
    wide = max(map(len, paths))
    keep = torch.tensor([p + [-7] * (wide - len(p)) for p in paths], dtype=torch.int32, device="cuda")
    n = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    want = []
    for b, p in enumerate(paths):
        rows = list(range(lens[b])) + [lens[b] + i for i in p] + list(range(lens[b] + len(p), lens[b] + new[b]))
        want.append(qrows(cache, b, rows))
    out = cache.keep(off, keep, n)
    assert cache.status_value() == 0
    assert out.tolist() == [a + len(p) for a, p in zip(lens, paths)]
    for b in range(len(lens)):
        for got, w in zip(qrows(cache, b, range(lens[b] + new[b])), want[b]):
            assert torch.equal(got, w), b


def test_keep_refuses_bad_lists():
    cache, off = qbatch([10, 20, 30, 40, 50], [4, 4, 4, 4, 4], 64, 2, 64, BF16, 91)
    names = ("k", "v", "k_scale", "v_scale")
    was = {x: getattr(cache, x).clone() for x in names}
    keep = torch.tensor([[0, 2, 1], [1, 1, 2], [2, 3, 4], [-1, 0, 1], [1, 2, 3]], dtype=torch.int32, device="cuda")
    n = torch.tensor([3, 2, 3, 3, 4], dtype=torch.int32, device="cuda")
    out = cache.keep(off, keep, n)
    assert cache.status_value() == -5 and out.tolist() == [10, 20, 30, 40, 50]
    assert all(torch.equal(getattr(cache, x), was[x]) for x in names)


# ------------------------------------------------------------------ a run of them together
def test_calls_on_another_stream():
    cache, off = qbatch([4000], [1], 64, 2, 128, BF16, 95)
    qs = [torch.randn(1, 8, 128, device="cuda", generator=gen(i)).to(BF16) for i in range(2)]
    want = [cache.attend(q, off, 1, 4001) for q in qs]
    read = cache.read(cache.lens, off, 1, rows=1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for _ in range(20):
        for i in range(2):
            outs[i].append(cache.attend(qs[i], off, 1, 4001, stream=streams[i]))
    other = cache.read(cache.lens, off, 1, rows=1, stream=streams[0])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])
    assert all(torch.equal(a, b) for a, b in zip(read, other))


def test_calls_in_a_captured_graph():
    """A step captured once and replayed over changing inputs, with eager work in between,
    gives what the eager calls give each time."""
    cache, off = qbatch([900, 2000], [3, 5], 64, 2, 128, BF16, 96)
    x = torch.randn(8, 12, 128, device="cuda", generator=gen(3)).to(BF16)
    w = 1 + 0.1 * torch.randn(128, device="cuda", generator=gen(4))
    keep = torch.tensor([[0, 2], [1, 4]], dtype=torch.int32, device="cuda")
    n, lens = torch.tensor([2, 2], dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    out, two = torch.empty(8, 8, 128, dtype=BF16, device="cuda"), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    k_out, v_out = (torch.empty(4, 2, 128, dtype=BF16, device="cuda") for _ in "kv")

    def step():
        q = cache.append(x[:, :8], x[:, 8:10], x[:, 10:], off, 5, w_q=w, w_k=w)
        cache.attend(q, off, 5, 2005, out=out)
        cache.keep(off, keep, n, len_out=lens)
        cache.read(cache.lens, two, 2, k_out=k_out, v_out=v_out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    big = torch.randn(8, 64, 128, device="cuda", generator=gen(4)).to(BF16)
    for s in [torch.cuda.current_stream(), side]:     # eager calls that need a larger workspace
        cache.attend(big, off, 5, 200000, stream=s)
    torch.cuda.synchronize()
    for i in range(4):
        x.copy_(torch.randn(8, 12, 128, device="cuda", generator=gen(10 + i)).to(BF16))
        step()
        torch.cuda.synchronize()
        every = (out, k_out, v_out, lens, cache.k, cache.v, cache.k_scale, cache.v_scale)
        want = [t.clone() for t in every]
        for t in every[:4]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(every, want))


def test_block_over_a_cache_in_8_bits():
    """A block with normed heads: over a cache in 8 bits a tree of drafts gives, for every path,
    what the tokens give one after another, and it is near to the same over 16 bits."""
    import moe_inputs as mi
    pkg = P()
    wk = mi.WORKLOADS["tiny"]
    d, Hq, Hkv, D = wk.layer.d_model, 4, 2, 64
    g = gen(77)

    def w(*shape):
        return 0.05 * torch.randn(*shape, device="cuda", generator=g)
    ang = torch.arange(256, device="cuda")[:, None] * 100.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
    inputs = mi.LayerInputs(wk.layer)
    blocks = [pkg.DecoderBlock(pkg.MoELayer(inputs, device="cuda:0"), w((Hq + 2 * Hkv) * D, d), w(d, Hq * D), Hq, Hkv, D,
                               dict(attn=1 + w(d), ffn=1 + w(d), q=1 + w(D), k=1 + w(D)), ang.cos(), ang.sin(), group=64)
              for _ in range(2)]
    embed = torch.randn(64, d, device="cuda", generator=g)

    def forward(caches, tokens, new, positions, mask):
        off = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        r = embed[tokens].clone()
        h = torch.empty(new, d, dtype=BF16, device="cuda")
        pkg.moe_block_norm(r, h, w_pre=blocks[0].norms["attn"])
        for i, b in enumerate(blocks):
            b.forward(r, h, caches[i], off, new, 200, positions, mask, blocks[1].norms["attn"] if i == 0 else None)
        return r.clone(), off
    parents = [-1, 0, 0, 1, 2, 4, -1, 6]
    tokens = torch.tensor([5, 9, 11, 3, 40, 8, 21, 2], device="cuda")
    depth = [0, 1, 1, 2, 2, 3, 0, 1]
    pos = torch.tensor([30 + x for x in depth], dtype=torch.int32, device="cuda")
    prompt = torch.arange(30, device="cuda") % 64
    results = []
    for kind in (pkg.QuantPagedCache, pkg.PagedCache):
        caches, plain = ([kind.create(1, 200, Hkv, D) for _ in blocks] for _ in range(2))
        for cs in (caches, plain):
            forward(cs, prompt, 30, None, None)
            for c in cs:
                c.lens.fill_(30)
        tree_r, off = forward(caches, tokens, 8, pos, pkg.tree_mask([parents]))
        path = [0, 2, 4, 5]
        for i, node in enumerate(path):
            one, _ = forward(plain, tokens[node:node + 1], 1, None, None)
            # bf16 activations of two layers, and codes that fall the other way with them
            assert ((one[0] - tree_r[node]).norm() / one[0].norm()).item() < 2e-2, i
            for c in plain:
                c.lens.add_(1)
        for c in caches:
            c.lens.copy_(c.keep(off, torch.tensor([path], dtype=torch.int32, device="cuda"),
                                torch.tensor([4], dtype=torch.int32, device="cuda")))
        a, _ = forward(caches, tokens[3:4], 1, None, None)
        b, _ = forward(plain, tokens[3:4], 1, None, None)
        assert ((a - b).norm() / b.norm()).item() < 2e-2
        assert all(c.status_value() == 0 for c in caches + plain)
        results.append(tree_r)
    # a code is off by 2^-8 of a row's largest value at most: less than a hundredth in norm, twice
    assert ((results[0] - results[1]).norm() / results[1].norm()).item() < 2e-2


def test_tensors_that_do_not_fit_are_refused():
    """Types, shapes, strides and devices, before any device work: nothing is written."""
    pkg = P()
    cache, off = qbatch([10, 20], [2, 3], 64, 2, 64, BF16, 4)
    was = cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone()
    kv = torch.randn(5, 2, 64, device="cuda").to(BF16)
    q, w, tab = torch.randn(5, 4, 64, device="cuda").to(BF16), torch.ones(64, device="cuda"), torch.ones(50, 32, device="cuda")
    pos = torch.arange(5, device="cuda").int()
    ok = dict(q=q, k=kv, v=kv, new_off=off, max_new=3, positions=pos, cos=tab, sin=tab, w_q=w, w_k=w)
    wide = torch.randn(5, 4, 128, device="cuda").to(BF16)
    for bad in (dict(k=kv.half()), dict(k=kv[:, :1]), dict(k=kv.cpu()), dict(v=kv[:4]), dict(q=wide[..., ::2]), dict(q=q.float()),
                dict(q=q.transpose(0, 1)), dict(q=q.cpu()), dict(w_q=w[:32]), dict(w_k=w.half()), dict(w_k=w.cpu()),
                dict(positions=pos.long()), dict(positions=pos[:4]), dict(cos=None), dict(sin=tab[:40]), dict(cos=tab.t()),
                dict(new_off=off[:2]), dict(new_off=off.long()), dict(q_out=q[:, :2]), dict(max_new=1 << 40), dict(k=None)):
        with pytest.raises((pkg.MoEError, AttributeError, TypeError)):
            cache.append(**dict(ok, **bad))
    with pytest.raises(pkg.MoEError):
        pkg.moe_cache_append_norm(cache.desc, cache.table, cache.lens, off, 3, q, kv, kv, q, w, w)   # another kind of cache
    mask = torch.zeros(5, 1, dtype=torch.int64, device="cuda")
    for bad in (dict(q=q.half()), dict(q=wide), dict(mask=mask.int()), dict(mask=mask[:3]), dict(out=q[:, :3]), dict(scale=math.inf),
                dict(new_off=off.cpu()), dict(q=wide[..., 1:65])):
        with pytest.raises(pkg.MoEError):
            cache.attend(**dict(dict(q=q, new_off=off, max_new=3, max_len=23), **bad))
    for bad in (dict(k_out=kv[:, :1]), dict(k_out=kv.half()), dict(first=cache.lens.long()), dict(row_off=off[:2]), dict(v_out=kv)):
        with pytest.raises(pkg.MoEError):
            cache.read(**dict(dict(first=cache.lens, row_off=off, max_rows=3, k_out=kv), **bad))
    with pytest.raises(pkg.MoEError):
        cache.read(cache.lens, off, 3)
    keep, n = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (dict(keep=keep.long()), dict(keep=keep.t()), dict(n_keep=n[:1]), dict(len_out=cache.lens), dict(len_out=n)):
        with pytest.raises(pkg.MoEError):
            cache.keep(**dict(dict(new_off=off, keep=keep if "keep" not in bad else None, n_keep=n), **bad))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(was, (cache.k, cache.v, cache.k_scale, cache.v_scale)))


def test_empty_masks_and_tables_are_refused():
    """They have no address, which would say that there is none: a chain, no rotation."""
    pkg = P()
    cache, off = qbatch([10, 20], [2, 3], 64, 2, 64, BF16, 4)
    kv, q = torch.randn(5, 2, 64, device="cuda").to(BF16), torch.randn(5, 4, 64, device="cuda").to(BF16)
    with pytest.raises(pkg.MoEError, match="mask"):
        cache.attend(q, off, 3, 23, mask=torch.zeros(5, 0, dtype=torch.int64, device="cuda"))
    plain = pkg.PagedCache.create(2, 64, 2, 64)
    for shape in ((0, 32), (50, 0)):
        none = torch.zeros(*shape, device="cuda")
        for c, kw in ((cache, {}), (plain, dict(w_k=torch.ones(64, device="cuda")))):
            with pytest.raises(pkg.MoEError, match="cos"):
                c.append(q, kv, kv, off, 3, cos=none, sin=none, **kw)
