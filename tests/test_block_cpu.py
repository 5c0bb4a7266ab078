"""The decoder block's entry points refuse bad arguments on the host, before any
device work (no compute call is made here); mask words of drafted trees."""
import ctypes as C

import numpy as np
import pytest

FAKE = 1 << 20                  # non-NULL, 16-byte aligned, never dereferenced
OTHER = 1 << 30
ODD = FAKE + 2
ARG, BITS, ALIGN, WS = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2503_21135_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2503_21135_amd import build
        build.build()
    return _lib.load()


def caller(f, ok):
    def call(**kw):
        assert set(kw) <= set(ok)
        return f(*dict(ok, **kw).values())
    return call


def test_linear_refusals(lib):
    call = caller(lib.moe_quant_linear, dict(
        x=FAKE, xt=0, ldx=256, T=4, K=256, codes=FAKE, ldc=32, sz=FAKE, srs=1, sgs=64, R=64, bits=4, group=64,
        bias=None, y=FAKE, yt=2, ldy=64, stream=None))
    for b in (2, 3, 8, 16, 5):
        assert call(bits=b) == BITS
    for kw in (dict(group=32), dict(K=200), dict(K=0), dict(T=-1), dict(R=-1), dict(xt=2), dict(xt=5), dict(yt=1),
               dict(yt=3), dict(T=1 << 23), dict(R=1 << 28, ldy=1 << 28), dict(x=None), dict(codes=None), dict(sz=None), dict(y=None), dict(ldx=248), dict(ldy=63),
               dict(ldc=28), dict(srs=0), dict(sgs=-1), dict(K=192, group=128)):
        assert call(**kw) == ARG, kw
    for kw in (dict(x=ODD), dict(ldx=260), dict(codes=ODD), dict(ldc=33), dict(sz=ODD), dict(y=ODD), dict(bias=ODD)):
        assert call(**kw) == ALIGN, kw
    assert call(T=0) == 0 and call(R=0) == 0    # nothing to do, no device call


def test_norm_refusals(lib):
    call = caller(lib.moe_block_norm, dict(
        y=FAKE, yt=2, ldy=64, r=OTHER, rt=0, ldr=64, T=4, d=64, wp=None, gate=None, gt=0, grs=0, gcs=0, a=1.0, b=1.0,
        w=None, eps=1e-6, ro=OTHER, ldro=64, h=OTHER + (1 << 20), ht=0, ldh=64, stream=None))
    for kw in (dict(T=-1), dict(d=0), dict(eps=-1.0), dict(eps=float("nan")), dict(yt=3), dict(rt=-1), dict(ht=9),
               dict(y=None, wp=FAKE), dict(y=None, gate=FAKE), dict(gate=FAKE, gcs=2), dict(gate=FAKE, grs=-1),
               dict(gate=FAKE, gt=7), dict(r=None), dict(ro=None, h=None), dict(ldr=63), dict(ldy=1), dict(ldro=8),
               dict(ldh=63),
               dict(h=OTHER),                   # both outputs in one place
               dict(h=OTHER + 2, ro=None),      # an output one element behind its input
               dict(ro=OTHER, ldro=72),         # in place with other rows
               dict(ro=None, h=FAKE)):          # in place over another type
        assert call(**kw) == ARG, kw
    for kw in (dict(y=FAKE + 2), dict(r=OTHER + 1, ro=None), dict(wp=ODD), dict(w=ODD), dict(h=OTHER + (1 << 20) + 1)):
        assert call(**kw) == ALIGN, kw
    assert call(T=0) == 0


def cache_desc(**kw):
    from paper_2503_21135_amd._lib import CacheDesc
    d = CacheDesc()
    for k, v in dict(dict(k=FAKE, v=OTHER, n_pages=8, n_heads=2, head_dim=64, page_size=32, type=0), **kw).items():
        setattr(d, k, v)
    return C.byref(d)


BAD_CACHE = [dict(n_pages=0), dict(n_heads=0), dict(head_dim=80), dict(page_size=16), dict(page_size=48),
             dict(page_size=2048), dict(type=2)]


def test_append_refusals(lib):
    call = caller(lib.moe_cache_append, dict(
        c=cache_desc(), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, N=6, mx=4, q=FAKE, ldq=256, Hq=4, k=FAKE, ldk=128,
        v=FAKE, ldv=128, pos=None, cos=None, sin=None, rot=0, mp=0, il=0, qo=OTHER, ldqo=256, st=None, stream=None))
    for kw in [dict(c=cache_desc(**b)) for b in BAD_CACHE] + [
            dict(c=None), dict(c=cache_desc(k=None)), dict(table=None), dict(pages=0), dict(lens=None), dict(off=None),
            dict(B=-1), dict(B=70000), dict(N=-1), dict(mx=-1), dict(qo=None), dict(q=None), dict(Hq=0), dict(ldq=255),
            dict(ldqo=128), dict(q=OTHER, ldq=512), dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=64), dict(cos=FAKE),
            dict(cos=FAKE, sin=FAKE, rot=3, mp=9), dict(cos=FAKE, sin=FAKE, rot=66, mp=9),
            dict(cos=FAKE, sin=FAKE, rot=64, mp=0)]:
        assert call(**kw) == ARG, kw
    for kw in (dict(c=cache_desc(v=ODD)), dict(table=ODD), dict(lens=ODD), dict(off=ODD), dict(q=FAKE + 1), dict(pos=ODD)):
        assert call(**kw) == ALIGN, kw
    assert call(B=0) == 0 and call(N=0) == 0 and call(mx=0) == 0


def test_attention_refusals(lib):
    ns, wb = C.c_int32(0), C.c_size_t(0)
    plan = lib.moe_tree_attention_plan
    assert plan(cache_desc(), 4, 2, 4, 40000, C.byref(ns), C.byref(wb)) == 0 and ns.value >= 1
    need = wb.value
    call = caller(lib.moe_tree_attention, dict(
        c=cache_desc(), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, N=6, mx=4, ml=40000, q=FAKE, ldq=256, Hq=4, mask=FAKE,
        mw=1, scale=0.125, out=OTHER, ldo=256, st=None, ws=FAKE, wsb=need, stream=None))
    for kw in [dict(c=cache_desc(**b)) for b in BAD_CACHE] + [
            dict(c=None), dict(c=cache_desc(v=None)), dict(table=None), dict(pages=0), dict(lens=None), dict(off=None),
            dict(B=-1), dict(N=-1), dict(mx=-1), dict(ml=-1), dict(Hq=3), dict(Hq=0), dict(Hq=130), dict(mw=0),
            dict(scale=float("inf")), dict(scale=float("nan")), dict(q=None), dict(out=None), dict(ldq=255), dict(ldo=8),
            dict(q=OTHER), dict(mx=1 << 24)]:
        assert call(**kw) == ARG, kw
    for kw in (dict(q=ODD), dict(ldq=260), dict(out=OTHER + 1), dict(mask=FAKE + 4), dict(c=cache_desc(k=ODD))):
        assert call(**kw) == ALIGN, kw
    if need:
        assert call(ws=None) == WS and call(wsb=need - 1) == WS
    assert call(B=0) == 0 and call(N=0) == 0 and call(mx=0) == 0
    for b in BAD_CACHE:
        assert plan(cache_desc(**b), 4, 2, 4, 100, None, None) == ARG
    assert plan(cache_desc(), 3, 2, 4, 100, None, None) == ARG


def test_keep_refusals(lib):
    call = caller(lib.moe_cache_keep, dict(c=cache_desc(), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, keep=FAKE, mk=4,
                                           n=FAKE, lo=OTHER, st=None, stream=None))
    for kw in [dict(c=cache_desc(**b)) for b in BAD_CACHE] + [
            dict(table=None), dict(pages=0), dict(lens=None), dict(B=-1), dict(B=70000), dict(mk=-1), dict(keep=None), dict(n=None),
            dict(lo=FAKE)]:
        assert call(**kw) == ARG, kw
    for kw in (dict(keep=ODD), dict(n=ODD), dict(lo=OTHER + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(B=0) == 0


def test_tensor_checks_before_the_call():
    import torch

    import paper_2503_21135_amd as P
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    sz = torch.zeros(1, 8, dtype=torch.int32)
    with pytest.raises(P.MoEError if hasattr(P, "MoEError") else RuntimeError):
        P.moe_quant_linear(x, torch.zeros(8, 8, dtype=torch.int32), sz, torch.zeros(2, 8))
    with pytest.raises(RuntimeError):
        P.moe_block_norm(x)
    with pytest.raises(RuntimeError):
        P.PagedCache(torch.zeros(1, 1, 32, 64), torch.zeros(1, 1, 64, 32), sz, sz)


def test_tree_mask_words():
    from paper_2503_21135_amd import MoEError, tree_mask
    m = tree_mask([[-1, 0, 0, 2], [-1]], device="cpu").numpy().view(np.uint64)
    assert m[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1101, 0b1]
    chain = tree_mask([list(range(-1, 129))], device="cpu").numpy().view(np.uint64)
    assert chain.shape == (130, 3)
    assert chain[63].tolist() == [2 ** 64 - 1, 0, 0] and chain[129].tolist() == [2 ** 64 - 1, 2 ** 64 - 1, 3]
    for bad in ([0], [-1, 1], [-2]):
        with pytest.raises(MoEError):
            tree_mask([bad], device="cpu")
