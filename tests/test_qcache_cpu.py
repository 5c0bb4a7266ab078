"""The cache in 8 bits, normed heads and the verification of drafts refuse bad arguments on
the host, before any device work (no compute call is made here)."""
import ctypes as C

import pytest

from test_block_cpu import ALIGN, ARG, BAD_CACHE, FAKE, ODD, OTHER, WS, cache_desc, caller, lib  # noqa: F401

FAR = 1 << 34


def qcache_desc(**kw):
    from paper_2503_21135_amd._lib import QuantCacheDesc
    d = QuantCacheDesc()
    for k, v in dict(dict(k=FAKE, v=OTHER, k_scale=FAR, v_scale=FAR + 65536, n_pages=8, n_heads=2, head_dim=64, page_size=64,
                          type=0), **kw).items():
        setattr(d, k, v)
    return C.byref(d)


BAD_QCACHE = BAD_CACHE + [dict(page_size=32), dict(head_dim=32), dict(type=-1)]


@pytest.mark.parametrize("kind", ["16", "8"])
def test_normed_append_refusals(lib, kind):  # noqa: F811
    desc, bad = (cache_desc, BAD_CACHE) if kind == "16" else (qcache_desc, BAD_QCACHE)
    call = caller(lib.moe_cache_append_norm if kind == "16" else lib.moe_qcache_append, dict(
        c=desc(), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, N=6, mx=4, q=FAKE, ldq=256, Hq=4, k=FAKE, ldk=128,
        v=FAKE, ldv=128, wq=FAKE, wk=FAKE, eps=1e-6, pos=None, cos=None, sin=None, rot=0, mp=0, il=0, qo=FAR + (1 << 20),
        ldqo=256, st=None, stream=None))
    for kw in [dict(c=desc(**b)) for b in bad] + [
            dict(c=None), dict(c=desc(k=None)), dict(table=None), dict(pages=0), dict(lens=None), dict(off=None),
            dict(B=-1), dict(B=70000), dict(N=-1), dict(mx=-1), dict(qo=None), dict(q=None), dict(Hq=0), dict(ldq=255),
            dict(ldqo=128), dict(q=FAR + (1 << 20), ldq=512), dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=64), dict(cos=FAKE),
            dict(cos=FAKE, sin=FAKE, rot=3, mp=9), dict(cos=FAKE, sin=FAKE, rot=66, mp=9), dict(qo=OTHER),
            dict(cos=FAKE, sin=FAKE, rot=64, mp=0), dict(eps=-1.0), dict(eps=float("nan"))]:
        assert call(**kw) == ARG, kw
    for kw in (dict(c=desc(v=ODD)), dict(table=ODD), dict(lens=ODD), dict(off=ODD), dict(q=FAKE + 1), dict(pos=ODD),
               dict(wq=ODD), dict(wk=FAKE + 1)):
        assert call(**kw) == ALIGN, kw
    if kind == "8":
        assert call(c=desc(k_scale=None)) == ARG and call(c=desc(v_scale=FAR + 8)) == ALIGN
        assert call(qo=FAR + 64) == ARG      # over the scales
    assert call(B=0) == 0 and call(N=0) == 0 and call(mx=0) == 0


def test_read_refusals(lib):  # noqa: F811
    call = caller(lib.moe_qcache_read, dict(c=qcache_desc(), table=FAKE, pages=4, first=FAKE, B=2, off=FAKE, N=6, mx=4,
                                            ko=FAR + (1 << 20), ldk=128, vo=FAR + (1 << 21), ldv=128, st=None, stream=None))
    for kw in [dict(c=qcache_desc(**b)) for b in BAD_QCACHE] + [
            dict(c=None), dict(table=None), dict(pages=0), dict(first=None), dict(off=None), dict(B=-1), dict(B=70000), dict(N=-1),
            dict(mx=-1), dict(ko=None, vo=None), dict(ldk=127), dict(ldv=127), dict(vo=FAR + (1 << 20)), dict(ko=OTHER),
            dict(vo=FAKE), dict(ko=FAR)]:
        assert call(**kw) == ARG, kw
    for kw in (dict(c=qcache_desc(k=ODD)), dict(first=ODD), dict(ko=FAR + (1 << 20) + 1), dict(vo=FAR + (1 << 21) + 1)):
        assert call(**kw) == ALIGN, kw
    assert call(B=0) == 0 and call(N=0) == 0 and call(mx=0) == 0


def test_attention_refusals(lib):  # noqa: F811
    ns, wb = C.c_int32(0), C.c_size_t(0)
    plan = lib.moe_qcache_attention_plan
    assert plan(qcache_desc(), 4, 2, 4, 40000, C.byref(ns), C.byref(wb)) == 0 and ns.value > 1
    need, away = wb.value, FAR + (1 << 20)
    call = caller(lib.moe_qcache_attention, dict(
        c=qcache_desc(), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, N=6, mx=4, ml=40000, q=FAKE, ldq=256, Hq=4, mask=FAKE,
        mw=1, scale=0.125, out=away, ldo=256, st=None, ws=FAKE, wsb=need, stream=None))
    for kw in [dict(c=qcache_desc(**b)) for b in BAD_QCACHE] + [
            dict(c=None), dict(c=qcache_desc(v=None)), dict(c=qcache_desc(v_scale=None)), dict(table=None), dict(pages=0),
            dict(lens=None), dict(off=None), dict(B=-1), dict(N=-1), dict(mx=-1), dict(ml=-1), dict(Hq=3), dict(Hq=0),
            dict(Hq=130), dict(mw=0), dict(scale=float("inf")), dict(scale=float("nan")), dict(q=None), dict(out=None),
            dict(ldq=255), dict(ldo=8), dict(q=away), dict(mx=1 << 24), dict(out=OTHER), dict(out=FAR)]:
        assert call(**kw) == ARG, kw
    for kw in (dict(q=ODD), dict(ldq=260), dict(out=away + 1), dict(mask=FAKE + 4), dict(c=qcache_desc(k=ODD)),
               dict(c=qcache_desc(k_scale=ODD))):
        assert call(**kw) == ALIGN, kw
    assert call(ws=None) == WS and call(wsb=need - 1) == WS and call(ws=ODD) == ALIGN
    assert call(B=0) == 0 and call(N=0) == 0 and call(mx=0) == 0
    for b in BAD_QCACHE:
        assert plan(qcache_desc(**b), 4, 2, 4, 100, None, None) == ARG
    assert plan(qcache_desc(), 3, 2, 4, 100, None, None) == ARG


def test_keep_refusals(lib):  # noqa: F811
    call = caller(lib.moe_qcache_keep, dict(c=qcache_desc(), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, keep=FAKE, mk=4,
                                            n=FAKE, lo=FAR + (1 << 20), st=None, stream=None))
    for kw in [dict(c=qcache_desc(**b)) for b in BAD_QCACHE] + [
            dict(table=None), dict(pages=0), dict(lens=None), dict(B=-1), dict(B=70000), dict(mk=-1), dict(keep=None), dict(n=None),
            dict(lo=FAKE), dict(lo=FAR)]:
        assert call(**kw) == ARG, kw
    for kw in (dict(keep=ODD), dict(n=ODD), dict(lo=FAR + (1 << 20) + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(B=0) == 0


def test_verify_refusals(lib):  # noqa: F811
    wb = C.c_size_t(0)
    plan = lib.moe_draft_verify_plan
    assert plan(2, 6, 4, 1000, C.byref(wb)) == 0
    need, out = wb.value, FAR
    call = caller(lib.moe_draft_verify, dict(
        lg=FAKE, lt=2, ld=1000, N=6, V=1000, tok=FAKE, par=FAKE, off=FAKE, B=2, mx=4, dr=FAKE, dt=0, ldd=1000, heat=FAKE, u=FAKE,
        un=FAKE, keep=out, nk=out + 64, nx=out + 128, st=None, ws=OTHER, wsb=need, stream=None))
    for kw in (dict(N=-1), dict(V=0), dict(B=-1), dict(B=70000), dict(mx=-1), dict(mx=1025), dict(lt=3), dict(dt=-1), dict(ld=999),
               dict(ldd=999), dict(lg=None), dict(tok=None), dict(off=None), dict(keep=None), dict(nk=None), dict(nx=None),
               dict(u=None), dict(un=None), dict(keep=FAKE), dict(nk=out), dict(nx=out + 68), dict(nx=OTHER), dict(keep=FAKE + 8)):
        assert call(**kw) == ARG, kw
    for kw in (dict(lg=ODD), dict(dr=FAKE + 1), dict(tok=ODD), dict(par=ODD), dict(off=ODD), dict(heat=ODD), dict(u=ODD), dict(un=ODD),
               dict(keep=out + 2), dict(nk=out + 66), dict(nx=out + 130), dict(st=ODD), dict(ws=OTHER + 8)):
        assert call(**kw) == ALIGN, kw
    assert call(ws=None) == WS and call(wsb=need - 1) == WS
    assert call(B=0) == 0
    for bad in ((-1, 6, 4, 1000), (2, -1, 4, 1000), (2, 6, 1025, 1000), (2, 6, 4, 0), (2, 6, 4, 1 << 29)):
        assert plan(*bad, None) == ARG


def test_tensor_checks_before_the_call():
    import torch

    import paper_2503_21135_amd as P
    i32 = torch.zeros(2, dtype=torch.int32)
    k, v, s = torch.zeros(1, 1, 64, 64, dtype=torch.int8), torch.zeros(1, 1, 64, 64, dtype=torch.int8), torch.zeros(1, 1, 64)
    for args, kw in (((k, v, s, s), {}),                              # host memory
                     ((k.float(), v, s, s), {}), ((k, v[:, :, :32], s, s), {}), ((k, v, s[..., :32], s), {}),
                     ((k, v, s.half(), s), {}), ((k, v, s, s), dict(dtype=torch.float32))):
        with pytest.raises(P.MoEError):
            P.QuantPagedCache(*args, i32.view(1, 2), i32[:1], **kw)
    out = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(P.MoEError):
        P.moe_draft_verify(torch.zeros(2, 10), i32, i32, 1, out[:1].view(1, 1), out[1:2], out[2:], torch.zeros(100))
    with pytest.raises(P.MoEError):
        P.moe_qcache_read(None, None, None, None, 1, None, None)
