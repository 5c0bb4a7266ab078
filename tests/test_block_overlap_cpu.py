"""Outputs of the decoder block's entry points that lie over inputs are refused on the host,
before any device work, wherever a row's stores could change another's loads."""
import pytest

from test_block_cpu import ARG, FAKE, caller, lib  # noqa: F401

R, Y, G, W, H = (FAKE + (i << 20) for i in range(5))     # far apart


def test_norm_outputs_over_gate_and_weights(lib):  # noqa: F811
    call = caller(lib.moe_block_norm, dict(
        y=Y, yt=2, ldy=64, r=R, rt=0, ldr=64, T=4, d=64, wp=None, gate=None, gt=0, grs=0, gcs=0, a=1.0, b=1.0,
        w=None, eps=1e-6, ro=None, ldro=64, h=H, ht=0, ldh=64, stream=None))
    element, channel, token = dict(grs=64, gcs=1), dict(grs=0, gcs=1), dict(grs=1, gcs=0)
    for kw in (dict(wp=H), dict(w=H), dict(w=H + 508), dict(wp=H - 252),         # a byte of 4 rows of 128
               dict(gate=H, **channel), dict(gate=H + 510, **channel), dict(gate=H, **token), dict(gate=H - 6, **token),
               dict(gate=H + 2, **element), dict(gate=H - 128, **element), dict(gate=H, grs=72, gcs=1),
               dict(gate=H, gt=1, **element),                                     # in place over another type
               dict(ro=R, gate=R + 2, **element), dict(ro=G, gate=G, gt=2, **element), dict(ro=W, w=W), dict(ro=W, wp=W)):
        assert call(**kw) == ARG, kw


def cache_at(k, v):
    """A cache of 8 pages, 2 heads of 64, 32 slots: 64 KB each for keys and values."""
    from test_block_cpu import cache_desc
    return cache_desc(k=k, v=v)


K, V, Q = FAKE + (8 << 20), FAKE + (9 << 20), FAKE + (10 << 20)


def test_attention_output_over_queries_and_cache(lib):  # noqa: F811
    call = caller(lib.moe_tree_attention, dict(
        c=cache_at(K, V), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, N=6, mx=4, ml=64, q=Q, ldq=256, Hq=4, mask=None,
        mw=0, scale=0.125, out=Q + (1 << 20), ldo=256, st=None, ws=None, wsb=0, stream=None))
    for kw in (dict(out=Q + 2), dict(out=Q - 2), dict(out=Q + 512 * 5 + 510), dict(out=Q - 512 * 6 + 2),   # rows of 512 bytes
               dict(ldq=512, ldo=512, out=Q + 256), dict(ldq=512, ldo=512, out=Q - 510),    # between rows, but too near
               dict(ldq=512, out=Q + 512),                                   # strides that differ: rows meet further on
               dict(N=1, B=1, ldq=4096, out=Q + 510),
               dict(out=K), dict(out=K + 65534), dict(out=V - 512 * 6 + 2), dict(out=V + 100)):
        assert call(**kw) == ARG, kw


def test_append_output_over_inputs_and_cache(lib):  # noqa: F811
    call = caller(lib.moe_cache_append, dict(
        c=cache_at(K, V), table=FAKE, pages=4, lens=FAKE, B=2, off=FAKE, N=6, mx=4, q=Q, ldq=512, Hq=4, k=Q + 512, ldk=512,
        v=Q + 768, ldv=512, pos=None, cos=None, sin=None, rot=0, mp=0, il=0, qo=Q + (1 << 20), ldqo=256, st=None, stream=None))
    for kw in (dict(qo=Q + 2, ldqo=512), dict(qo=Q + 16), dict(qo=Q + 512, ldqo=512), dict(qo=Q + 766, ldqo=512),
               dict(qo=Q - 2, ldqo=512), dict(qo=K), dict(qo=V + 65534), dict(qo=V - 512 * 6 + 2)):
        assert call(**kw) == ARG, kw


def test_keep_lengths_over_inputs(lib):  # noqa: F811
    call = caller(lib.moe_cache_keep, dict(c=cache_at(K, V), table=Q, pages=4, lens=FAKE, B=3, off=G, keep=W, mk=4, n=H, lo=R + 512,
                                           st=None, stream=None))
    for kw in (dict(lo=FAKE + 8), dict(lo=FAKE - 8), dict(lo=G + 12), dict(lo=H + 4), dict(lo=W + 44), dict(lo=Q + 40),
               dict(lo=K), dict(lo=V + 65532)):
        assert call(**kw) == ARG, kw
