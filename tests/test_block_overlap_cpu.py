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
