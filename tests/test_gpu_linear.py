"""moe_quant_linear: single rows, and sums held to what independent roundings leave."""
import pytest
import torch

from linear_bounds import rms, rms_bound
from test_gpu_block import BF16, FP16, FP32, P, gen, linear_bound, packed, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("words", [32, 35, 40])
def test_one_row_of_any_length(T, words):
    """A matrix of one row has no row stride that could be out of line."""
    K = 256
    codes, sz, w, mag = packed(1, K, 64, 3, pad=16)
    x = torch.randn(T, K, device="cuda", generator=gen(T)).to(BF16)
    y = torch.empty(T, 1, device="cuda")
    P().moe_quant_linear(x, codes[:, :words], sz, y)
    want = x.double() @ w.t()
    within(y, want, linear_bound(x, mag, K, FP32, want), "one row")


def parts(codes, sz, K, group):
    """Codes [R][K], zeros and scales [R][K / group] of packed rows."""
    at = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device="cuda")
    q = (codes[:, :K // 8, None] >> at & 15).reshape(codes.shape[0], K)
    s, z = ((w.t().to(torch.int16).view(FP16)) for w in (sz & 0xFFFF, sz >> 16))
    return q, z, s


PATHS = [   # tokens, rows, channels, group: every kernel, its row and token tiles, long and short K
    (1, 130, 14336, 128), (1, 8200, 2048, 64), (2, 130, 11008, 64), (2, 8200, 2048, 128), (3, 130, 14336, 128),
    (16, 130, 4096, 128), (20, 130, 11008, 64), (33, 130, 14336, 64), (48, 200, 4096, 128), (64, 130, 14336, 128),
    (70, 130, 4096, 64), (12, 8200, 2048, 64), (40, 8200, 2048, 128), (64, 8200, 2048, 64), (40, 20500, 1024, 64),
    (64, 20500, 1024, 128)]


@pytest.mark.parametrize("xt", [BF16, FP16])
@pytest.mark.parametrize("T,R,K,group", PATHS)
def test_fp32_sums_as_near_as_independent_roundings(T, R, K, group, xt):
    codes, sz, w, _ = packed(R, K, group, T + R)
    x = torch.randn(T, K, device="cuda", generator=gen(5))
    x[:, ::97] *= 20
    x = x.to(xt)
    y = torch.empty(T, R, device="cuda")
    P().moe_quant_linear(x, codes, sz, y)
    off, most = rms(y.double() - x.double() @ w.t()), rms_bound(x, *parts(codes, sz, K, group), group)
    assert off <= most, "rms off by %.3g, bound %.3g" % (off, most)


@pytest.mark.parametrize("T,R,K,group", PATHS)
def test_first_and_last_channels_count(T, R, K, group):
    """Activations of eight channels alone, so that a channel left out or taken twice is an error
    of the result's own size."""
    codes, sz, w, mag = packed(R, K, group, T + R + 1)
    for first in (0, group - 8, K - group, K - 32, K - 8):
        x = torch.zeros(T, K, device="cuda", dtype=BF16)
        x[:, first:first + 8] = torch.randn(T, 8, device="cuda", generator=gen(first)).to(BF16)
        y = torch.empty(T, R, device="cuda")
        P().moe_quant_linear(x, codes, sz, y)
        want = x.double() @ w.t()
        within(y, want, linear_bound(x, mag, K, FP32, want), "channels from %d" % first)
