"""The bound that moe_quant_linear's sums are held to passes fp32 sums in several orders and
finds what a mistake leaves out, at the lengths where a worst-case bound no longer does."""
import numpy as np
import pytest
import torch

from linear_bounds import rms, rms_bound


def case(T, R, K, group, seed):
    r = np.random.default_rng(seed)
    q, z = r.integers(0, 16, (R, K)), r.integers(5, 11, (R, K // group))
    s = (0.004 * (1 + r.random((R, K // group)))).astype(np.float16)
    x = r.standard_normal((T, K)).astype(np.float32)
    x[:, ::97] *= 20
    x = torch.from_numpy(x).to(torch.bfloat16)
    return x, torch.from_numpy(q), torch.from_numpy(z), torch.from_numpy(s)


def product(x, q, z, s, group, dtype, lanes):
    """Sums of a group in `lanes` interleaved chains, joined one after the other."""
    y = torch.zeros(x.shape[0], q.shape[0], dtype=dtype)
    x = x.to(dtype)
    for g in range(q.shape[1] // group):
        p, sx = (torch.zeros(x.shape[0], q.shape[0], lanes, dtype=dtype) for _ in range(2))
        for k in range(0, group, lanes):
            c = slice(g * group + k, g * group + k + lanes)
            p += x[:, None, c] * (16 + q[:, c].to(dtype))
            sx += x[:, None, c]
        tp, tx = p[..., 0], sx[..., 0]
        for i in range(1, lanes):
            tp, tx = tp + p[..., i], tx + sx[..., i]
        y = y + s[:, g].to(dtype) * (tp - (16 + z[:, g].to(dtype)) * tx)
    return y


@pytest.mark.parametrize("T,R,K,group", [(4, 24, 14336, 128), (3, 24, 11008, 64), (2, 40, 4096, 128)])
def test_bound(T, R, K, group):
    x, q, z, s = case(T, R, K, group, K)
    exact = product(x, q, z, s, group, torch.float64, 4)
    bound = rms_bound(x, q, z, s, group)
    assert bound < 3e-5 * rms(exact)
    for lanes in (1, 4, 32):
        assert rms(product(x, q, z, s, group, torch.float32, lanes).double() - exact) <= bound
    # what mistakes would give: an input left out or taken twice, outputs in 16 bits, a group's zero point
    short = x.clone()
    short[:, -8:] = 0
    assert rms(product(short, q, z, s, group, torch.float64, 4) - exact) > bound
    for t in (torch.bfloat16, torch.float16):
        assert rms(exact.to(t).double() - exact) > bound
    other = z.clone()
    other[:, -1] = z[:, 0]
    assert rms(product(x, q, other, s, group, torch.float64, 4) - exact) > bound
