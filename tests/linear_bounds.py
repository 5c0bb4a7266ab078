"""How far moe_quant_linear's fp32 sums may be from the exact ones when their roundings are
independent, as a root mean square over the outputs.

Codes enter as 16 + q, and each group's partial sum P loses (16 + z) X, X the group's sum of
activations, before its scale is applied.  A sum of n terms in any order rounds at most n
times, each time by at most 2^-24 of a partial sum, whose own mean square is at most that
of the whole sum's terms added up.  The joined groups round three times each (zero point,
scale, addition), by 2^-24 of what is there.
"""
import torch

E32 = 2.0 ** -24


def rms(v):
    return v.double().square().mean().sqrt().item()


def rms_bound(x, q, z, s, group):
    """x [T][K], codes q [R][K], zeros z and scales s [R][K / group], in 64 bits.  Twice the
    root mean square of the roundings' sum over all outputs."""
    total, done = 0.0, 0.0
    for g in range(q.shape[1] // group):
        c = slice(g * group, (g + 1) * group)
        xs, zg, sg = x[:, c].double(), z[:, g, None].double(), s[:, g, None].double()
        codes = 16 + q[:, c].double()
        terms = codes.square() @ xs.square().t()                    # [R][T]: mean square of P
        taken = (16 + zg).square() * xs.square().sum(1)             # of (16 + z) X
        total = total + sg.square() * E32 ** 2 * ((group + 1) * (terms + taken) + 2 * (terms + taken))
        done = done + sg.square() * ((q[:, c].double() - zg).square() @ xs.square().t())
        total = total + E32 ** 2 * done
    return 2 * total.mean().sqrt().item()
