"""Plain 64-bit forms of the operators inside a worker's step (gated feed-forward block, dropout, verification of
drafted tokens), on the device of their inputs, and the error bounds that their tests allow.  Written from the
definitions; shares no code with the package.

u = 2^-24 is the unit roundoff of binary32, unit(T) that of the stored type.
"""
import math

import torch

from lm_reference import TINY, U, UNIT


def product(a, b, at):
    """a b^T and what 32-bit sums of it may be off by: products of 16-bit elements are exact in 32 bits; each addition is off by
    at most a step (2 u, whatever the rounding) of what has been added so far, itself at most the sum of magnitudes."""
    a, b = a.double(), b.double()
    return a @ b.T, at * 2 * U * 1.01 * (a.abs() @ b.abs().T)


def activation(t, name):
    """Value, slope, and bounds of both in 32 bits.  The exponential is off by 2^-21 + |t| 2^-23 relative, a few
    roundings follow; the error function is off by 2^-22, multiplied by |t| / 2."""
    if name == "silu":
        s, r = torch.sigmoid(t), torch.sigmoid(-t)
        value, slope = t * s, s + t * s * r
        rel = (t.abs() + 16) * 2.0 ** -22
        return value, slope, rel * value.abs() + 2.0 ** -126, rel * s * (1 + t.abs())
    cdf = torch.special.ndtr(t)
    bell = torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)
    rel = 2.0 ** -20 * (1 + t * t * 0.125)
    return t * cdf, cdf + t * bell, t.abs() * 2.0 ** -21 + 2.0 ** -126, 2.0 ** -21 + rel * (t * bell).abs()


def rounded(ref, off, kind):
    """A value with error `off` rounded to `kind`."""
    return off + (ref.abs() + off) * UNIT[kind] * 1.01 + TINY[kind]


def gated(x, w_gate, w_up, name):
    """{output: (value, bound)} of the forward pass."""
    kind = x.dtype
    x, wg, wu = x.reshape(-1, x.shape[-1]), w_gate.to(kind), w_up.to(kind)
    gate, off_g = product(x, wg, x.shape[-1])
    up, off_u = product(x, wu, x.shape[-1])
    value, _, off_a, _ = activation(gate, name)
    off_a = off_a + 1.13 * off_g  # the slope of both activations is below 1.13
    h = value * up
    off_h = off_a * (up.abs() + off_u) + value.abs() * off_u + h.abs() * U
    return {"h": (h, rounded(h, off_h, kind)), "gate": (gate, rounded(gate, off_g, kind)), "up": (up, rounded(up, off_u, kind))}


def gated_grad(x, w_gate, w_up, gate, up, dh, name, dw_kind=None, old=None):
    """{output: (value, bound)} of the backward pass; `old`: what dw_gate and dw_up are added to."""
    kind = x.dtype
    dw_kind = kind if dw_kind is None else dw_kind
    x, wg, wu = x.reshape(-1, x.shape[-1]).double(), w_gate.to(kind).double(), w_up.to(kind).double()
    t, v, d = (q.reshape(-1, q.shape[-1]).double() for q in (gate, up, dh))
    value, slope, off_v, off_s = activation(t, name)
    dg, du = d * v * slope, d * value
    off_dg = rounded(dg, (d * v).abs() * off_s + dg.abs() * 3 * U, kind)
    off_du = rounded(du, d.abs() * off_v + du.abs() * 2 * U, kind)
    big_g, big_u = dg.abs() + off_dg, du.abs() + off_du
    n, f = dg.shape
    out = {}
    dx = dg @ wg + du @ wu
    off = off_dg @ wg.abs() + off_du @ wu.abs() + 2 * f * 2 * U * 1.01 * (big_g @ wg.abs() + big_u @ wu.abs())
    out["dx"] = dx, rounded(dx, off, kind)
    for key, part, off_part, big, before in (("dw_gate", dg, off_dg, big_g, 0), ("dw_up", du, off_du, big_u, 1)):
        dw = part.T @ x
        off = off_part.T @ x.abs() + n * 2 * U * 1.01 * (big.T @ x.abs())
        if old is not None:
            dw = dw + old[before].double()
        out[key] = dw, rounded(dw, off, dw_kind)
    return out


def within(got, ref, bound, what):
    got = got.reshape(ref.shape).double()
    same = (got == ref) | (got.isnan() & ref.isnan())
    bad = ~(same | ((got - ref).abs() <= bound))
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, worst "
                                 f"{float(((got - ref).abs() / bound)[bad].max()):.3g} times")
