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


# --------------------------------------------------------------------------- dropout

def philox(block, offset, seed):
    """Four 32-bit words of Philox4x32-10, by Python integers."""
    c = [block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(shape, p, seed, offset):
    t, n = round(p * 65536), math.prod(shape)
    bits = []
    for block in range(-(-n // 8)):
        for word in philox(block, offset, seed):
            bits += [word & 0xFFFF, word >> 16]
    return torch.tensor([b >= t for b in bits[:n]], dtype=torch.bool).view(shape)


def dropout(x, p, seed, offset, residual, kind):
    """Value and bound: the factor, the product, the addition and the result are rounded once each."""
    t = round(p * 65536)
    keep = kept(tuple(x.shape), p, seed, offset).to(x.device)
    y = torch.where(keep, x.double() * (65536 / (65536 - t)), torch.zeros((), dtype=torch.float64, device=x.device))
    r = torch.zeros_like(y) if residual is None else residual.double()
    return y + r, rounded(y + r, (3 * y.abs() + r.abs()) * U * 1.01, kind)


# --------------------------------------------------------------------------- drafted tokens

def verify(target, tokens, uniforms, draft, inv_temp, draft_inv_temp):
    """Sequence by sequence, in 64 bits: accepted, tokens, logp, and how near any decision was to its border."""
    c, e = (float(torch.tensor(v, dtype=torch.float32)) for v in (inv_temp, draft_inv_temp))
    z, u, tok = target.cpu().double() * c, uniforms.cpu().double(), tokens.cpu().long()
    zq = None if draft is None else draft.cpu().double() * e
    b, many, v = z.shape
    accepted, out, logp = torch.zeros(b, dtype=torch.int64), torch.full((b, many), -1), torch.zeros(b, many, dtype=torch.float64)
    near = 1.0
    for s in range(b):
        for i in range(many):
            p = torch.softmax(z[s, i], -1)
            x = int(tok[s, i]) if i < many - 1 else -1
            left = p
            if 0 <= x < v:
                q = torch.zeros(v, dtype=torch.float64) if zq is None else torch.softmax(zq[s, i], -1)
                if zq is None:
                    q[x] = 1.0
                if q[x] > 0 or p[x] > 0:  # (0 < 0 is no matter of rounding)
                    near = min(near, abs(float(u[s, i] * q[x] - p[x])) / max(float(p[x]), 1e-300))
                if u[s, i] * q[x] < p[x]:
                    out[s, i], logp[s, i] = x, torch.log_softmax(z[s, i], -1)[x]
                    continue
                left = (p - q).clamp(min=0)
                if not bool(left.sum() != 0):
                    left = p
            accepted[s] = i
            total = left.cumsum(0)
            if not bool(total[-1] > 0):
                logp[s, i] = float("nan")
                break
            bound = u[s, many - 1] * total[-1]
            j = int(((total > bound) & (left > 0)).long().argmax())
            near = min(near, float((total - bound).abs().min() / total[-1]))
            out[s, i], logp[s, i] = j, torch.log_softmax(z[s, i], -1)[j]
            break
    return accepted, out, logp, near
