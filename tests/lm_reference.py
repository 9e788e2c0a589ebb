"""Plain 64-bit forms of the language-model operators, on the CPU, and the error bounds that their
tests allow.  Written from the definitions; shares no code with the package.

u = 2^-24 is the unit roundoff of binary32, unit(T) that of the stored type.
"""
import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half the distance of two subnormals: what a rounding can lose near zero
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def host(t):
    return t.detach().cpu().double()


def lookup(tokens, table, scale):
    tok, tab = tokens.cpu().long(), host(table)
    ok = (tok >= 0) & (tok < tab.shape[0])
    out = tab[tok.clamp(0, tab.shape[0] - 1)] * scale
    return torch.where(ok[..., None], out, torch.zeros((), dtype=torch.float64))


def lookup_bound(ref, dtype):
    """One rounding of the product and one to the stored type."""
    return ref.abs() * (U + UNIT[dtype]) * 1.01 + TINY[dtype]


def embed_grad(tokens, grad, vocab, scale, padding=None, old=None):
    """The gradient, and its bound: a sum of n terms in any order is off by at most (n - 1) u times
    the sum of magnitudes; the scale and the addition to an old value round once each."""
    tok = tokens.cpu().long().reshape(-1)
    g = host(grad).reshape(tok.numel(), grad.shape[-1])
    ok = (tok >= 0) & (tok < vocab)
    if padding is not None:
        ok &= tok != padding
    out = torch.zeros(vocab, g.shape[1], dtype=torch.float64)
    mag, cnt = torch.zeros_like(out), torch.zeros(vocab, dtype=torch.float64)
    out.index_add_(0, tok[ok], g[ok])
    mag.index_add_(0, tok[ok], g[ok].abs())
    cnt.index_add_(0, tok[ok], torch.ones(int(ok.sum()), dtype=torch.float64))
    out, mag = out * scale, mag * abs(scale)
    if old is not None:
        hit = (cnt > 0)[:, None]
        mag = mag + torch.where(hit, host(old).abs(), torch.zeros_like(mag))
        out = out + host(old)
    return out, (cnt[:, None] + 2) * U * 1.01 * mag + TINY[torch.float32]


def scores(logits, labels, c):
    z, y = host(logits) * c, labels.cpu().long()
    ok = (y >= 0) & (y < z.shape[-1])
    lse = torch.logsumexp(z, -1)
    logp = z.gather(-1, y.clamp(0, z.shape[-1] - 1)[..., None])[..., 0] - lse
    zero = torch.zeros_like(lse)
    return torch.where(ok, logp, zero), torch.where(ok, lse, zero), ok


def score_bound(logits, c, logp):
    """Absolute error allowed in logp and lse.

    exp: 2^-22 relative from the function, and u times the sizes of the numbers its argument is
    made of (c z, c m, their difference), each at most 4 times the largest finite |c z|; the sum
    over the row goes through fewer than 64 additions one after another (64 in a thread, then
    trees) in the smaller cases and rounds of them joined in the larger ones; log and the last
    two subtractions round the result and |c z| once each.
    """
    z = host(logits)
    top = torch.where(torch.isfinite(z), z.abs(), torch.zeros_like(z)).amax(-1) * c
    return 2.0 ** -22 + U * (128 + 8 * top + 4 * torch.nan_to_num(logp).abs())


def policy(logits, labels, old, adv, w, ref=None, lo=0.2, hi=0.2, beta=0.0, c=1.0, gs=1.0):
    """dict of the results and their bounds (for ratios that are not within 1e-3 of a clip bound)."""
    logp, _, ok = scores(logits, labels, c)
    old, adv, w = host(old), host(adv), host(w)
    live = ok & (w != 0)
    zero = torch.zeros_like(logp)
    e = score_bound(logits, c, logp)
    r = torch.exp(logp - old)
    rc = r.clamp(1 - lo, 1 + hi)
    cut = r * adv > rc * adv
    pg = -torch.minimum(r * adv, rc * adv)
    d = host(ref) - logp if ref is not None else zero
    kl = torch.expm1(d) - d
    g = torch.where(cut, zero, -adv * r) - beta * torch.expm1(d)
    k = w * g * c * gs
    z = host(logits) * c
    p = torch.softmax(z, -1)
    hot = torch.zeros_like(p).scatter_(-1, labels.cpu().long().clamp(0, p.shape[-1] - 1)[..., None], 1.0)
    dz = torch.where(live[..., None], k[..., None] * (hot - p), torch.zeros_like(p))
    zl = lambda x: torch.where(live, x, zero)  # noqa: E731
    pg, kl, cl = zl(w * pg), zl(w * kl), zl(torch.where(cut, w, zero))
    stats = torch.stack([pg.sum() + beta * kl.sum(), pg.sum(), kl.sum(), cl.sum()])
    # bounds: r and exp(d) carry the error of logp, and eight roundings in all
    big_pg = w.abs() * adv.abs() * r * (e + 8 * U)
    big_kl = w.abs() * (torch.exp(d) + 1 + d.abs()) * (e + 8 * U)
    ek = (w.abs() * (adv.abs() * r + abs(beta) * (torch.exp(d) + 1))) * (e + 8 * U) * c * abs(gs)
    t = logits.dtype
    ez = (k.abs() * (e + 8 * U))[..., None] * p + ek[..., None] * (hot - p).abs() + dz.abs() * UNIT[t] * 1.01 + 2 * U * k.abs()[..., None] * (hot + p) + TINY[t]
    s_pg, s_kl = zl(big_pg).sum(), zl(big_kl).sum()
    es = torch.stack([s_pg + abs(beta) * s_kl, s_pg, s_kl, zl(w.abs()).sum() * U]) + 2 * U * stats.abs()
    return {"logp": zl(logp), "dlogits": dz, "stats": stats, "live": live,
            "e_logp": e, "e_dlogits": torch.where(live[..., None], ez, torch.zeros_like(ez)), "e_stats": es}


def clip(tensors, max_norm):
    """Norm of the list and the scaled tensors, in 64 bits."""
    total = sum(float((host(t) ** 2).sum()) for t in tensors)
    norm = total ** 0.5
    k = max_norm / norm if norm > max_norm else 1.0
    return norm, k, [host(t) * k for t in tensors]


def clip_bound(ref, dtype):
    """The factor is rounded once, the product once, and once more to the stored type."""
    return ref.abs() * (3 * U + UNIT[dtype]) * 1.01 + TINY[dtype] + TINY[torch.float32]


def within(got, ref, bound, what=""):
    got = host(got)
    both_nan = torch.isnan(got) & torch.isnan(ref)
    err = torch.where(both_nan, torch.zeros_like(ref), (got - ref).abs())
    same_inf = torch.isinf(ref) & (got == ref)
    bad = ~((err <= bound) | both_nan | same_inf)
    if bool(bad.any()):
        i = int(torch.nonzero(bad.reshape(-1))[0])
        b = torch.broadcast_to(torch.as_tensor(bound, dtype=torch.float64), ref.shape).reshape(-1)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside their bound; first at {i}: "
                             f"{float(got.reshape(-1)[i])!r}, expected {float(ref.reshape(-1)[i])!r} +- {float(b[i]):.3e}")
