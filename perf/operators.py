"""Measured cases of the language-model operators around the OD-SGD update.

A worker's step on a language model: token embedding lookup, (the model), token scores or the
clipped policy loss with its gradient, (the model), the embedding's gradient, and the clipped
gradient laid out in the arena the server reads.  Each case is one of those calls.

`own = False` computes them in elementary torch operations in 32 bits; `own = True` calls the
package.  `exact` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False
DEV = "cuda"

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# --------------------------------------------------------------------------- cases

def listed():
    return [
        # a small network's gradients from four workers, every step of a cache-resident training run
        {"name": "clip-small-4w-f32", "op": "clip", "set": "lenet5", "workers": 4, "type": "f32", "over": 3.0},
        # one worker's 161 bf16 gradient tensors, as a mixed-precision backward pass leaves them
        {"name": "clip-161-tensors-bf16", "op": "clip", "set": "resnet50", "workers": 1, "type": "bf16", "over": 2.0},
        # eight workers' full-precision gradients clipped one by one before the server sums them
        {"name": "clip-8w-f32", "op": "clip", "set": "alexnet", "workers": 8, "type": "f32", "over": 1.5},
        # lookup of the few tokens a batch of generating sequences takes in one step
        {"name": "lookup-13-tokens", "op": "lookup", "batch": 13, "seq": 1, "vocab": 32000, "dim": 1000, "table": "f32",
         "type": "bf16"},
        # a long training batch from the fp32 weight arena into bf16 activations
        {"name": "lookup-32k-tokens", "op": "lookup", "batch": 8, "seq": 4095, "vocab": 50021, "dim": 4096, "table": "f32",
         "type": "bf16"},
        # the gradient of a short batch, full precision, a small model's width
        {"name": "embgrad-short-f32", "op": "embgrad", "batch": 4, "seq": 255, "vocab": 8000, "dim": 776, "type": "f32"},
        # the gradient of a long batch with natural token frequencies
        {"name": "embgrad-32k-bf16", "op": "embgrad", "batch": 8, "seq": 4095, "vocab": 50021, "dim": 2048, "type": "bf16"},
        # score of one token per generated step: one row, wide vocabulary
        {"name": "score-1-token", "op": "score", "batch": 1, "seq": 1, "vocab": 131072, "type": "bf16"},
        # scores of whole sequences by the reference policy; rows are a shifted view, vocabulary of odd width
        {"name": "score-8k-odd", "op": "score", "batch": 8, "seq": 1023, "vocab": 50021, "type": "bf16"},
        # a small policy in full precision
        {"name": "policy-small-f32", "op": "policy", "batch": 4, "seq": 47, "vocab": 1000, "type": "f32"},
        # a training batch of a mid-size policy
        {"name": "policy-4k-bf16", "op": "policy", "batch": 8, "seq": 511, "vocab": 32000, "type": "bf16"},
        # the largest: wide vocabulary, long sequences
        {"name": "policy-8k-wide", "op": "policy", "batch": 8, "seq": 1024, "vocab": 131072, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["clip", "lookup", "embgrad", "score", "policy"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op == "clip":
        # a transformer-like set of `layers` blocks of width `dim`, tied table of `vocab` rows
        return {"op": op, "set": "blocks", "layers": rng.randint(1, 12), "dim": _log_int(rng, 33, 1100),
                "vocab": _log_int(rng, 100, 20000), "workers": rng.randint(1, 6), "type": kind,
                "over": rng.choice([0.5, 1.5, 4.0])}
    batch, seq = rng.randint(1, 16), _log_int(rng, 1, 2048)
    if op == "lookup":
        return {"op": op, "batch": batch, "seq": seq, "vocab": _log_int(rng, 100, 140000), "dim": _log_int(rng, 17, 5000),
                "table": rng.choice(["f32", kind]), "type": kind}
    if op == "embgrad":
        return {"op": op, "batch": batch, "seq": seq, "vocab": _log_int(rng, 100, 100000), "dim": _log_int(rng, 17, 2600),
                "type": kind}
    vocab = _log_int(rng, 100, 200000)
    most = 500_000_000 // (vocab * _BYTES[kind])  # about a quarter of the largest listed case
    return {"op": op, "batch": batch, "seq": max(1, min(seq, most // batch)), "vocab": vocab, "type": kind}


# --------------------------------------------------------------------------- shapes

def _conv_bn(t, cout, cin, k):
    t += [cout * cin * k * k, cout, cout]


def _sizes(case):
    """Elements of each gradient tensor of one worker."""
    if case["set"] == "lenet5":
        return [500, 20, 25000, 50, 400000, 500, 5000, 10]
    if case["set"] == "alexnet":
        return [96 * 363, 96, 256 * 1200, 256, 384 * 2304, 384, 384 * 1728, 384, 256 * 1728, 256,
                4096 * 9216, 4096, 4096 * 4096, 4096, 1000 * 4096, 1000]
    t = []
    if case["set"] == "resnet50":
        _conv_bn(t, 64, 3, 7)
        cin = 64
        for blocks, width in ((3, 64), (4, 128), (6, 256), (3, 512)):
            for b in range(blocks):
                _conv_bn(t, width, cin, 1)
                _conv_bn(t, width, width, 3)
                _conv_bn(t, 4 * width, width, 1)
                if b == 0:
                    _conv_bn(t, 4 * width, cin, 1)
                cin = 4 * width
        return t + [1000 * 2048, 1000]
    d = case["dim"]
    t = [case["vocab"] * d]
    for _ in range(case["layers"]):
        t += [d, 3 * d * d, d * d, d, 4 * d * d, 4 * d, 4 * d * d, d]
    return t + [d]


def _offsets(sizes):
    """Arena offsets as the framework lays tensors out: each start on a 16-byte boundary."""
    off, at = [], 0
    for n in sizes:
        off.append(at)
        at = (at + n + 3) // 4 * 4
    return off, at


def _lengths(case):
    """Tokens of each sequence; the rest of its row is padding."""
    s = case["seq"]
    return [max(1, s - (b * 5) % (s // 4 + 1)) for b in range(case["batch"])]


def _prompts(case):
    """Tokens of each sequence that belong to its prompt and carry no loss (at least one does)."""
    return [min(n - 1, (b * 3 + 2) * n // 40) for b, n in enumerate(_lengths(case))]


def _active_rows(case):
    if case["op"] == "policy":
        return sum(n - p for n, p in zip(_lengths(case), _prompts(case)))
    return sum(_lengths(case))


def _masked_vocab(case):
    """Trailing vocabulary entries that pad the table to its width; their logits are -inf."""
    return case["vocab"] // 400


def _token_probs(vocab, device):
    """Natural token frequencies: rank r has weight 1 / (r + 2.7)."""
    p = 1.0 / (torch.arange(vocab, dtype=torch.float64, device=device) + 2.7)
    return p / p.sum()


def _unique_rows(case):
    n = sum(_lengths(case))
    p = _token_probs(case["vocab"], "cpu")
    return float((1.0 - torch.exp(n * torch.log1p(-p.clamp(max=1 - 1e-12)))).sum())


def work(case):
    op = case["op"]
    if op == "clip":
        n = sum(_sizes(case)) * case["workers"]
        return {"bytes": n * (_BYTES[case["type"]] + 4), "flops": 3 * n}
    n, valid = case["batch"] * case["seq"], sum(_lengths(case))
    es = _BYTES[case["type"]]
    if op == "lookup":
        d = case["dim"]
        return {"bytes": 8 * n + _unique_rows(case) * d * _BYTES[case["table"]] + n * d * es, "flops": valid * d}
    if op == "embgrad":
        d = case["dim"]
        return {"bytes": 8 * n + valid * d * es + case["vocab"] * d * 4, "flops": 2 * valid * d}
    rows, v = _active_rows(case), case["vocab"]
    if op == "score":
        return {"bytes": rows * v * es + 16 * n, "flops": 4 * rows * v}
    return {"bytes": rows * v * es + n * v * es + 28 * n + 16, "flops": 8 * rows * v}


# --------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 17)
    return g


def _length_mask(case):
    n = torch.tensor(_lengths(case), device=DEV)
    return torch.arange(case["seq"], device=DEV)[None, :] < n[:, None]


def _make_tokens(case, g):
    v = case["vocab"]
    cdf = torch.cumsum(_token_probs(v, DEV), 0)
    u = torch.rand(case["batch"], case["seq"], generator=g, device=DEV, dtype=torch.float64)
    rank = torch.searchsorted(cdf, u).clamp(max=v - 1)
    step = next(k for k in (7919, 7907, 7901) if math.gcd(k, v) == 1)
    return torch.where(_length_mask(case), (rank * step + 13) % v, -1)


def _make_logits(case, g):
    """Logits of `seq + 1` positions; the view without the last one scores the next token."""
    b, s, v = case["batch"], case["seq"], case["vocab"]
    whole = torch.empty(b, s + 1, v, dtype=_TYPES[case["type"]], device=DEV)
    for i in range(b):
        whole[i] = torch.randn(s + 1, v, generator=g, device=DEV) * 2.5
    whole[:, :, v - _masked_vocab(case):] = float("-inf")
    return whole[:, :-1]


def _log_prob_32(logits, labels, scale):
    """Log-probability of each label, sequence by sequence (only makes inputs)."""
    out = torch.empty(labels.shape, device=DEV)
    for i in range(labels.shape[0]):
        for a in range(0, labels.shape[1], 256):
            z = logits[i, a:a + 256].float() * scale
            y = labels[i, a:a + 256].clamp(min=0)
            out[i, a:a + 256] = z.gather(-1, y[:, None])[:, 0] - torch.logsumexp(z, -1)
    return out


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    st = {"case": dict(case)}
    if op == "clip":
        sizes, kind = _sizes(case), _TYPES[case["type"]]
        off, n = _offsets(sizes)
        groups = []
        for w in range(case["workers"]):
            sig = [10.0 ** (-3 + 2 * ((7 * i + w) % 11) / 10) for i in range(len(sizes))]
            groups.append([(torch.randn(k, generator=g, device=DEV) * s).to(kind) for k, s in zip(sizes, sig)])
        ends = off[1:] + [n]
        pads = [torch.zeros(e - o - k, device=DEV) for o, e, k in zip(off, ends, sizes)]
        # a bound that the norms pass by about `over` (below 1: nothing is clipped)
        exp2 = sum(k * 10.0 ** (2 * (-3 + 2 * ((7 * i) % 11) / 10)) for i, k in enumerate(sizes))
        st.update(groups=groups, offsets=off, pads=pads, max_norm=math.sqrt(exp2) / case["over"],
                  arenas=torch.zeros(case["workers"], n, device=DEV), norms=torch.zeros(case["workers"], device=DEV))
        return st
    if op in ("lookup", "embgrad"):
        st["tokens"] = _make_tokens(case, g)
        v, d = case["vocab"], case["dim"]
        st["scale"] = math.sqrt(d)
        if op == "lookup":
            st["table"] = (torch.randn(v, d, generator=g, device=DEV) * 0.02).to(_TYPES[case["table"]])
        else:
            st["dout"] = (torch.randn(case["batch"], case["seq"], d, generator=g, device=DEV) * 1e-3).to(_TYPES[case["type"]])
            st["dtable"] = torch.zeros(v, d, device=DEV)
        return st
    b, s, v = case["batch"], case["seq"], case["vocab"]
    st["inv_temp"] = 1.0 / 0.9
    st["logits"] = _make_logits(case, g)
    # labels: the likeliest of a few candidates, as a sampled token is
    cand = torch.randint(0, v - _masked_vocab(case), (b, s, 16), generator=g, device=DEV)
    pick = st["logits"].gather(-1, cand).argmax(-1, keepdim=True)
    st["labels"] = torch.where(_length_mask(case), cand.gather(-1, pick)[..., 0], -100)
    if op == "policy":
        logp = _log_prob_32(st["logits"], st["labels"], st["inv_temp"])
        st["old"] = logp + 0.15 * torch.randn(b, s, generator=g, device=DEV)
        st["ref"] = logp + 0.3 * torch.randn(b, s, generator=g, device=DEV)
        st["adv"] = torch.randn(b, 1, generator=g, device=DEV).expand(b, s)
        pos = torch.arange(s, device=DEV)[None, :]
        first = torch.tensor(_prompts(case), device=DEV)[:, None]
        live = (pos >= first) & _length_mask(case)
        st["weight"] = live.float() / _active_rows(case)
        # half-precision gradients of this size need a loss scale
        st.update(clip_low=0.2, clip_high=0.28, kl=0.05, grad_scale=4096.0 if case["type"] == "f16" else 1.0)
    return st


# --------------------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


def _own_clip(st):
    from paper_2005_06728_b200 import lm

    if "set" not in st:  # the checked table of gradient tensors, kept by a training loop like a bound gradient table
        st["set"] = lm.GradSet(st["groups"], offsets=st["offsets"], arenas=list(st["arenas"]))
    norms = st["set"].clip(st["max_norm"], out=st["norms"])
    return {"norms": norms, "arenas": st["arenas"]}


def _own_lookup(st):
    from paper_2005_06728_b200 import lm

    return lm.embed_lookup(st["tokens"], st["table"], scale=st["scale"], dtype=_TYPES[st["case"]["type"]])


def _own_embgrad(st):
    from paper_2005_06728_b200 import lm

    return lm.embed_grad(st["tokens"], st["dout"], st["dtable"], scale=st["scale"])


def _own_score(st):
    from paper_2005_06728_b200 import lm

    r = lm.token_logprob(st["logits"], st["labels"], inv_temp=st["inv_temp"])
    return {"logp": r.logp, "lse": r.lse}


def _own_policy(st):
    from paper_2005_06728_b200 import lm

    r = lm.policy_loss(st["logits"], st["labels"], st["old"], st["adv"], st["weight"], ref_logp=st["ref"],
                       clip_low=st["clip_low"], clip_high=st["clip_high"], kl_coef=st["kl"], inv_temp=st["inv_temp"],
                       grad_scale=st["grad_scale"])
    return {"stats": r.stats, "logp": r.logp, "dlogits": r.dlogits}


_OWN = {"clip": _own_clip, "lookup": _own_lookup, "embgrad": _own_embgrad, "score": _own_score, "policy": _own_policy}


def _plain_clip_one(tensors, pads, max_norm):
    flat = torch.cat([x.float() for pair in zip(tensors, pads) for x in pair])
    norm = flat.square().sum().sqrt()
    return norm, flat * torch.where(norm > max_norm, max_norm / norm, torch.ones_like(norm))


def _plain_clip(st):
    got = [_plain_clip_one(t, st["pads"], st["max_norm"]) for t in st["groups"]]
    return {"norms": torch.stack([n for n, _ in got]), "arenas": torch.stack([a for _, a in got])}


def _plain_lookup(st):
    tok = st["tokens"]
    rows = st["table"][tok.clamp(min=0)].float() * st["scale"]
    return torch.where((tok >= 0)[..., None], rows, torch.zeros((), device=DEV)).to(_TYPES[st["case"]["type"]])


def _plain_embgrad(st):
    tok = st["tokens"].reshape(-1)
    d = st["dout"].reshape(tok.numel(), -1).float()
    d = torch.where((tok >= 0)[:, None], d * st["scale"], torch.zeros((), device=DEV))
    return torch.zeros_like(st["dtable"]).index_add_(0, tok.clamp(min=0), d)


def _plain_softmax(st):
    z = st["logits"].float() * st["inv_temp"]
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    s = e.sum(-1, keepdim=True)
    y = st["labels"]
    lse = m + s.log()
    logp = z.gather(-1, y.clamp(min=0)[..., None]) - lse
    return e, s, logp[..., 0], lse[..., 0], y


def _plain_score(st):
    _, _, logp, lse, y = _plain_softmax(st)
    zero = torch.zeros_like(logp)
    return {"logp": torch.where(y >= 0, logp, zero), "lse": torch.where(y >= 0, lse, zero)}


def _plain_policy(st):
    e, s, logp, _, y = _plain_softmax(st)
    w, a = st["weight"], st["adv"]
    live = (w != 0) & (y >= 0)
    ratio = (logp - st["old"]).exp()
    bounded = ratio.clamp(1.0 - st["clip_low"], 1.0 + st["clip_high"])
    free = ratio * a <= bounded * a
    pg = -torch.where(free, ratio * a, bounded * a)
    d = st["ref"] - logp
    kl = d.exp() - d - 1.0
    zero = torch.zeros_like(logp)
    pg, kl = torch.where(live, w * pg, zero), torch.where(live, w * kl, zero)
    clipped = torch.where(live & ~free, w, zero)
    stats = torch.stack([pg.sum() + st["kl"] * kl.sum(), pg.sum(), kl.sum(), clipped.sum()])
    coef = w * (torch.where(free, -a * ratio, zero) + st["kl"] * (1.0 - d.exp())) * (st["inv_temp"] * st["grad_scale"])
    coef = torch.where(live, coef, zero)
    grad = e.mul_(-(coef[..., None] / s))
    grad.scatter_add_(-1, y.clamp(min=0)[..., None], coef[..., None])
    return {"stats": stats, "logp": torch.where(live, logp, zero), "dlogits": grad.to(_TYPES[st["case"]["type"]])}


_PLAIN = {"clip": _plain_clip, "lookup": _plain_lookup, "embgrad": _plain_embgrad, "score": _plain_score,
          "policy": _plain_policy}


# --------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        norms, arenas = [], []
        for tensors in st["groups"]:
            total = sum(float((t.double() ** 2).sum()) for t in tensors)
            norm = math.sqrt(total)
            factor = min(1.0, st["max_norm"] / norm) if norm > 0 else 1.0
            row = torch.zeros(st["arenas"].shape[1], dtype=torch.float64, device=DEV)
            for t, o in zip(tensors, st["offsets"]):
                row[o:o + t.numel()] = t.double() * factor
            norms.append(norm)
            arenas.append(row)
        return {"norms": torch.tensor(norms, dtype=torch.float64), "arenas": torch.stack(arenas)}
    if op == "lookup":
        tok = st["tokens"]
        out = torch.zeros(*tok.shape, case["dim"], dtype=torch.float64, device=DEV)
        ok = tok >= 0
        out[ok] = st["table"][tok[ok]].double() * st["scale"]
        return out
    if op == "embgrad":
        tok = st["tokens"].reshape(-1)
        keep = torch.nonzero(tok >= 0)[:, 0]
        out = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device=DEV)
        src = st["dout"].reshape(tok.numel(), -1)
        for a in range(0, keep.numel(), 8192):
            k = keep[a:a + 8192]
            out.index_add_(0, tok[k], src[k].double())
        return out * st["scale"]
    b, s = case["batch"], case["seq"]
    c, y = st["inv_temp"], st["labels"]
    logp = torch.zeros(b, s, dtype=torch.float64, device=DEV)
    norm = torch.zeros(b, s, dtype=torch.float64, device=DEV)
    grad = torch.zeros(b, s, case["vocab"], dtype=torch.float64, device=DEV) if op == "policy" else None
    sums = torch.zeros(3, dtype=torch.float64, device=DEV)
    for i in range(b):
        for a in range(0, s, 128):
            rows = slice(a, min(s, a + 128))
            lab = y[i, rows]
            ok = lab >= 0
            if op == "policy":
                ok = ok & (st["weight"][i, rows] != 0)
            at = torch.nonzero(ok)[:, 0]
            if at.numel() == 0:
                continue
            z = st["logits"][i, rows][at].double() * c
            lse = torch.logsumexp(z, -1)
            lp = z[torch.arange(at.numel(), device=DEV), lab[at]] - lse
            logp[i, a + at] = lp
            norm[i, a + at] = lse
            if op != "policy":
                continue
            w, adv = st["weight"][i, rows][at].double(), st["adv"][i, rows][at].double()
            r = torch.exp(lp - st["old"][i, rows][at].double())
            rc = torch.clamp(r, 1.0 - st["clip_low"], 1.0 + st["clip_high"])
            gap = torch.exp(st["ref"][i, rows][at].double() - lp)
            kl = gap - torch.log(gap) - 1.0
            cut = r * adv > rc * adv
            sums += torch.stack([-(w * torch.minimum(r * adv, rc * adv)).sum(), (w * kl).sum(), w[cut].sum()])
            k = st["grad_scale"] * c * w * (torch.where(cut, 0.0, -adv * r) + st["kl"] * (1.0 - gap))
            p = torch.exp(z - lse[:, None])
            p[torch.arange(at.numel(), device=DEV), lab[at]] -= 1.0
            grad[i, a + at] = -k[:, None] * p
    if op == "score":
        return {"logp": logp, "lse": norm}
    stats = torch.stack([sums[0] + st["kl"] * sums[1], sums[0], sums[1], sums[2]])
    return {"stats": stats, "logp": logp, "dlogits": grad}
