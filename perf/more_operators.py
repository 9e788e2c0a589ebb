"""Measured cases of the language-model operators inside a worker's step: the gated feed-forward block with
its backward pass, dropout by a counter-based generator, and the verification of drafted tokens.

A worker's model between the token lookup and the loss (block, dropout on its way back into the residual
stream), and the worker acting: tokens drafted by an older copy of the weights, verified under the current ones.

`own = False` computes them in elementary torch operations in 32 bits (in 64 where a value next to a
border decides a token); `own = True` calls the package.  `exact` evaluates the definitions in 64 bits.
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
        # one sequence generating: a single token through the block, a read of both weights
        {"name": "gated-1-token", "op": "gated", "batch": 1, "seq": 1, "dim": 2048, "width": 5440, "type": "bf16", "weights": "same",
         "act": "silu", "save": False},
        # 48 sequences generating at once through a wide block
        {"name": "gated-48-tokens", "op": "gated", "batch": 48, "seq": 1, "dim": 4096, "width": 11000, "type": "bf16", "weights": "same",
         "act": "silu", "save": False},
        # a training batch of a small model of odd widths, half precision
        {"name": "gated-odd-f16", "op": "gated", "batch": 4, "seq": 509, "dim": 1001, "width": 2731, "type": "f16", "weights": "same",
         "act": "gelu", "save": True},
        # the largest forward pass: long sequences through a wide block, pre-activations kept for the backward pass
        {"name": "gated-8k-wide", "op": "gated", "batch": 8, "seq": 1024, "dim": 4096, "width": 11008, "type": "bf16", "weights": "same",
         "act": "silu", "save": True},
        # backward pass of a mid-size model whose weights are read from the fp32 arena
        {"name": "gatedgrad-4k-arena", "op": "gatedgrad", "batch": 8, "seq": 511, "dim": 2048, "width": 5440, "type": "bf16",
         "weights": "f32", "act": "silu"},
        # backward pass of the largest
        {"name": "gatedgrad-8k-wide", "op": "gatedgrad", "batch": 8, "seq": 1024, "dim": 4096, "width": 11008, "type": "bf16",
         "weights": "same", "act": "silu"},
        # a short full-precision batch, no residual stream: the form that a backward pass takes too
        {"name": "dropout-short-f32", "op": "dropout", "batch": 4, "seq": 255, "dim": 776, "type": "f32", "residual": "none", "p": 0.1},
        # a long batch back into its residual stream
        {"name": "dropout-32k-residual", "op": "dropout", "batch": 8, "seq": 4095, "dim": 4096, "type": "bf16", "residual": "bf16",
         "p": 0.1},
        # one sequence, four tokens drafted, wide vocabulary
        {"name": "verify-1-sequence", "op": "verify", "batch": 1, "drafts": 4, "vocab": 131072, "type": "bf16", "draft": True},
        # a few short answers of a small policy, drafted without a distribution (copied from earlier text)
        {"name": "verify-copied-f32", "op": "verify", "batch": 8, "drafts": 3, "vocab": 1000, "type": "f32", "draft": False},
        # a batch at a vocabulary of odd width
        {"name": "verify-16-odd", "op": "verify", "batch": 16, "drafts": 5, "vocab": 50021, "type": "bf16", "draft": True},
        # the largest: many sequences, seven tokens drafted, wide vocabulary
        {"name": "verify-48-wide", "op": "verify", "batch": 48, "drafts": 7, "vocab": 131072, "type": "bf16", "draft": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated", "gated", "gatedgrad", "dropout", "verify"])
    half = rng.choice(["bf16", "f16"])
    kind = rng.choice(["f32", "bf16", "f16"])
    batch, seq = rng.randint(1, 16), _log_int(rng, 1, 1024)
    if op in ("gated", "gatedgrad"):
        dim, width = _log_int(rng, 64, 4200), _log_int(rng, 100, 11100)
        if rng.random() < 0.5:  # widths as models have them; the others are odd as often as not
            dim, width = -(-dim // 64) * 64, -(-width // 64) * 64
        case = {"op": op, "batch": batch, "seq": seq, "dim": dim, "width": width, "type": half, "weights": rng.choice(["same", "same", "f32"]),
                "act": rng.choice(["silu", "gelu"])}
        most = 8192 * 4096 * 11008 // 3 // (dim * width * batch)  # a third of the largest listed case
        case["seq"] = max(1, min(seq, most))
        if op == "gated":
            case["save"] = rng.random() < 0.5
        return case
    if op == "dropout":
        return {"op": op, "batch": batch, "seq": 2 * seq, "dim": _log_int(rng, 17, 4100), "type": kind,
                "residual": rng.choice(["none", "f32", kind]), "p": rng.choice([0.05, 0.1, 0.5])}
    vocab, drafts = _log_int(rng, 100, 160000), rng.randint(1, 8)
    most = 30_000_000 // (vocab * (drafts + 1))
    return {"op": op, "batch": max(1, min(_log_int(rng, 1, 64), most)), "drafts": drafts, "vocab": vocab, "type": kind,
            "draft": rng.random() < 0.75}


# --------------------------------------------------------------------------- work

def work(case):
    op = case["op"]
    b, es = case["batch"], _BYTES[case["type"]]
    if op == "gated":
        n, d, f = b * case["seq"], case["dim"], case["width"]
        ws = es if case["weights"] == "same" else 4
        return {"bytes": n * d * es + 2 * d * f * ws + (3 if case["save"] else 1) * n * f * es, "flops": 4 * n * d * f}
    if op == "gatedgrad":
        n, d, f = b * case["seq"], case["dim"], case["width"]
        ws = es if case["weights"] == "same" else 4
        return {"bytes": 2 * n * d * es + 2 * d * f * (ws + es) + 3 * n * f * es, "flops": 8 * n * d * f}
    if op == "dropout":
        n = b * case["seq"] * case["dim"]
        out = case["residual"] if case["residual"] != "none" else case["type"]
        return {"bytes": n * (es + (2 * _BYTES[out] if case["residual"] != "none" else _BYTES[out])), "flops": 2 * n}
    k, v = case["drafts"], case["vocab"]
    rows = b * (k + 1 + (k if case["draft"] else 0))
    return {"bytes": rows * v * es + b * (k * 8 + (k + 1) * 16 + 4), "flops": 4 * rows * v}


# --------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _randn(g, *shape, scale=1.0, kind=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale).to(kind)


def _drafts(case, q, g):
    """Tokens drafted from logits q; some sequences drafted fewer, the rest of theirs is padding."""
    b, k, v = q.shape
    tok = torch.multinomial(torch.softmax(q.float() * 1.25, -1).view(b * k, v), 1, generator=g).view(b, k)
    many = torch.tensor([k - (i * 3) % (k + 1) if i % 4 == 3 else k for i in range(b)], device=DEV)
    return torch.where(torch.arange(k, device=DEV)[None, :] < many[:, None], tok, -1)


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    st = {"case": dict(case)}
    kind = _TYPES[case["type"]]
    if op in ("gated", "gatedgrad"):
        b, s, d, f = case["batch"], case["seq"], case["dim"], case["width"]
        wk = kind if case["weights"] == "same" else torch.float32
        st["x"] = _randn(g, b, s, d, kind=kind)
        st["w_gate"] = _randn(g, f, d, scale=d ** -0.5, kind=wk)
        st["w_up"] = _randn(g, f, d, scale=d ** -0.5, kind=wk)
        if op == "gatedgrad":
            st["gate"] = st["x"] @ st["w_gate"].to(kind).t()  # what the forward pass kept
            st["up"] = st["x"] @ st["w_up"].to(kind).t()
            st["dh"] = _randn(g, b, s, f, scale=1e-3 if case["type"] == "bf16" else 0.1, kind=kind)
        return st
    if op == "dropout":
        shape = case["batch"], case["seq"], case["dim"]
        st["x"] = _randn(g, *shape, kind=kind)
        st["residual"] = None if case["residual"] == "none" else _randn(g, *shape, scale=3.0, kind=_TYPES[case["residual"]])
        st["seed"], st["offset"] = int(seed) * 0x9E3779B97F4A7C15 % (1 << 63), 5 + int(seed) % 1000
        return st
    b, k, v = case["batch"], case["drafts"], case["vocab"]
    base = torch.randn(b, k + 1, v, generator=g, device=DEV) * 2.5
    st["target"] = base.to(kind)
    near = base[:, :k] + 0.6 * torch.randn(b, k, v, generator=g, device=DEV)  # the drafting policy: an older copy
    draft = near.to(kind)
    pad = v // 400  # trailing entries that pad the vocabulary to its width
    st["target"][..., v - pad:] = float("-inf")
    draft[..., v - pad:] = float("-inf")
    st["draft_tokens"] = _drafts(case, draft if case["draft"] else 3.0 * draft, g)  # copied text is mostly likely text
    st["draft"] = draft if case["draft"] else None
    st["uniforms"] = torch.rand(b, k + 1, generator=g, device=DEV)
    st["inv_temp"] = 1.25
    return st


# --------------------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


def _own_gated(st):
    from paper_2005_06728_b200 import lm

    r = lm.gated_ffn(st["x"], st["w_gate"], st["w_up"], activation=st["case"]["act"], save=st["case"]["save"])
    return {"h": r.h, "gate": r.gate, "up": r.up} if st["case"]["save"] else {"h": r.h}


def _own_gatedgrad(st):
    from paper_2005_06728_b200 import lm

    r = lm.gated_ffn_grad(st["x"], st["w_gate"], st["w_up"], st["gate"], st["up"], st["dh"], activation=st["case"]["act"])
    return {"dx": r.dx, "dw_gate": r.dw_gate, "dw_up": r.dw_up}


def _own_dropout(st):
    from paper_2005_06728_b200 import lm

    return lm.dropout(st["x"], st["case"]["p"], st["seed"], offset=st["offset"], residual=st["residual"])


def _own_verify(st):
    from paper_2005_06728_b200 import lm

    r = lm.verify_draft(st["target"], st["draft_tokens"], st["uniforms"], draft=st["draft"], inv_temp=st["inv_temp"])
    return {"accepted": r.accepted, "tokens": r.tokens, "logp": r.logp}


_OWN = {"gated": _own_gated, "gatedgrad": _own_gatedgrad, "dropout": _own_dropout, "verify": _own_verify}


def _weights_32(st, kind):
    """Weights take part in the activations' type: those of an fp32 arena are rounded to it."""
    return st["w_gate"].to(kind).float(), st["w_up"].to(kind).float()


def _plain_gated(st):
    kind = st["x"].dtype
    wg, wu = _weights_32(st, kind)
    x = st["x"].float()
    gate, up = x @ wg.t(), x @ wu.t()
    if st["case"]["act"] == "silu":
        a = gate / (1.0 + (-gate).exp())
    else:
        a = 0.5 * gate * (1.0 + (gate * math.sqrt(0.5)).erf())
    h = (a * up).to(kind)
    return {"h": h, "gate": gate.to(kind), "up": up.to(kind)} if st["case"]["save"] else {"h": h}


def _plain_gatedgrad(st):
    kind = st["x"].dtype
    wg, wu = _weights_32(st, kind)
    x, gate, up, dh = (st[k].float().flatten(0, 1) for k in ("x", "gate", "up", "dh"))
    if st["case"]["act"] == "silu":
        sig = 1.0 / (1.0 + (-gate).exp())
        a, da = gate * sig, sig * (1.0 + gate * (1.0 - sig))
    else:
        cdf = 0.5 * (1.0 + (gate * math.sqrt(0.5)).erf())
        a, da = gate * cdf, cdf + gate * (-0.5 * gate * gate).exp() / math.sqrt(2.0 * math.pi)
    dg, du = dh * up * da, dh * a
    dx = (dg @ wg + du @ wu).to(kind)
    return {"dx": dx.view(st["x"].shape), "dw_gate": (dg.t() @ x).to(kind), "dw_up": (du.t() @ x).to(kind)}


def _mul_32(a, m):
    """High and low word of a * m, for int64 tensors a of 32-bit values and a 32-bit number m."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)  # each below 2^48
    mid = (low >> 16) + high
    return mid >> 16, (low & 0xFFFF) | ((mid & 0xFFFF) << 16)


def _philox_step(c0, c1, c2, c3, k0, k1):
    h0, l0 = _mul_32(c0, 0xD2511F53)
    h1, l1 = _mul_32(c2, 0xCD9E8D57)
    return h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0


def _kept(n, seed, offset, threshold):
    """Which of n elements are kept: element e has 16 bits of word (e % 8) / 2 of Philox4x32-10 at counter
    (e / 8, offset) under key seed, low half first, and is kept where they are at least the threshold."""
    block = torch.arange(-(-n // 8), device=DEV)
    c0, c1 = block & 0xFFFFFFFF, block >> 32
    c2, c3 = torch.full_like(block, offset & 0xFFFFFFFF), torch.full_like(block, offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        c0, c1, c2, c3 = _philox_step(c0, c1, c2, c3, k0, k1)
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).view(-1)[:n] >= threshold


def _dropout_parts(st):
    threshold = round(st["case"]["p"] * 65536)
    x = st["x"]
    return _kept(x.numel(), st["seed"], st["offset"], threshold).view(x.shape), 65536.0 / (65536 - threshold)


def _plain_dropout(st):
    keep, scale = _dropout_parts(st)
    y = torch.where(keep, st["x"].float() * scale, torch.zeros((), device=DEV))
    if st["residual"] is None:
        return y.to(st["x"].dtype)
    return (y + st["residual"].float()).to(st["residual"].dtype)


def _plain_verify(st):
    b, n = st["uniforms"].shape
    k = n - 1
    z = st["target"].double() * st["inv_temp"]
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    s = e.sum(-1, keepdim=True)
    p = e / s
    tok, u = st["draft_tokens"], st["uniforms"].double()
    at = tok.clamp(min=0)[..., None]
    if st["draft"] is None:
        q = torch.zeros_like(p[:, :k]).scatter_(-1, at, 1.0)
    else:
        zq = st["draft"].double() * st["inv_temp"]
        q = (zq - zq.amax(-1, keepdim=True)).exp()
        q = q / q.sum(-1, keepdim=True)
    valid = tok >= 0
    ok = valid & (u[:, :k] * q.gather(-1, at)[..., 0] < p[:, :k].gather(-1, at)[..., 0])
    accepted = ok.long().cumprod(-1).sum(-1)
    # where a draft was refused: what the target has beyond the draft; behind the last draft: the target
    pos = torch.arange(n, device=DEV)[None, :]
    refused = torch.cat([valid, torch.zeros_like(valid[:, :1])], 1).gather(1, accepted[:, None])
    pn = p.gather(1, accepted[:, None, None].expand(b, 1, p.shape[-1]))[:, 0]
    qn = q.gather(1, accepted.clamp(max=k - 1)[:, None, None].expand(b, 1, p.shape[-1]))[:, 0]
    left = torch.where(refused, (pn - qn).clamp(min=0.0), pn)
    cum = left.cumsum(-1)
    drawn = (cum > u[:, k:] * cum[:, -1:]).long().argmax(-1)
    whole = torch.cat([tok, tok[:, :1]], 1)
    tokens = torch.where(pos < accepted[:, None], whole, torch.where(pos == accepted[:, None], drawn[:, None], -1))
    logp = z.gather(-1, tokens.clamp(min=0)[..., None])[..., 0] - (m + s.log())[..., 0]
    return {"accepted": accepted.int(), "tokens": tokens, "logp": torch.where(tokens >= 0, logp, torch.zeros_like(logp)).float()}


_PLAIN = {"gated": _plain_gated, "gatedgrad": _plain_gatedgrad, "dropout": _plain_dropout, "verify": _plain_verify}


# --------------------------------------------------------------------------- 64 bits

def _phi(x):
    return torch.special.ndtr(x)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("gated", "gatedgrad"):
        kind = st["x"].dtype
        rows = st["x"].reshape(-1, case["dim"]).double()
        wg, wu = (st[k].to(kind).double() for k in ("w_gate", "w_up"))
        silu = case["act"] == "silu"
        if op == "gated":
            gate, up = rows @ wg.T, rows @ wu.T
            shape = *st["x"].shape[:2], case["width"]
            h = (gate * torch.sigmoid(gate) if silu else gate * _phi(gate)) * up
            out = {"h": h, "gate": gate, "up": up} if case["save"] else {"h": h}
            return {k: v.view(shape) for k, v in out.items()}
        t, v, dh = (st[k].reshape(-1, case["width"]).double() for k in ("gate", "up", "dh"))
        if silu:
            s = torch.sigmoid(t)
            a, slope = t * s, s + t * s * torch.sigmoid(-t)
        else:
            a, slope = t * _phi(t), _phi(t) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)
        du = dh * a
        dg = dh * v * slope
        dx = torch.mm(dg, wg).add_(torch.mm(du, wu))
        return {"dx": dx.view(st["x"].shape), "dw_gate": torch.mm(dg.T, rows), "dw_up": torch.mm(du.T, rows)}
    if op == "dropout":
        keep, _ = _dropout_parts(st)
        chance = round(case["p"] * 65536) / 65536
        y = torch.zeros(st["x"].shape, dtype=torch.float64, device=DEV)
        y[keep] = st["x"][keep].double() / (1.0 - chance)
        return y if st["residual"] is None else y + st["residual"].double()
    logp = torch.zeros(st["uniforms"].shape, dtype=torch.float64, device=DEV)
    for i in range(case["batch"]):  # sequence by sequence, token by token
        k = case["drafts"]
        for j in range(k + 1):
            p = torch.log_softmax(st["target"][i, j].double() * st["inv_temp"], -1)
            y = int(st["draft_tokens"][i, j]) if j < k else -1
            u, last = float(st["uniforms"][i, j]), float(st["uniforms"][i, k])
            left = torch.exp(p)
            if y >= 0:
                if st["draft"] is None:
                    if u < float(left[y]):
                        logp[i, j] = p[y]
                        continue
                    left[y] = 0.0
                else:
                    q = torch.softmax(st["draft"][i, j].double() * st["inv_temp"], -1)
                    if u * float(q[y]) < float(left[y]):
                        logp[i, j] = p[y]
                        continue
                    left = torch.relu(left - q)
            mass = torch.cumsum(left, 0)
            logp[i, j] = p[int(torch.searchsorted(mass, last * mass[-1], right=True))]
            break
    return {"accepted": None, "tokens": None, "logp": logp}
