"""A small token policy trained by OD-SGD with several workers, all on one GPU.

    python -m paper_2005_06728_b200.policy_example [--steps N] [--workers M] [--vocab V] [--dim D]
                                                   [--block F] [--drop P] [--drafts K]

Each worker acts with the weights that the state machine of Algorithm 2 lets it train on (global
weights in the warm-up, its own local weights afterwards): it reads tokens, samples an answer to each
and is rewarded for the right one, (3 token + 1) mod vocab.  It learns from a batch of answers for
`reuse` steps, while its weights move away from the ones it acted with; that is what the ratio in the
loss corrects for.  Its step around the model is made of the language-model calls of the library:

    embed_lookup    rows of the embedding in the worker's weight arena -> activations
    token_logprob   scores of the answers under the acting and the reference policy
    policy_loss     clipped loss with a KL term, gradient of the logits (written over them)
    embed_grad      gradient of the embedding, summed by sorted tokens
    GradSet.clip    all gradients of all workers clipped by their norm, into the gradient arenas

and `Odsgd.step_update` does the rest.  The two matrix products of the model, and their gradients, are
torch's.

With --block the model is a gated feed-forward block of that width on a residual stream, in bfloat16 from the float32 arena
(`gated_ffn`, `gated_ffn_grad`), what it adds dropped out with probability --drop (`dropout`, whose gradient is the
same call).  With --drafts a worker's answers are drafted by the reference policy, so many at a time, and verified under the
weights it acts with (`verify_draft`), which gives the scores that the loss takes as the acting policy's.  Answers do not depend on one
another here, so the acting policy's logits are known for all positions beforehand and no time is saved: the option shows the call in its
place (rounds of drafts, ragged sequences, scores into the loss), not what drafting is for.
"""
from __future__ import annotations

import argparse
import math
from typing import Dict, List, NamedTuple

import torch

from . import binding, lm


class Report(NamedTuple):
    rewards: List[float]      # mean reward of each step, over all workers
    losses: List[float]
    norms: List[List[float]]  # gradient norm of each worker, before clipping, in each step
    weights: torch.Tensor     # the global weights after the last step


class Model:
    """Views of a flat parameter arena: embedding, a square layer, output head."""

    def __init__(self, vocab: int, dim: int):
        self.vocab, self.dim = vocab, dim
        self.shapes = [("embedding", (vocab, dim)), ("layer", (dim, dim)), ("head", (vocab, dim))]
        self.offsets, at = [], 0
        for _, shape in self.shapes:
            self.offsets.append(at)
            at += -(-math.prod(shape) // 4) * 4
        self.numel = at

    def views(self, arena: torch.Tensor) -> Dict[str, torch.Tensor]:
        return {name: arena[o:o + math.prod(s)].view(s) for (name, s), o in zip(self.shapes, self.offsets)}

    def init(self, seed: int, device) -> torch.Tensor:
        arena = torch.zeros(self.numel, device=device)
        g = torch.Generator(device=device).manual_seed(seed)
        for name, view in self.views(arena).items():
            view.normal_(0.0, 1.0 / self.dim if name == "embedding" else 1.0 / math.sqrt(self.dim), generator=g)
        return arena

    def logits(self, w: Dict[str, torch.Tensor], tokens: torch.Tensor):
        x = lm.embed_lookup(tokens, w["embedding"], scale=math.sqrt(self.dim))
        h = torch.tanh(x @ w["layer"])
        return x, h, h @ w["head"].t()


class GatedModel(Model):
    """Views of a flat parameter arena: embedding, gated block, output head.  Activations and the gradients of matrix products
    are bfloat16; the arena stays float32."""

    def __init__(self, vocab: int, dim: int, width: int, drop: float = 0.0):
        self.vocab, self.dim, self.drop = vocab, dim, drop
        self.shapes = [("embedding", (vocab, dim)), ("gate", (width, dim)), ("up", (width, dim)), ("down", (dim, width)), ("head", (vocab, dim))]
        self.offsets, at = [], 0
        for _, shape in self.shapes:
            self.offsets.append(at)
            at += -(-math.prod(shape) // 4) * 4
        self.numel = at

    def gradients(self, device) -> List[torch.Tensor]:
        """What a backward pass writes: the embedding's and the block's gradients in float32, the products' in bfloat16."""
        half = ("down", "head")
        return [torch.empty(shape, device=device, dtype=torch.bfloat16 if name in half else torch.float32) for name, shape in self.shapes]

    def forward(self, w: Dict[str, torch.Tensor], tokens: torch.Tensor, seed: int = 0, offset: int = 0, training: bool = False):
        """Logits, and what the backward pass needs."""
        drop = self.drop if training else 0.0
        x = lm.embed_lookup(tokens, w["embedding"], scale=math.sqrt(self.dim), dtype=torch.bfloat16)
        block = lm.gated_ffn(x, w["gate"], w["up"], save=training)
        y = block.h @ w["down"].to(torch.bfloat16).t()
        s = lm.dropout(y, drop, seed, offset=offset, residual=x)
        return s @ w["head"].to(torch.bfloat16).t(), (x, block, s, seed, offset)

    def backward(self, w: Dict[str, torch.Tensor], tokens: torch.Tensor, kept, dz: torch.Tensor, out: List[torch.Tensor]) -> None:
        """Gradients of all tensors, into `out` as gradients() makes it."""
        x, block, s, seed, offset = kept
        dz = dz.view(-1, self.vocab)
        torch.mm(dz.t(), s.view(-1, self.dim), out=out[4])
        ds = (dz @ w["head"].to(torch.bfloat16)).view(x.shape)
        dy = lm.dropout(ds, self.drop, seed, offset=offset)
        torch.mm(dy.view(-1, self.dim).t(), block.h.view(-1, block.h.shape[-1]), out=out[3])
        dh = dy @ w["down"].to(torch.bfloat16)
        g = lm.gated_ffn_grad(x, w["gate"], w["up"], block.gate, block.up, dh, dw_gate=out[1], dw_up=out[2])
        lm.embed_grad(tokens, g.dx + ds, out[0], scale=math.sqrt(self.dim))

    def logits(self, w: Dict[str, torch.Tensor], tokens: torch.Tensor):
        z, kept = self.forward(w, tokens)
        return kept[0], kept[2], z


def drafted_answers(z: torch.Tensor, draft: torch.Tensor, counts: torch.Tensor, drafts: int, gen: torch.Generator):
    """Answers to all positions, drafted from the logits `draft` so many at a time and verified under `z`, and their
    log-probabilities under `z`.  Positions that do not count (a sequence's end) end its drafts."""
    batch, seq, vocab = z.shape
    answers = torch.zeros(batch, seq, dtype=torch.int64, device=z.device)
    acting = torch.zeros(batch, seq, device=z.device)
    at = torch.zeros(batch, 1, dtype=torch.int64, device=z.device)
    step = torch.arange(drafts + 1, device=z.device)[None, :]
    rows = torch.arange(batch, device=z.device)[:, None]
    for _ in range(seq):  # (each round settles one position of a sequence at least)
        place = (at + step).clamp(max=seq - 1)
        open_ = (at + step < seq) & counts.gather(1, place)
        target, near = z[rows, place], draft[rows, place[:, :-1]]
        probs = torch.softmax(near.float(), -1).view(-1, vocab)
        tokens = torch.multinomial(probs, 1, generator=gen).view(batch, drafts) if drafts else place[:, :0]
        u = torch.rand(batch, drafts + 1, generator=gen, device=z.device)
        r = lm.verify_draft(target, torch.where(open_[:, :-1], tokens, -1), u, draft=near)
        settled = open_ & (step <= r.accepted[:, None])
        rows_, cols = rows.expand_as(place)[settled], place[settled]
        answers[rows_, cols], acting[rows_, cols] = r.tokens[settled], r.logp[settled]
        at = at + r.accepted[:, None] + 1
        if not bool((at < counts.sum(1, keepdim=True)).any()):
            break
    return answers, acting


def train(steps: int = 60, workers: int = 3, vocab: int = 61, dim: int = 32, batch: int = 16, seq: int = 24, lr: float = 1.0,
          warmup: int = 5, max_norm: float = 0.5, kl_coef: float = 0.002, reuse: int = 2, seed: int = 1, block: int = 0, drop: float = 0.0,
          drafts: int = 0) -> Report:
    dev = torch.device("cuda", torch.cuda.current_device())
    if drop and not block:
        raise ValueError("drop: the model has dropout behind its gated block only")
    model = GatedModel(vocab, dim, block, drop) if block else Model(vocab, dim)
    w0 = model.init(seed, dev)
    reference = model.views(w0.clone())
    ctx = binding.Odsgd(w0, torch.zeros_like(w0), n_workers=workers, lr=lr, local_lr=lr, momentum=0.5, wd=0.0,
                        w_b=torch.zeros_like(w0), local=[torch.zeros_like(w0) for _ in range(workers)],
                        tensor_offsets=[*model.offsets, model.numel])
    ctx.set_warmup(warmup)
    arenas = [torch.zeros_like(w0) for _ in range(workers)]
    bound = ctx.bind_grads(arenas)
    # a worker's gradients as its backward pass leaves them, and the set that clips and packs them all
    raw = [model.gradients(dev) if block else [torch.empty(shape, device=dev) for _, shape in model.shapes] for _ in range(workers)]
    clipper = lm.GradSet(raw, offsets=model.offsets, arenas=arenas)
    gen = torch.Generator(device=dev).manual_seed(seed + 1)
    lengths = torch.tensor([seq - i % (seq // 2) for i in range(batch)], device=dev)
    counts = torch.arange(seq, device=dev)[None, :] < lengths[:, None]
    weights = counts.float() / counts.sum()
    batches = [None] * workers
    rewards, losses, norms = [], [], []
    stalled = lm.stalled_waits()
    for step in range(steps):
        reward_sum, loss_sum = torch.zeros((), device=dev), torch.zeros((), device=dev)
        for m in range(workers):
            w = model.views(ctx.train_weights(m))
            fresh = step % reuse == 0
            if fresh:
                tokens = torch.randint(0, vocab, (batch, seq), generator=gen, device=dev)
                tokens = torch.where(counts, tokens, -1)  # ragged sequences: padding
            else:
                tokens, answers, acting, ref, advantages, mean = batches[m]
            x, h, z = model.logits(w, tokens)
            if fresh:
                if drafts:
                    answers, acting = drafted_answers(z, model.logits(reference, tokens)[2], counts, drafts, gen)
                else:
                    answers = torch.multinomial(torch.softmax(z.float(), -1).view(-1, vocab), 1, generator=gen).view(batch, seq)
                reward = (answers == (3 * tokens + 1) % vocab).float() * counts
                mean = (reward * weights).sum()
                advantages = (reward - mean) * vocab ** 0.5
                if not drafts:
                    acting = lm.token_logprob(z, answers).logp
                ref = lm.token_logprob(model.logits(reference, tokens)[2], answers).logp
                batches[m] = tokens, answers, acting, ref, advantages, mean
            if block:
                z, kept = model.forward(w, tokens, seed, step * workers + m, training=True)
            loss = lm.policy_loss(z, answers, acting, advantages, weights, ref_logp=ref, kl_coef=kl_coef, dlogits=z)
            if block:
                model.backward(w, tokens, kept, loss.dlogits, raw[m])
            else:
                dz = loss.dlogits.view(-1, vocab)
                torch.mm(dz.t(), h.view(-1, dim), out=raw[m][2])
                dh = (dz @ w["head"]) * (1.0 - h.view(-1, dim) ** 2)
                torch.mm(x.view(-1, dim).t(), dh, out=raw[m][1])
                lm.embed_grad(tokens, (dh @ w["layer"].t()).view(batch, seq, dim), raw[m][0], scale=math.sqrt(dim))
            reward_sum += mean
            loss_sum += loss.loss
        norm = clipper.clip(max_norm)
        ctx.step_update(bound)
        rewards.append(float(reward_sum) / workers)
        losses.append(float(loss_sum) / workers)
        norms.append(norm.tolist())
    if lm.stalled_waits() != stalled:
        raise RuntimeError("a product of the gated block was cut short: the run is void")
    out = Report(rewards, losses, norms, ctx.weights().clone())
    clipper.close()
    bound.unbind()
    ctx.close()
    return out


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=3)
    ap.add_argument("--vocab", type=int, default=61)
    ap.add_argument("--dim", type=int, default=32)
    ap.add_argument("--lr", type=float, default=1.0)
    ap.add_argument("--block", type=int, default=0, help="width of a gated feed-forward block (0: a square layer)")
    ap.add_argument("--drop", type=float, default=0.0, help="dropout behind the block")
    ap.add_argument("--drafts", type=int, default=0, help="answers drafted by the reference policy at a time")
    a = ap.parse_args(argv)
    r = train(steps=a.steps, workers=a.workers, vocab=a.vocab, dim=a.dim, lr=a.lr, block=a.block, drop=a.drop, drafts=a.drafts)
    every = max(1, a.steps // 20)
    for k in range(0, a.steps, every):
        print(f"step {k:4d}  reward {r.rewards[k]:.3f}  loss {r.losses[k]:+.4f}  norms {' '.join(f'{x:.3f}' for x in r.norms[k])}")
    print(f"mean reward of the last ten steps: {sum(r.rewards[-10:]) / len(r.rewards[-10:]):.3f} (chance: {1 / a.vocab:.3f})")


if __name__ == "__main__":
    main()
