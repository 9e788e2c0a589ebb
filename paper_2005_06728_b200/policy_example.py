"""A small token policy trained by OD-SGD with several workers, all on one GPU.

    python -m paper_2005_06728_b200.policy_example [--steps N] [--workers M] [--vocab V] [--dim D]

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


def train(steps: int = 60, workers: int = 3, vocab: int = 61, dim: int = 32, batch: int = 16, seq: int = 24, lr: float = 1.0,
          warmup: int = 5, max_norm: float = 0.5, kl_coef: float = 0.002, reuse: int = 2, seed: int = 1) -> Report:
    dev = torch.device("cuda", torch.cuda.current_device())
    model = Model(vocab, dim)
    w0 = model.init(seed, dev)
    reference = model.views(w0.clone())
    ctx = binding.Odsgd(w0, torch.zeros_like(w0), n_workers=workers, lr=lr, local_lr=lr, momentum=0.5, wd=0.0,
                        w_b=torch.zeros_like(w0), local=[torch.zeros_like(w0) for _ in range(workers)],
                        tensor_offsets=[*model.offsets, model.numel])
    ctx.set_warmup(warmup)
    arenas = [torch.zeros_like(w0) for _ in range(workers)]
    bound = ctx.bind_grads(arenas)
    # a worker's gradients as its backward pass leaves them, and the set that clips and packs them all
    raw = [[torch.empty(shape, device=dev) for _, shape in model.shapes] for _ in range(workers)]
    clipper = lm.GradSet(raw, offsets=model.offsets, arenas=arenas)
    gen = torch.Generator(device=dev).manual_seed(seed + 1)
    lengths = torch.tensor([seq - i % (seq // 2) for i in range(batch)], device=dev)
    counts = torch.arange(seq, device=dev)[None, :] < lengths[:, None]
    weights = counts.float() / counts.sum()
    batches = [None] * workers
    rewards, losses, norms = [], [], []
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
                answers = torch.multinomial(torch.softmax(z, -1).view(-1, vocab), 1, generator=gen).view(batch, seq)
                reward = (answers == (3 * tokens + 1) % vocab).float() * counts
                mean = (reward * weights).sum()
                advantages = (reward - mean) * vocab ** 0.5
                acting = lm.token_logprob(z, answers).logp
                ref = lm.token_logprob(model.logits(reference, tokens)[2], answers).logp
                batches[m] = tokens, answers, acting, ref, advantages, mean
            loss = lm.policy_loss(z, answers, acting, advantages, weights, ref_logp=ref, kl_coef=kl_coef, dlogits=z)
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
    a = ap.parse_args(argv)
    r = train(steps=a.steps, workers=a.workers, vocab=a.vocab, dim=a.dim, lr=a.lr)
    every = max(1, a.steps // 20)
    for k in range(0, a.steps, every):
        print(f"step {k:4d}  reward {r.rewards[k]:.3f}  loss {r.losses[k]:+.4f}  norms {' '.join(f'{x:.3f}' for x in r.norms[k])}")
    print(f"mean reward of the last ten steps: {sum(r.rewards[-10:]) / len(r.rewards[-10:]):.3f} (chance: {1 / a.vocab:.3f})")


if __name__ == "__main__":
    main()
