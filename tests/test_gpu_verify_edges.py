"""Verification of drafted tokens where its arithmetic is at its ends: what 64 bits hardly hold, far masks, high and low temperatures.

Expected values are block_reference's 64-bit form on rows that were shifted by their maximum beforehand (in 64 bits, where the
difference of two elements is exact); logp is bounded as in test_gpu_block."""
import math

import pytest
import torch

import block_reference as R
from paper_2005_06728_b200 import lm
from test_gpu_block import drafted
from test_gpu_lm import BF16, DEV, F16, F32, gen, randn

pytestmark = pytest.mark.gpu
NEXT_TO_ONE = 1 - 2.0 ** -24


def shifted(z):
    z = z.double()
    top = z.amax(-1, keepdim=True)
    return z - top.masked_fill(top == float("-inf"), 0.0)


def check(target, tok, u, draft, c=1.0, e=None, exact=False):
    """Equal decisions, draws and scores, where nothing is nearer to a border than 64-bit sums are off: 1e-11, some 2^53 / 90000, is more
    than any sum of a row here added one by one, and far more than the tree sums of the kernel.  `exact`: some decisions are made on
    zeros, which are borders by themselves, without any rounding."""
    e = c if e is None else e
    r = lm.verify_draft(target, tok, u, draft=draft, inv_temp=c, draft_inv_temp=e)
    accepted, tokens, logp, near = R.verify(shifted(target), tok, u, None if draft is None else shifted(draft), c, e)
    assert exact or near > 1e-11, "on the border: choose another seed"
    assert torch.equal(r.accepted.cpu().long(), accepted)
    assert torch.equal(r.tokens.cpu().long(), tokens)
    # the difference to the maximum, its product with the temperature and the sum's logarithm: a few roundings of 2^-24 of logp, and
    # the error of the sum as in test_gpu_block
    R.within(r.logp.cpu(), logp, 2.0 ** -19 + logp.abs().nan_to_num() * 2.0 ** -21, "logp")
    return r


# --------------------------------------------------------------------------- next to nothing left

@pytest.mark.parametrize("vocab", [700, 20000, 70001])
def test_what_is_left_is_small_everywhere(vocab):
    """All of the target's mass is taken off, what is left are elements of 2^-909: no part of the vocabulary reaches 2^-900, their sum
    does."""
    z = torch.full((3, 2, vocab), -909 * math.log(2.0), device=DEV)
    z[..., 100] = 0.0
    q = torch.full((3, 1, vocab), float("-inf"), device=DEV)
    q[..., 100], q[..., 300] = 0.0, -100 * math.log(2.0)
    tok = torch.full((3, 1), 300, device=DEV)
    u = torch.tensor([[0.5, 0.37], [0.25, 0.9], [0.75, 0.0123]], device=DEV)
    r = check(z, tok, u, q)
    assert r.accepted.tolist() == [0, 0, 0]


@pytest.mark.parametrize("vocab", [40, 700, 5000, 70001])
@pytest.mark.parametrize("way", ["same", "permuted", "shifted"])
def test_differences_that_64_bits_hardly_hold(vocab, way):
    """Two rows that differ in a token of 1e-20 of their mass, and in the order of their elements or by a constant: what is drawn is a
    token all the same, not the refused one, with its score."""
    n = 48
    base = randn(n, 1, vocab, seed=600 + vocab, sigma=2.0)
    x = torch.randint(0, vocab, (n, 1), generator=gen(601), device=DEV)
    base.scatter_(2, x[..., None], base.amax(-1, keepdim=True) - 46.0)
    q = base.clone()
    if way == "permuted":
        half = vocab // 2
        q[..., half:] = q[..., half:][..., torch.randperm(vocab - half, generator=gen(602), device=DEV)]
    elif way == "shifted":
        q = (q + 0.1) - 0.1
    q.scatter_(2, x[..., None], base.gather(2, x[..., None]) + 1.0)
    u = torch.rand(n, 2, generator=gen(603), device=DEV)
    u[:, 0] = 0.9
    u[:n // 4, 1], u[n // 4:n // 2, 1] = 0.0, NEXT_TO_ONE
    z = torch.cat((base, base), 1)
    r = lm.verify_draft(z, x, u, draft=q)
    assert not bool(r.accepted.any())
    t = r.tokens[:, :1]
    assert bool(((t >= 0) & (t < vocab) & (t != x)).all()) and bool((r.tokens[:, 1] == -1).all())
    want = torch.log_softmax(base[:, 0].double(), -1).gather(1, t)[:, 0]
    R.within(r.logp[:, 0].cpu(), want.cpu(), (2.0 ** -19 + want.abs() * 2.0 ** -21).cpu(), "logp")


@pytest.mark.parametrize("vocab", [40, 700, 20000])
def test_probabilities_at_the_end_of_64_bits(vocab):
    """Drafts of e^-704 of a row's largest element are still compared by their probabilities."""
    z = torch.full((5, 2, vocab), -5.0, device=DEV)
    z[..., 7] = 0.0
    z[..., 11] = -704.0
    q = z[:, :1].clone()
    q[3:, :, 11] = -700.0
    tok = torch.full((5, 1), 11, device=DEV)
    u = torch.tensor([[0.5, 0.3], [0.0, 0.6], [NEXT_TO_ONE, 0.2], [0.01, 0.9], [0.03, 0.4]], device=DEV)
    r = check(z, tok, u, q, exact=True)  # (u = 0: a border by itself)
    assert r.accepted.tolist() == [1, 1, 1, 1, 0]


# --------------------------------------------------------------------------- masks

@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [40, 700, 20000])
def test_masked_drafts_are_refused(kind, vocab):
    """A draft that the target's mask leaves nothing is refused, whatever the mask's value, the random number and the draft's own mask and
    temperature."""
    for mask in (float("-inf"), torch.finfo(kind).min, -6e4):
        target, tok, u, draft = drafted(8, 2, vocab, kind, 610)
        target[..., ::3] = mask
        draft[:4, ..., ::3] = mask
        tok = tok // 3 * 3
        u[::2, 0] = 0.0
        for q, c, e in ((draft, 1.0, 1.0), (draft, 0.5, 1.0), (draft, 1.0, 0.25), (None, 1.0, 1.0)):
            r = check(target, tok, u, q, c, e, exact=True)
            assert not bool(r.accepted.any()) and bool((r.tokens[:, 0] % 3 != 0).all())


@pytest.mark.parametrize("kind,mask,c", [(F32, -1e9, 2.0), (F32, -1e9, 1.5), (F32, -1e9, 2.97), (BF16, -1e9, 2.0), (F32, -2e9, 1.0), (F32, -1.5e9, 1.0),
                                         (BF16, -2.5e9, 1.0), (F32, -1e4, 2e5), (F16, -6e4, 4e4), (F32, -1e9, 1.0), (F32, -3.5e9, 1.0), (BF16, -1e12, 1.0)])
@pytest.mark.parametrize("vocab", [40, 700, 20000])
def test_masks_far_below(kind, mask, c, vocab):
    """Masks whose exponent is about 2^31 to 2^32: nothing of them counts, drafts of masked tokens are refused, and none is drawn."""
    target, tok, u, draft = drafted(12, 2, vocab, kind, 620, sigma=2.5 / max(c, 1.0), int_kind=torch.int64)
    keep = torch.arange(vocab, device=DEV) % 7 == 3
    target, draft = target.masked_fill(~keep, mask), draft.masked_fill(~keep, mask)
    tok = tok // 7 * 7 + 3
    tok[tok >= vocab] = 3
    tok[::4] -= 1  # a masked token
    for q in (draft, None):
        r = check(target, tok, u, q, c)
        drawn = r.tokens.gather(1, r.accepted.long()[:, None])
        assert bool((drawn % 7 == 3).all())
