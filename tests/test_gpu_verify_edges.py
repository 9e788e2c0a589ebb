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
    """Equal decisions, draws and scores, where nothing is nearer to a border than 64-bit sums are off: 70001 elements, the most here, added
    one by one 7.8e-12 of the whole, the kernel's sums far less.  `exact`: some decisions are made on zeros, which are borders by
    themselves, without any rounding."""
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


# --------------------------------------------------------------------------- temperatures

@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [40, 700, 20000])
@pytest.mark.parametrize("c", [1e-30, 1e-3, 30.0, 1e3, 1e6, 1e8, 1e9, 1e10, 1e12, 1e30])
def test_temperatures(kind, vocab, c):
    """From flat rows to rows that are nothing but their largest elements, the target's, the draft's or both; drafts are the most likely
    tokens of either row, or any."""
    target, tok, u, draft = drafted(24, 3, vocab, kind, 630 + vocab)
    target[::5, :, ::3] = float("-inf")
    top, near = target[:, :3].argmax(-1), draft.argmax(-1)
    pick = torch.randint(0, 4, tok.shape, generator=gen(631), device=DEV)
    tok = torch.where(pick == 0, tok, torch.where(pick == 1, top, near))
    for q, e in ((draft, c), (draft, 1.0), (None, c)):
        check(target, tok, u, q, c, e)
    check(target, tok, u, draft, 1.0, c)
    if c >= 1e6:  # one element is all of the row (or a few equal ones): whatever the random number
        u = u.clone()
        u[:12, 3], u[12:, 3] = 0.0, NEXT_TO_ONE
        r = lm.verify_draft(target, tok, u, draft=draft, inv_temp=c)
        t = r.tokens.gather(1, r.accepted.long()[:, None])
        row = target.gather(1, r.accepted.long()[:, None, None].expand(-1, -1, vocab))[:, 0]
        assert torch.equal(row.gather(1, t)[:, 0], row.amax(-1))
        score = r.logp.gather(1, r.accepted.long()[:, None])[:, 0]
        many = (row == row.amax(-1, keepdim=True)).sum(-1)
        assert float((score + many.double().log()).abs().max()) <= 2.0 ** -23 * math.log(vocab) + 2.0 ** -30


@pytest.mark.parametrize("offset,c", [(1e9, 1.0), (-1e9, 0.01), (1e9, 0.001), (1e12, 1e-5), (1e9, 1e9), (-3e38, 1e-30)])
@pytest.mark.parametrize("vocab", [40, 700, 20000])
def test_rows_far_from_zero(offset, c, vocab):
    """32-bit logits whose size is far above their differences."""
    step = float(torch.tensor(abs(offset)) - torch.nextafter(torch.tensor(abs(offset)), torch.tensor(0.0)))
    whole = lambda *s, seed: (randn(*s, seed=seed, sigma=4.0).round().double() * step + offset).to(F32)  # noqa: E731
    target, draft = whole(12, 3, vocab, seed=640), whole(12, 2, vocab, seed=641)
    target[::3, :, ::4] = float("-inf")
    tok = torch.randint(0, vocab, (12, 2), generator=gen(642), device=DEV)
    tok[::2] = draft.argmax(-1)[::2]
    u = torch.rand(12, 3, generator=gen(643), device=DEV)
    for q in (draft, None):
        check(target, tok, u, q, c)


def test_the_lowest_value_beside_infinities():
    """The type's lowest value is an element like others where it is the largest."""
    for kind in (F32, BF16, F16):
        for v in (40, 700, 20000):
            z = torch.full((3, 1, v), float("-inf"), dtype=kind, device=DEV)
            z[..., v // 2], z[..., v - 1] = torch.finfo(kind).min, torch.finfo(kind).min
            u = torch.tensor([[0.0], [0.49], [0.51]], device=DEV)
            r = lm.verify_draft(z, torch.zeros(3, 0, dtype=torch.int64, device=DEV), u)
            assert r.tokens.tolist() == [[v // 2], [v // 2], [v - 1]]
            assert float((r.logp + math.log(2.0)).abs().max()) <= 2.0 ** -24


def test_what_is_left_leaves_the_refused_token_out():
    """As test_gpu_block's masks at both ends, at a temperature where the draft's share is still well above rounding."""
    for kind in (F32, BF16, F16):
        for v in (40, 700, 20000):
            z = torch.full((4, 2, v), float("-inf"), dtype=kind, device=DEV)
            lo, hi = v // 3, 2 * v // 3
            z[..., lo:hi] = randn(4, 2, hi - lo, seed=650, dtype=kind, sigma=0.01)
            q = z[:, :1].clone()
            q[..., lo] += 0.25  # e^7.5 times its share at 30
            tok = torch.full((4, 1), lo, device=DEV)
            u = torch.tensor([[NEXT_TO_ONE, 0.0], [NEXT_TO_ONE, NEXT_TO_ONE], [0.0, 0.0], [0.0, NEXT_TO_ONE]], device=DEV)
            r = lm.verify_draft(z, tok, u, draft=q, inv_temp=30.0)
            t = r.tokens.tolist()
            assert r.accepted.tolist() == [0, 0, 1, 1] and lo < t[0][0] < hi and lo < t[1][0] < hi
            assert t[2] == [lo, lo] and t[3][0] == lo and lo <= t[3][1] < hi


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [40, 700, 20000])
def test_void_rows(kind, vocab):
    """NaN of either sign, +inf and rows of nothing but -inf, in the target's or the draft's row of a place that counts: nothing is drawn
    there.  In rows that do not count they change nothing."""
    target, tok, u, draft = drafted(6, 2, vocab, kind, 660)
    u[:, :2] = 0.999
    target.scatter_(2, tok[:, :1, None].expand(-1, 1, 1), -4.0)  # the first draft is refused
    draft.scatter_(2, tok[:, :1, None], draft.amax(-1)[:, :1, None])
    want = check(target, tok, u, draft)
    assert not bool(want.accepted.any())
    negative = torch.full((1,), float("nan"), dtype=kind, device=DEV)
    negative = torch.copysign(negative, torch.tensor([-1.0], dtype=kind, device=DEV))
    for bad in (float("nan"), negative, float("inf"), None):
        for rows, place in ((target, 0), (draft, 0), (target, 1), (draft, 1), (target, 2)):
            t, q = target.clone(), draft.clone()
            spoiled = t if rows is target else q
            if bad is None:
                spoiled[3, place] = float("-inf")
            else:
                spoiled[3, place, vocab // 2] = bad if isinstance(bad, float) else bad[0]
            r = lm.verify_draft(t, tok, u, draft=q)
            if place == 0:
                assert r.accepted[3] == 0 and r.tokens[3].tolist() == [-1] * 3 and math.isnan(float(r.logp[3, 0])) and not bool(r.logp[3, 1:].any())
            keep = [k for k in range(6) if k != 3 or place > 0]
            for a, b in zip(r, want):
                assert torch.equal(a[keep], b[keep])
