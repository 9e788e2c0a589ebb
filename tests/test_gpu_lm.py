"""The language-model operators around the update, against plain 64-bit forms.

Tolerances are the bounds of lm_reference, derived from the arithmetic."""
import math

import pytest
import torch

import lm_reference as R
from paper_2005_06728_b200 import binding, lm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
POISON = 777.0


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(*shape, seed=0, dtype=F32, sigma=1.0):
    return (torch.randn(*shape, generator=gen(seed), device=DEV) * sigma).to(dtype)


def in_poison(shape, dtype, offset=0, pad=0):
    """A view [..., n] with `pad` spare elements behind each row, `offset` elements into a poisoned
    buffer; returns (view, check), check() asserting that nothing outside the view was written."""
    *lead, n = shape
    rows = math.prod(lead)
    whole = torch.full((64 + offset + rows * (n + pad) + 64,), POISON, dtype=dtype, device=DEV)
    view = whole[64 + offset:64 + offset + rows * (n + pad)].view(*lead, n + pad)[..., :n]

    def check():
        mask = torch.ones_like(whole, dtype=torch.bool)
        mask[64 + offset:64 + offset + rows * (n + pad)].view(*lead, n + pad)[..., :n] = False
        assert bool((whole[mask] == POISON).all()), "written outside the output"
    return view, check


def tokens_of(shape, vocab, seed, dtype=torch.int64, bad=True):
    t = torch.randint(0, vocab, shape, generator=gen(seed), device=DEV, dtype=dtype)
    if bad and t.numel() >= 4:
        f = t.reshape(-1)
        f[0], f[1], f[-1] = -1, vocab, (2 ** 40 if dtype == torch.int64 else 2 ** 31 - 1)
        t = f.view(shape)
    return t


# --------------------------------------------------------------------------- lookup

@pytest.mark.parametrize("table_type", [F32, BF16, F16])
@pytest.mark.parametrize("out_type", [F32, BF16, F16])
@pytest.mark.parametrize("shape,vocab,dim", [((), 5, 8), ((1,), 1, 1), ((6,), 9, 3), ((3, 7), 50, 64), ((2, 3, 5), 20, 17),
                                             ((4, 33), 1000, 1000), ((7,), 30, 4104)])
def test_lookup(table_type, out_type, shape, vocab, dim):
    table = randn(vocab, dim, seed=1, dtype=table_type)
    tok = tokens_of(shape, vocab, 2)
    out, check = in_poison((*shape, dim), out_type)
    got = lm.embed_lookup(tok, table, scale=1.7, out=out)
    assert got is out
    ref = R.lookup(tok, table, float(torch.tensor(1.7)))
    R.within(out, ref, R.lookup_bound(ref, out_type), "lookup")
    check()


@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 8), (4, 4), (1, 0), (0, 3)])
def test_lookup_strides_and_alignment(offset, pad):
    """Tables inside an arena at any offset, rows further apart than their width, shifted and
    transposed tokens, int32 tokens."""
    vocab, dim = 40, 72
    whole = randn(offset + vocab * (dim + pad), seed=3)
    table = whole[offset:].view(vocab, dim + pad)[:, :dim]
    both = tokens_of((5, 12), vocab, 4, torch.int32, bad=False)
    for tok in (both[:, 1:], both.t(), both[:, ::2], both[1]):
        out, check = in_poison((*tok.shape, dim), BF16, offset, pad)
        lm.embed_lookup(tok, table, out=out)
        ref = R.lookup(tok, table, 1.0)
        R.within(out, ref, R.lookup_bound(ref, BF16), "lookup")
        check()
    assert lm.embed_lookup(both[:0], table).shape == (0, 12, dim)
    assert torch.equal(lm.embed_lookup(both, table), table[both.long()]), "scale 1 copies"


def test_lookup_beyond_32_bit_offsets():
    table = torch.empty(70000, 65536, dtype=BF16, device=DEV)  # 4.6e9 elements
    table[69999] = 3.0
    table[66000] = 5.0
    out = lm.embed_lookup(torch.tensor([69999, 66000, -1], device=DEV), table, scale=2.0)
    assert bool((out[0] == 6).all()) and bool((out[1] == 10).all()) and bool((out[2] == 0).all())


# --------------------------------------------------------------------------- embedding gradient

def test_embed_grad_beyond_32_bit_offsets():
    dt = torch.full((70000, 65536), POISON, device=DEV)  # 4.6e9 elements
    tok = torch.tensor([69999, 5, 69999, 66001, -1], device=DEV)
    g = randn(5, 65536, seed=119, dtype=BF16)
    lm.embed_grad(tok, g, dt, scale=2.0)
    assert torch.equal(dt[69999], 2 * (g[0].float() + g[2].float())) and torch.equal(dt[66001], 2 * g[3].float())
    assert torch.equal(dt[5], 2 * g[1].float())
    for row in (0, 4, 6, 32767, 65535, 65536, 66000, 66002, 69998):
        assert not bool(dt[row].any()), "rows that no token names are zero"
    assert float(dt[::7].double().abs().sum()) == float(dt[[r for r in (5, 66001, 69999) if r % 7 == 0]].double().abs().sum())


def check_grad(tok, grad, vocab, scale=1.0, padding=None, accumulate=False, offset=0, pad=0):
    dim = grad.shape[-1]
    dt, check = in_poison((vocab, dim), F32, offset, pad)
    old = None
    if accumulate:
        old = randn(vocab, dim, seed=77)
        dt.copy_(old)
    scale32 = float(torch.tensor(scale, dtype=F32))
    ref, bound = R.embed_grad(tok, grad, vocab, scale32, padding, old)
    lm.embed_grad(tok, grad, dt, scale=scale, padding_token=padding, accumulate=accumulate)
    R.within(dt, ref, bound, "embedding gradient")
    check()
    # equal inputs, equal bits, whatever the workspace held
    again, _ = in_poison((vocab, dim), F32, offset, pad)
    if accumulate:
        again.copy_(old)
    need = lm.embed_grad_workspace(tok, grad, dt)
    ws = torch.full((max(16, need),), 0xAB, dtype=torch.uint8, device=DEV)
    lm.embed_grad(tok, grad, again, scale=scale, padding_token=padding, accumulate=accumulate, workspace=ws)
    assert torch.equal(dt, again)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("shape,vocab,dim", [((1,), 1, 1), ((0,), 3, 5), ((5,), 1, 8), ((33,), 7, 16), ((3, 50), 40, 129),
                                             ((2, 700), 600, 64), ((2, 3, 41), 3000, 24), ((9, 200), 70000, 8),
                                             ((4, 100), 300000, 4), ((2, 600), 90, 1100)])
def test_embed_grad(dtype, accumulate, shape, vocab, dim):
    tok = tokens_of(shape, vocab, 5)
    check_grad(tok, randn(*shape, dim, seed=6, dtype=dtype), vocab, 2.5, None, accumulate)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["one token", "one token and padding", "none valid", "natural", "runs", "sorted"])
def test_embed_grad_token_frequencies(dtype, kind):
    n, vocab, dim = 5003, 997, 40
    padding = None
    if kind == "one token":
        tok = torch.full((n,), 3, device=DEV)
    elif kind == "one token and padding":
        tok = torch.where(torch.arange(n, device=DEV) % 3 == 0, 3, 996)
        padding = 996
    elif kind == "none valid":
        tok = torch.full((n,), -1, device=DEV)
    elif kind == "natural":
        u = torch.rand(n, generator=gen(8), device=DEV)
        tok = (vocab ** u - 1).long().clamp(0, vocab - 1)
    elif kind == "runs":  # lengths around the block sizes, one after another
        lens = [15, 16, 17, 31, 32, 33, 1, 1, 64, 127, 128, 129, 255, 257, 3]
        tok = torch.cat([torch.full((k,), i, device=DEV) for i, k in enumerate(lens * 4)])[:n]
    else:
        tok = torch.arange(n, device=DEV) * vocab // n
    grad = randn(tok.numel(), dim, seed=9, dtype=dtype)
    check_grad(tok, grad, vocab, 1.0, padding)
    check_grad(tok, grad, vocab, 1.0, padding, accumulate=True)


@pytest.mark.parametrize("vocab", [1, 2, 30, 255, 256, 511, 512, 513, 131071, 262144])
@pytest.mark.parametrize("n", [1024, 1025, 3000, 33000])
def test_embed_grad_digits(vocab, n):
    """One to three digit passes of every width, and the two sorts on either side of their border."""
    check_grad(tokens_of((n,), vocab, 17), randn(n, 4, seed=18), vocab)


@pytest.mark.parametrize("n", [1023, 1024, 1026, 1031, 2047, 2048, 2049, 4095, 4097, 8183, 8191, 8192, 8193, 8201, 12007])
@pytest.mark.parametrize("kind", ["all different", "few tokens", "one and none"])
def test_embed_grad_sort_borders(n, kind):
    """Around the powers of two and the borders between the three sorts, at parts that are full, ragged and empty."""
    if kind == "all different":
        vocab = n + 5
        tok = (torch.arange(n, device=DEV) * 4799 + 11) % n
    elif kind == "few tokens":
        vocab = 3
        tok = torch.arange(n, device=DEV) % 4 - 1
    else:
        vocab = 70001
        tok = torch.where(torch.arange(n, device=DEV) * 13 % 8 < 5, 70000, vocab)
    check_grad(tok, randn(n, 8, seed=19, dtype=BF16), vocab)


@pytest.mark.parametrize("vocab", [4194302, 4194303, 4194304, 5000001])
@pytest.mark.parametrize("n", [1, 33, 700, 1024, 1500, 8192])
def test_embed_grad_large_vocabularies(n, vocab):
    """On either side of the vocabulary whose tokens are sorted in 32 bits with their place."""
    tok = tokens_of((n,), vocab, 21)
    tok[::3] = vocab - 1
    tok[1::7] = vocab
    check_grad(tok, randn(n, 1, seed=22), vocab)


@pytest.mark.parametrize("n,dim", [(70001, 32), (300000, 8), (4096, 2056)])
def test_embed_grad_many_tokens(n, dim):
    vocab = 5000
    u = torch.rand(n, generator=gen(10), device=DEV)
    tok = (vocab ** u - 1).long().clamp(0, vocab - 1)
    check_grad(tok, randn(n, dim, seed=11, dtype=BF16), vocab)


@pytest.mark.parametrize("offset,pad", [(0, 8), (4, 4), (1, 0), (0, 3), (2, 2)])
def test_embed_grad_strides_and_alignment(offset, pad):
    vocab, dim = 50, 24
    tok = tokens_of((6, 90), vocab, 12, torch.int32)
    g = randn(6, 90, dim + pad, seed=13)[..., :dim]
    check_grad(tok[:, 1:], g[:, :-1], vocab, 1.5, None, False, offset, pad)
    check_grad(tok.t(), g.transpose(0, 1), vocab, 1.5, None, True, offset, pad)
    # one gradient row for all positions of a sequence
    check_grad(tok, g[:, :1].expand(6, 90, dim), vocab, 1.0, None, False, offset, pad)


def test_embed_grad_is_the_lookup_transposed():
    """<grad, lookup(E)> == <embed_grad(grad), E> for any table E (the lookup is linear in its
    table, so this is its directional derivative)."""
    tok = tokens_of((4, 60), 80, 14)
    grad, E = randn(4, 60, 32, seed=15), randn(80, 32, seed=16)
    a = (R.host(grad) * R.host(lm.embed_lookup(tok, E, scale=0.7))).sum()
    dt = lm.embed_grad(tok, grad, torch.empty(80, 32, device=DEV), scale=0.7)
    b = (R.host(dt) * R.host(E)).sum()
    mag = (R.host(grad).abs() * R.host(lm.embed_lookup(tok, E, scale=0.7)).abs()).sum()
    assert abs(a - b) <= 240 * R.U * mag


# --------------------------------------------------------------------------- scores

VOCABS = [(F32, 1), (F32, 2), (F32, 7), (F32, 129), (F32, 1000), (F32, 4099), (F32, 131072), (F32, 131080),
          (BF16, 1), (BF16, 9), (BF16, 33), (BF16, 1000), (BF16, 32768), (BF16, 50021), (BF16, 262144), (BF16, 262153),
          (F16, 5), (F16, 4099), (F16, 70000)]


@pytest.mark.parametrize("dtype,vocab", VOCABS)
@pytest.mark.parametrize("rows", [1, 5])
def test_scores(dtype, vocab, rows):
    z = randn(rows, vocab, seed=20, dtype=dtype, sigma=3.0)
    y = tokens_of((rows,), vocab, 21)
    got = lm.token_logprob(z, y, inv_temp=1.25)
    logp, lse, ok = R.scores(z, y, 1.25)
    R.within(got.logp, logp, R.score_bound(z, 1.25, logp), "logp")
    R.within(got.lse, lse, R.score_bound(z, 1.25, lse), "lse")


def test_scores_of_many_rows():
    z = randn(3, 701, 517, seed=22, dtype=BF16, sigma=3.0)
    y = tokens_of((3, 701), 517, 23)
    got = lm.token_logprob(z[:, :-1], y[:, 1:])  # the shifted view that scores the next token
    logp, lse, _ = R.scores(z[:, :-1], y[:, 1:], 1.0)
    R.within(got.logp, logp, R.score_bound(z[:, :-1], 1.0, logp), "logp")
    R.within(got.lse, lse, R.score_bound(z[:, :-1], 1.0, lse), "lse")
    t = lm.token_logprob(z.transpose(0, 1), y.t())
    whole = lm.token_logprob(z, y)
    assert torch.equal(t.logp, whole.logp.t()) and torch.equal(t.lse, whole.lse.t())
    one = lm.token_logprob(z[1, 2], y[1, 2])
    assert one.logp.shape == () and lm.token_logprob(z[:0], y[:0]).logp.shape == (0, 701)


# --------------------------------------------------------------------------- policy loss

def policy_inputs(z, y, seed, c, beta=True):
    """Ratios on both sides of the clip bounds and between them, none near a bound."""
    logp, _, _ = R.scores(z, y, c)
    logp = torch.nan_to_num(logp, nan=-3.0, neginf=-3.0, posinf=0.0).float().to(DEV)
    n = logp.numel()
    step = torch.tensor([-0.9, -0.4, -0.1, 0.0, 0.05, 0.15, 0.5, 0.8], device=DEV)
    r = step[torch.randint(0, 8, (n,), generator=gen(seed), device=DEV)].view(logp.shape)
    adv = torch.randn(logp.shape, generator=gen(seed + 1), device=DEV)
    ref = logp + 0.5 * torch.randn(logp.shape, generator=gen(seed + 2), device=DEV)
    w = torch.rand(logp.shape, generator=gen(seed + 3), device=DEV) / max(1, n)
    w = torch.where(torch.rand(logp.shape, generator=gen(seed + 4), device=DEV) < 0.25, torch.zeros_like(w), w)
    return logp - r, adv, w, (ref if beta else None)


def check_policy(z, y, seed=30, c=1.25, beta=0.07, gs=1.0, dlogits=None, extra=None):
    old, adv, w, ref = policy_inputs(z, y, seed, c, beta != 0)
    if extra is not None:
        old, adv, w, ref = extra(old, adv, w, ref)
    want = R.policy(z, y, old, adv, w, ref, 0.2, 0.28, beta, c, gs)
    got = lm.policy_loss(z, y, old, adv, w, ref_logp=ref, clip_low=0.2, clip_high=0.28, kl_coef=beta, inv_temp=c,
                         grad_scale=gs, dlogits=dlogits)
    R.within(got.logp, want["logp"], want["e_logp"], "logp")
    R.within(got.dlogits, want["dlogits"], want["e_dlogits"], "dlogits")
    R.within(got.stats, want["stats"], want["e_stats"], "stats")
    assert got.loss.data_ptr() == got.stats.data_ptr()
    return got


@pytest.mark.parametrize("dtype,vocab", VOCABS)
@pytest.mark.parametrize("rows", [1, 6])
def test_policy_loss(dtype, vocab, rows):
    z = randn(rows, vocab, seed=31, dtype=dtype, sigma=3.0)
    check_policy(z, tokens_of((rows,), vocab, 32), gs=512.0 if dtype == F16 else 1.0)


@pytest.mark.parametrize("dtype,vocab", [(F32, 1000), (BF16, 4104), (BF16, 517), (F16, 33)])
def test_policy_loss_of_many_rows(dtype, vocab):
    z = randn(4, 151, vocab, seed=33, dtype=dtype, sigma=2.0)
    y = tokens_of((4, 151), vocab, 34)
    gs = 4096.0 if dtype == F16 else 1.0
    a = check_policy(z, y, gs=gs)
    b = check_policy(z, y, gs=gs)
    for p, q in zip(a, b):
        assert torch.equal(p, q), "equal inputs give equal bits"
    check_policy(z[:, :-1], y[:, 1:], beta=0.0, gs=gs)
    check_policy(z.transpose(0, 1), y.t(), gs=gs)


@pytest.mark.parametrize("dtype,vocab", [(F32, 37), (BF16, 1000), (BF16, 50021), (BF16, 300000), (F32, 140000)])
def test_policy_loss_in_place(dtype, vocab):
    z = randn(2, 3, vocab, seed=35, dtype=dtype, sigma=3.0)
    y = tokens_of((2, 3), vocab, 36, bad=False)
    out = check_policy(z, y)
    old, adv, w, ref = policy_inputs(z, y, 30, 1.25)
    copy = z.clone()
    got = lm.policy_loss(copy, y, old, adv, w, ref_logp=ref, clip_low=0.2, clip_high=0.28, kl_coef=0.07, inv_temp=1.25,
                         dlogits=copy)
    assert got.dlogits.data_ptr() == copy.data_ptr()
    assert torch.equal(got.dlogits, out.dlogits) and torch.equal(got.stats, out.stats)


@pytest.mark.parametrize("zo,zp,do,dp", [(0, 8, 0, 8), (1, 0, 1, 0), (1, 0, 0, 0), (0, 0, 3, 5), (5, 3, 2, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_loss_alignment(dtype, zo, zp, do, dp):
    vocab = 1003
    z, _ = in_poison((3, 4, vocab), dtype, zo, zp)
    z.copy_(randn(3, 4, vocab, seed=37, sigma=2.0))
    dz, check = in_poison((3, 4, vocab), dtype, do, dp)
    check_policy(z, tokens_of((3, 4), vocab, 38), dlogits=dz)
    check()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [40, 1000, 70000])
def test_policy_loss_masks(dtype, vocab):
    """Masked vocabulary entries (-inf, and the type's lowest value), rows that do not count and hold
    anything, a row whose mask leaves nothing."""
    z = randn(9, vocab, seed=39, dtype=dtype, sigma=2.0)
    y = torch.arange(9, device=DEV) * 3 % (vocab // 2)
    z[:, vocab // 2:] = float("-inf")
    z[1, vocab // 2:] = torch.finfo(dtype).min
    z[2, 1:] = float("-inf")
    y[2] = 0
    z[3] = float("-inf")
    z[4] = float("nan")
    z[5] = float("inf")
    z[6] = float("nan")
    y[6] = -100
    z[8, 11] = float("nan")

    def extra(old, adv, w, ref):
        w = torch.full_like(w, 0.1)
        w[4] = w[5] = 0.0
        w[3] = w[8] = 0.0
        return old, adv, w, ref
    got = check_policy(z, y, extra=extra, c=1.0)
    assert bool((got.dlogits[3:7] == 0).all()) and bool((got.dlogits[:3, vocab // 2 + 1:] == 0).all())
    assert float(got.logp[2]) == 0.0, "one entry left: probability one"
    # the same rows counted: NaN in their own results, and only there
    old, adv, w, ref = policy_inputs(z, y, 30, 1.0)
    w = torch.full_like(w, 0.1)
    got = lm.policy_loss(z, y, old, adv, w, ref_logp=ref, kl_coef=0.1)
    bad = torch.isnan(got.dlogits).any(-1).cpu()
    assert bad.tolist() == [False, False, False, True, True, True, False, False, True]
    assert bool(torch.isnan(got.stats[0]))
    sc = lm.token_logprob(z, y)
    assert torch.isnan(sc.logp).cpu().tolist() == bad.tolist()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_rows_of_the_lowest_value(dtype):
    """Nothing but the type's lowest value: every entry equally likely, at any temperature."""
    vocab = 3001
    z = torch.full((2, vocab), torch.finfo(dtype).min, dtype=dtype, device=DEV)
    z[1] = torch.finfo(dtype).max
    y = torch.tensor([7, 3000], device=DEV)
    for c in (0.5, 1.0, 2.0):
        got = lm.token_logprob(z, y, inv_temp=c)
        assert bool(((got.logp + math.log(vocab)).abs() < 1e-5).all())
        one = torch.ones(2, device=DEV)
        p = lm.policy_loss(z, y, got.logp, one, one, inv_temp=c)
        want = torch.full((2, vocab), c / vocab, dtype=torch.float64)
        want[0, 7] -= c
        want[1, 3000] -= c
        R.within(p.dlogits, want, want.abs() * (R.UNIT[dtype] + 1e-5) + R.TINY[dtype], "dlogits")


def test_policy_loss_beyond_32_bit_offsets():
    rows, vocab = 34000, 131072  # 4.5e9 logits, in place
    z = torch.empty(rows, vocab, dtype=BF16, device=DEV)
    for a in range(0, rows, 2000):
        z[a:a + 2000] = torch.randn(2000, vocab, generator=gen(120 + a), device=DEV, dtype=BF16)
    pick = torch.tensor([0, 16383, 16384, 32767, 32768, 33999], device=DEV)
    few = z[pick].clone()
    y = torch.randint(0, vocab, (rows,), generator=gen(121), device=DEV)
    adv, w = randn(rows, seed=122), torch.full((rows,), 1.0, device=DEV)
    old = torch.full((rows,), -12.0, device=DEV)
    want = lm.policy_loss(few, y[pick], old[pick], adv[pick], w[pick])
    got = lm.policy_loss(z, y, old, adv, w, dlogits=z)
    # fewer rows are cut differently: the same sums in another order
    R.within(got.logp[pick], R.host(want.logp), 2 * R.score_bound(few, 1.0, R.host(want.logp)), "logp")
    g = R.host(want.dlogits)
    R.within(z[pick], g, g.abs() * (2 * R.UNIT[BF16] + 1e-4) + R.TINY[BF16], "dlogits")


def test_policy_loss_label_of_probability_zero():
    z = randn(4, 64, seed=40)
    z[:, 5] = float("-inf")
    y = torch.full((4,), 5, device=DEV)
    adv = torch.tensor([1.0, -1.0, 2.0, 0.0], device=DEV)
    w = torch.full((4,), 0.25, device=DEV)
    got = lm.policy_loss(z, y, torch.zeros(4, device=DEV), adv, w)
    assert bool(torch.isinf(got.logp).all()) and bool((got.dlogits == 0).all())
    # ratio 0: min(0, (1 - low) A): the bound is active where the advantage is negative
    assert abs(float(got.stats[0]) - 0.25 * 0.8) < 1e-6 and abs(float(got.stats[3]) - 0.25) < 1e-6


def test_policy_loss_broadcast_inputs_and_empty():
    z = randn(5, 21, 300, seed=41, dtype=BF16)
    y = tokens_of((5, 21), 300, 42)

    def extra(old, adv, w, ref):
        return old, adv[:, :1].expand(5, 21), torch.full((), 1 / 105, device=DEV).expand(5, 21), ref
    check_policy(z, y, extra=extra)
    e = lm.policy_loss(z[:, :0], y[:, :0], *[torch.zeros(5, 0, device=DEV)] * 3)
    assert e.dlogits.shape == (5, 0, 300) and bool((e.stats == 0).all())


def test_int32_labels():
    z = randn(4, 19, 700, seed=47, dtype=BF16)
    y = tokens_of((4, 20), 700, 48)[:, 1:].clamp(-100, 5000)
    old, adv, w, _ = policy_inputs(z, y, 49, 1.0)
    a, b = lm.token_logprob(z, y), lm.token_logprob(z, y.int())
    assert torch.equal(a.logp, b.logp) and torch.equal(a.lse, b.lse)
    p, q = lm.policy_loss(z, y, old, adv, w), lm.policy_loss(z, y.int(), old, adv, w)
    assert all(torch.equal(s, t) for s, t in zip(p, q))


def test_policy_loss_gradient_against_differences():
    """Central differences of the 64-bit loss.  Its third derivative along one logit is below
    8 c^3 |w| (|A| r + beta (e^d + 1)), so the difference quotient with step h is off by less than
    h^2 / 6 times that; its own rounding is 2^-53 times the terms over h."""
    c, beta, h = 1.25, 0.07, 1e-4
    z = randn(6, 11, seed=43, sigma=2.0)
    y = tokens_of((6,), 11, 44, bad=False)
    old, adv, w, ref = policy_inputs(z, y, 45, c)
    w = torch.full_like(w, 1 / 6)
    got = lm.policy_loss(z, y, old, adv, w, ref_logp=ref, clip_low=0.2, clip_high=0.28, kl_coef=beta, inv_temp=c)
    want = R.policy(z, y, old, adv, w, ref, 0.2, 0.28, beta, c)
    z64 = z.double()
    loss = lambda x: R.policy(x, y, old, adv, w, ref, 0.2, 0.28, beta, c)["stats"][0]  # noqa: E731
    R.UNIT[torch.float64], R.TINY[torch.float64] = 0.0, 0.0
    size = float((w.abs().cpu() * (adv.abs().cpu() * 4 + beta * 8)).max())
    for i in range(6):
        for j in range(11):
            up, dn = z64.clone(), z64.clone()
            up[i, j] += h
            dn[i, j] -= h
            num = float(loss(up) - loss(dn)) / (2 * h)
            bound = h * h / 6 * 8 * c ** 3 * size + 1e-11 + float(want["e_dlogits"][i, j])
            assert abs(num - float(got.dlogits[i, j])) <= bound


# --------------------------------------------------------------------------- norm and clip

SIZES = [1, 5, 0, 4096, 4097, 100001, 16, 33000]


def grads_of(groups, dtypes, seed, sizes=SIZES, sigma=0.01):
    return [[randn(n, seed=seed + 100 * g + k, dtype=dtypes[(k + g) % len(dtypes)], sigma=sigma) for k, n in enumerate(sizes)]
            for g in range(groups)]


def check_clip(groups, max_norm, offsets, arena_len, shift=0):
    arenas, checks = zip(*[in_poison((arena_len,), F32, shift) for _ in groups])
    st = lm.GradSet(groups, offsets=offsets, arenas=arenas)
    norms = None
    for _ in range(3):  # the set is used every iteration
        norms = st.clip(max_norm)
    for g, tensors in enumerate(groups):
        norm, k, scaled = R.clip(tensors, float(torch.tensor(max_norm)))
        assert abs(float(norms[g]) - norm) <= norm * R.U * 1.01
        covered = torch.zeros(arena_len, dtype=torch.bool)
        for t, o, s in zip(tensors, offsets, scaled):
            R.within(arenas[g][o:o + t.numel()], s.reshape(-1), R.clip_bound(s.reshape(-1), F32), "arena")
            covered[o:o + t.numel()] = True
        assert bool((arenas[g].cpu()[~covered] == POISON).all()), "padding between tensors is not written"
        checks[g]()
    assert torch.equal(st.norm(), norms)
    st.close()


def packed(sizes, gap):
    off, at = [], 0
    for n in sizes:
        off.append(at)
        at += n + gap if gap < 0 or gap > 3 else (n + 3) // 4 * 4 + gap
    return off, at + 8


@pytest.mark.parametrize("dtypes", [[F32], [BF16], [F16], [F32, BF16, F16]])
@pytest.mark.parametrize("over", [0.5, 3.0])
@pytest.mark.parametrize("gap,shift", [(0, 0), (1, 0), (0, 1), (5, 3)])
def test_clip_into_arenas(dtypes, over, gap, shift):
    groups = grads_of(3, dtypes, 50)
    norm = R.clip(groups[0], 1e30)[0]
    check_clip(groups, norm / over, *packed(SIZES, gap), shift=shift)


def test_clip_large_sets_and_misaligned_sources():
    sizes = [3_000_001, 7_000_000, 12, 999_999]
    groups = [[t[1:] for t in g] for g in grads_of(2, [BF16, F32], 60, [n + 1 for n in sizes])]
    check_clip(groups, 0.5, *packed(sizes, 0))
    groups = grads_of(1, [F32], 61, [12_000_000])  # above the size where chunks grow
    check_clip(groups, 0.5, [0], 12_000_000)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_clip_in_place(dtype):
    groups = grads_of(2, [dtype], 70)
    keep = [[t.clone() for t in g] for g in groups]
    st = lm.GradSet(groups)
    norm = [R.clip(g, 1e30)[0] for g in keep]
    got = st.clip(norm[0] * norm[1] * 1e9)  # nothing to clip: every bit stays
    for g in range(2):
        assert abs(float(got[g]) - norm[g]) <= norm[g] * R.U * 1.01
        assert all(torch.equal(a, b) for a, b in zip(groups[g], keep[g]))
    bound = min(norm) * 0.25
    st.clip(bound)
    for g in range(2):
        _, _, scaled = R.clip(keep[g], float(torch.tensor(bound)))
        for a, s in zip(groups[g], scaled):
            R.within(a, s, R.clip_bound(s, dtype), "in place")


def test_norm_range_and_special_values():
    """64-bit sums of squares: tiny and huge elements count; infinities and NaN as documented."""
    tiny, huge = torch.full((1000,), 1e-30, device=DEV), torch.full((1000,), 1e30, device=DEV)
    inf, nan = huge.clone(), huge.clone()
    inf[3], nan[5] = float("inf"), float("nan")
    zero = torch.zeros(1000, device=DEV)
    groups = [[tiny], [huge], [inf], [nan], [zero], []]
    arenas = [torch.full((1000,), POISON, device=DEV) for _ in groups]
    st = lm.GradSet(groups, offsets=[0], arenas=arenas)
    n = st.clip(1.0).cpu()
    for got, want in ((n[0], 1e-30 * 1000 ** 0.5), (n[1], 1e30 * 1000 ** 0.5)):
        assert abs(float(got) / want - 1) < 1e-6
    assert math.isinf(float(n[2])) and math.isnan(float(n[3])) and float(n[4]) == 0 and float(n[5]) == 0
    assert torch.equal(arenas[0], tiny), "below the bound: copied"
    assert abs(float(arenas[1].double().norm()) - 1) < 1e-6
    assert bool((arenas[2][torch.arange(1000) != 3] == 0).all()) and bool(torch.isnan(arenas[2][3]))
    assert bool((arenas[3][torch.arange(1000) != 5] == huge[0]).all()) and bool(torch.isnan(arenas[3][5]))
    assert torch.equal(arenas[4], zero) and bool((arenas[5] == POISON).all())
    st.clip(0.0)
    assert bool((arenas[1] == 0).all())
    empty = lm.GradSet([[], []])
    assert empty.clip(1.0).tolist() == [0.0, 0.0]


def test_clip_equal_bits_each_time():
    groups = grads_of(2, [BF16], 80, [1_000_003, 77])
    arenas = [torch.zeros(1_000_100, device=DEV) for _ in groups]
    st = lm.GradSet(groups, offsets=[0, 1_000_004], arenas=arenas)
    first = st.clip(0.1).clone()
    a = [x.clone() for x in arenas]
    for _ in range(20):
        assert torch.equal(st.clip(0.1), first)
    assert all(torch.equal(x, y) for x, y in zip(a, arenas))


# --------------------------------------------------------------------------- streams, graphs, refusals

def test_side_stream_and_graph():
    """The whole chain on another stream, and captured into a graph and replayed on new inputs."""
    V, D, B, S = 400, 64, 3, 20
    tok = tokens_of((B, S), V, 90)
    table, head = randn(V, D, seed=91, sigma=0.5), randn(D, V, seed=92, sigma=0.3)
    old, adv = randn(B, S, seed=93, sigma=0.1) - 6.0, randn(B, S, seed=94)
    w = torch.full((B, S), 1 / (B * S), device=DEV)
    arena = torch.zeros(V * D, device=DEV)
    dtable = torch.empty(V, D, device=DEV)
    st = lm.GradSet([[dtable]], offsets=[0], arenas=[arena])
    norms = torch.zeros(1, device=DEV)

    def step(stream=None):
        x = lm.embed_lookup(tok, table, scale=8.0, stream=stream)
        p = lm.policy_loss(x @ head, tok, old, adv, w, stream=stream)
        lm.embed_grad(tok, p.dlogits @ head.t(), dtable, scale=8.0, stream=stream)
        st.clip(0.01, out=norms, stream=stream)
        return p.stats

    want = step().clone()
    want_arena = arena.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    arena.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(arena, want_arena)
    arena.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stats = step()
        with pytest.raises(binding.OdsgdError) as e:
            lm.GradSet([[dtable]])
        assert e.value.code == binding.ERR_STATE
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(stats, want) and torch.equal(arena, want_arena)
    tok.copy_((tok + 7) % V)
    graph.replay()
    torch.cuda.synchronize()
    replayed, replayed_arena = stats.clone(), arena.clone()
    assert torch.equal(step(), replayed) and torch.equal(arena, replayed_arena)


def refused(code, f, *a, **k):
    with pytest.raises(binding.OdsgdError) as e:
        f(*a, **k)
    assert e.value.code == code, str(e.value)
    return str(e.value)


def test_refusals():
    tok = torch.zeros(4, 3, dtype=torch.int64, device=DEV)
    table = randn(10, 8)
    z = randn(4, 3, 16)
    v = torch.zeros(4, 3, device=DEV)
    with pytest.raises(TypeError):
        lm.embed_lookup(tok.float(), table)
    with pytest.raises(TypeError):
        lm.embed_lookup(tok.cpu(), table)
    with pytest.raises(TypeError):
        lm.embed_lookup(tok, table.double())
    with pytest.raises(ValueError):
        lm.embed_lookup(tok, table.t())
    with pytest.raises(ValueError):
        lm.embed_lookup(tok, table, out=torch.empty(4, 3, 9, device=DEV))
    with pytest.raises(ValueError):
        lm.embed_lookup(torch.zeros(2, 3, 4, 5, dtype=torch.int64, device=DEV).transpose(0, 2), table)
    flat = torch.zeros(400, device=DEV)
    assert "overlap" in refused(binding.ERR_OVERLAP, lm.embed_lookup, tok, flat[:80].view(10, 8), out=flat[40:136].view(4, 3, 8))
    assert "rows" in refused(binding.ERR_OVERLAP, lm.embed_lookup, tok, table, out=flat[:8].expand(4, 3, 8))
    refused(binding.ERR_ARG, lm.embed_lookup, tok, table, scale=float("nan"))
    with pytest.raises(TypeError):
        lm.embed_grad(tok, randn(4, 3, 8), table.bfloat16())
    with pytest.raises(ValueError):
        lm.embed_grad(tok, randn(4, 3, 9), table)
    assert "workspace" in refused(binding.ERR_ARG, lm.embed_grad, tok, randn(4, 3, 8), table, workspace=flat[:4])
    refused(binding.ERR_ALIGN, lm.embed_grad, tok, randn(4, 3, 8), table, workspace=torch.zeros(1 << 16, device=DEV)[1:])
    refused(binding.ERR_OVERLAP, lm.embed_grad, tok, flat[:96].view(4, 3, 8), flat[90:170].view(10, 8))
    with pytest.raises(ValueError):
        lm.token_logprob(z, tok[:, :2])
    refused(binding.ERR_ARG, lm.token_logprob, z, tok, inv_temp=0.0)
    refused(binding.ERR_ARG, lm.token_logprob, z, tok, inv_temp=float("inf"))
    ok = (z, tok, v, v, v)
    assert "ref_logp" in refused(binding.ERR_ARG, lm.policy_loss, *ok, kl_coef=0.1)
    refused(binding.ERR_ARG, lm.policy_loss, *ok, clip_low=-0.1)
    refused(binding.ERR_ARG, lm.policy_loss, *ok, clip_high=float("nan"))
    refused(binding.ERR_ARG, lm.policy_loss, *ok, grad_scale=float("inf"))
    with pytest.raises(TypeError):
        lm.policy_loss(z, tok, v.double(), v, v)
    with pytest.raises(ValueError):
        lm.policy_loss(z, tok, v[:, :1], v, v)
    with pytest.raises(TypeError):
        lm.policy_loss(*ok, dlogits=z.bfloat16())
    whole = randn(4, 4, 16)
    assert "dlogits" in refused(binding.ERR_OVERLAP, lm.policy_loss, whole[:, :-1], tok, v, v, v, dlogits=whole[:, 1:])
    refused(binding.ERR_OVERLAP, lm.policy_loss, *ok, dlogits=flat[:16].expand(4, 3, 16))
    g = randn(100)
    with pytest.raises(ValueError):
        lm.GradSet([])
    with pytest.raises(ValueError):
        lm.GradSet([[randn(4, 4).t()]])
    with pytest.raises(ValueError):
        lm.GradSet([[g]], arenas=[flat])
    with pytest.raises(TypeError):
        lm.GradSet([[g.double()]])
    refused(binding.ERR_OVERLAP, lm.GradSet, [[g, g[50:]]])
    refused(binding.ERR_OVERLAP, lm.GradSet, [[g, g.clone()]], offsets=[0, 50], arenas=[flat])
    refused(binding.ERR_OVERLAP, lm.GradSet, [[flat[:100]]], offsets=[0], arenas=[flat])
    refused(binding.ERR_ARG, lm.GradSet, [[g]], offsets=[301], arenas=[flat])
    refused(binding.ERR_ARG, lm.GradSet, [[g]] * 65)
    st = lm.GradSet([[g]])
    refused(binding.ERR_OVERLAP, st.clip, 1.0, out=g[99:])
    refused(binding.ERR_ARG, st.clip, -1.0)
    refused(binding.ERR_ARG, st.clip, float("nan"))
    with pytest.raises(ValueError):
        st.norm(out=torch.zeros(2, device=DEV))
    st.close()
    with pytest.raises(ValueError):
        st.norm()
    lm.GradSet([[g, g[50:]]], offsets=[0, 100], arenas=[flat])  # sources may share memory
    torch.cuda.synchronize()


# --------------------------------------------------------------------------- the calls together

def test_policy_example_learns_and_repeats():
    """The example's workers find most of the right answers (chance is 1 in 61), and a second run has
    the same bits."""
    from paper_2005_06728_b200 import policy_example

    a = policy_example.train(steps=120)
    assert sum(a.rewards[:10]) / 10 < 0.1 and sum(a.rewards[-10:]) / 10 > 0.5
    assert max(max(n) for n in a.norms) > 0.5, "some gradients were clipped"
    b = policy_example.train(steps=120)
    assert torch.equal(a.weights, b.weights) and a.losses == b.losses and a.norms == b.norms


def test_chain_against_autograd():
    """Lookup, two products, loss and both gradients against torch's derivative of the 64-bit loss.
    The longest sums have 400 terms and there are four of them one after another: 4 * 400 u = 1e-4
    of the sums of magnitudes, which here stay within a few times the results' norm."""
    V, D, B, S = 53, 24, 5, 80
    tok, y = tokens_of((B, S), V, 110), tokens_of((B, S), V, 111, bad=False)
    E, H = randn(V, D, seed=112, sigma=0.5), randn(V, D, seed=113, sigma=0.4)
    x = lm.embed_lookup(tok, E, scale=2.0)
    z = x @ H.t()
    old, adv, w, ref = policy_inputs(z, y, 114, 1.25)
    r = lm.policy_loss(z, y, old, adv, w, ref_logp=ref, clip_low=0.2, clip_high=0.28, kl_coef=0.07, inv_temp=1.25)
    dz = r.dlogits.view(-1, V)
    dH = dz.t() @ x.view(-1, D)
    dE = lm.embed_grad(tok, (dz @ H).view(B, S, D), torch.empty_like(E), scale=2.0)
    e64, h64 = E.double().cpu().requires_grad_(), H.double().cpu().requires_grad_()
    t = tok.cpu()
    ok = (t >= 0) & (t < V)
    x64 = e64[t.clamp(0, V - 1)] * 2.0 * ok[..., None]
    lp = torch.log_softmax(x64 @ h64.t() * 1.25, -1).gather(-1, y.cpu()[..., None])[..., 0]
    rt = torch.exp(lp - R.host(old))
    pg = -torch.minimum(rt * R.host(adv), rt.clamp(0.8, 1.28) * R.host(adv))
    d = R.host(ref) - lp
    loss = (R.host(w) * (pg + 0.07 * (torch.expm1(d) - d))).sum()
    loss.backward()
    assert abs(float(r.loss) - float(loss.detach())) <= 1e-4 * float((R.host(w) * R.host(adv).abs()).sum())
    for got, want in ((dE, e64.grad), (dH, h64.grad)):
        assert float((R.host(got) - want).norm()) <= 1e-4 * float(want.norm())
