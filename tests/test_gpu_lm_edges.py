"""The language-model operators where alignment, run lengths and special values meet: cases beside
those of test_gpu_lm, against the same 64-bit forms and bounds."""
import pytest
import torch

import lm_reference as R
from paper_2005_06728_b200 import binding, lm
from test_gpu_lm import BF16, DEV, F16, F32, check_grad, in_poison, randn, tokens_of

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- embedding gradient: alignment

@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("dim", [24, 2048])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_workspace_on_16_bytes(dtype, dim, accumulate):
    """A workspace needs 16-byte alignment and no more: runs that cross blocks leave the same bits in it
    wherever it starts."""
    vocab = 7
    tok = torch.cat([torch.full((k,), i % vocab, device=DEV) for i, k in enumerate([1, 40, 16, 100, 3, 64, 15, 17])])
    grad = randn(tok.numel(), dim, seed=130, dtype=dtype)
    old = randn(vocab, dim, seed=131) if accumulate else torch.zeros(vocab, dim, device=DEV)
    ref, bound = R.embed_grad(tok, grad, vocab, 1.5, None, old if accumulate else None)
    need = lm.embed_grad_workspace(tok, grad, old)
    got = []
    for base in (0, 16, 48, 112):
        buffer = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device=DEV)
        assert buffer.data_ptr() % 256 == 0
        dt = old.clone()
        lm.embed_grad(tok, grad, dt, scale=1.5, accumulate=accumulate, workspace=buffer[base:base + need])
        assert bool((buffer[:base] == 0x5A).all()) and bool((buffer[base + need:] == 0x5A).all()), "written outside the workspace"
        got.append(dt)
    R.within(got[0], ref, bound, "embedding gradient")
    assert all(torch.equal(got[0], x) for x in got[1:])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("offset,pad", [(4, 0), (4, 4), (0, 4), (4, 8), (8, 8), (2, 0), (0, 2)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_16_bit_rows_into_tables_on_16_bytes(dtype, offset, pad, accumulate):
    """Eight columns a thread, into table rows of which all, some or none start on 32 bytes."""
    vocab, dim = 50, 24
    tok = tokens_of((6, 90), vocab, 132)
    tok[2] = 11  # a run over several blocks
    grad = randn(6, 90, dim + 8, seed=133, dtype=dtype)[..., :dim]
    check_grad(tok, grad, vocab, 1.5, 3, accumulate, offset, pad)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("offset,pad", [(0, 0), (4, 0), (0, 4), (4, 4)])
def test_embed_grad_late_zeros_into_tables_on_16_bytes(dtype, offset, pad):
    """A table with more rows than are zeroed beside the sort: those behind are zeroed beside the sums."""
    vocab, dim, n = 9003, 2048, 1500  # 74 MB, of which 58 MB are written beside the sort
    tok = tokens_of((n,), vocab, 134)
    tok[::4] = vocab - 1
    grad = randn(n, dim, seed=135, dtype=dtype)
    dt, check = in_poison((vocab, dim), F32, offset, pad)
    lm.embed_grad(tok, grad, dt, scale=0.5)
    ref, bound = R.embed_grad(tok, grad, vocab, 0.5)
    R.within(dt, ref, bound, "embedding gradient")
    check()


# --------------------------------------------------------------------------- no rows

@pytest.mark.parametrize("shape", [(2, 0, 3), (0, 2, 3), (2, 3, 0), (2, 0, 3, 5)])
def test_empty_batches_of_many_axes(shape):
    tok = torch.zeros(shape, dtype=torch.int64, device=DEV)
    table = randn(10, 8)
    assert lm.embed_lookup(tok, table).shape == (*shape, 8)
    dt = torch.full((10, 8), 5.0, device=DEV)
    lm.embed_grad(tok, torch.zeros(*shape, 8, device=DEV), dt, accumulate=True)
    assert bool((dt == 5).all())
    assert bool((lm.embed_grad(tok, torch.zeros(*shape, 8, device=DEV), dt) == 0).all())
    z = torch.zeros(*shape, 12, device=DEV)
    assert lm.token_logprob(z, tok).logp.shape == shape
    v = torch.zeros(shape, device=DEV)
    r = lm.policy_loss(z, tok, v, v, v)
    assert r.dlogits.shape == z.shape and r.logp.shape == shape and bool((r.stats == 0).all())
    r = lm.policy_loss(z, tok, v, v, v, ref_logp=v, kl_coef=0.1)
    assert bool((r.stats == 0).all())


# --------------------------------------------------------------------------- policy loss: special values

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [40, 5003])
def test_reference_for_the_kl_sum_alone(dtype, vocab):
    """With kl_coef 0 the reference is there for the KL sum: loss and gradient do not depend on it, whatever
    exp(ref - logp) is."""
    z = randn(6, vocab, seed=140, dtype=dtype, sigma=2.0)
    z[1, 3] = float("-inf")
    y = torch.tensor([0, 3, 5, 7, -1, 9], device=DEV)
    old, adv = randn(6, seed=141, sigma=0.1) - 8.0, randn(6, seed=142)
    w = torch.full((6,), 1 / 6, device=DEV)
    old[1] = -200.0
    want = lm.policy_loss(z, y, old, adv, w)
    ref = old.clone()
    ref[0] = 300.0  # exp overflows
    ref[2] = float("inf")
    ref[3] = float("-inf")
    got = lm.policy_loss(z, y, old, adv, w, ref_logp=ref)
    assert torch.equal(got.dlogits, want.dlogits) and torch.equal(got.logp, want.logp)
    assert bool(torch.isfinite(got.dlogits).all()) and bool(torch.isfinite(got.stats[0]))
    assert torch.equal(got.stats[[0, 1, 3]], want.stats[[0, 1, 3]]) and not bool(torch.isfinite(got.stats[2]))
    # without rows that overflow, the sum itself
    ref = want.logp + 0.3
    got = lm.policy_loss(z[2:4], y[2:4], old[2:4], adv[2:4], w[2:4], ref_logp=ref[2:4])
    kl = 2 / 6 * (torch.exp(torch.tensor(0.3, dtype=torch.float64)) - 1.3)
    assert abs(float(got.stats[2]) - float(kl)) < 1e-5


# --------------------------------------------------------------------------- calls back to back

@pytest.mark.parametrize("vocab,dim", [(64, 40), (3001, 512)])
def test_back_to_back_calls_see_what_the_ones_ahead_wrote(vocab, dim):
    """Every kernel may be scheduled while the one ahead of it still runs.  Clip into an arena, update,
    lookup in the updated weights, clip in place, norm: the same bits with and without waiting in between."""
    rounds = 12
    tok = tokens_of((257,), vocab, 150)
    g = [randn(vocab, dim, seed=151, dtype=BF16), randn(vocab, dim, seed=152, dtype=BF16)]
    w0 = randn(vocab * dim, seed=153)

    def chain(wait):
        w, v = w0.clone(), torch.zeros_like(w0)
        arenas = [torch.zeros_like(w0) for _ in range(2)]
        ctx = binding.Odsgd(w, v, n_workers=2, lr=0.5, local_lr=0.5, momentum=0.9, wd=0.01)
        into = lm.GradSet([[g[0]], [g[1]]], offsets=[0], arenas=arenas)
        own = [[t.float()] for t in g]
        place = lm.GradSet(own)
        outs = torch.zeros(rounds, 257, dim, dtype=BF16, device=DEV)
        norms = torch.zeros(rounds, 3, 2, device=DEV)
        torch.cuda.synchronize()
        sync = torch.cuda.synchronize if wait else (lambda: None)
        table = w.view(vocab, dim)
        for k in range(rounds):
            into.clip(10.0 + 3.0 * (k * 5 % rounds), out=norms[k, 0])
            sync()
            ctx.ssgd_step(arenas)
            sync()
            lm.embed_lookup(tok, table, out=outs[k])
            sync()
            place.clip(30.0 - 2.0 * k, out=norms[k, 1])
            sync()
            place.norm(out=norms[k, 2])
            sync()
        torch.cuda.synchronize()
        ctx.close()
        return w, outs, norms, own

    want, got = chain(True), chain(False)
    assert all(torch.equal(a, b) for a, b in zip(want[:3], got[:3]))
    assert all(torch.equal(a[0], b[0]) for a, b in zip(want[3], got[3]))
    for k in range(rounds):  # clipped in place to ever smaller norms
        assert bool(((got[2][k, 2] / (30.0 - 2.0 * k) - 1).abs() < 1e-5).all())
    assert not torch.equal(got[1][0], got[1][-1])


# --------------------------------------------------------------------------- embedding gradient: lengths of runs

@pytest.mark.parametrize("n", [2300, 37903, 37904, 75807, 75808, 80001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_embed_grad_runs_around_blocks(n, dtype):
    """Blocks of 16, 32 and 64 positions (37904 and 75808 tokens are the first of the larger ones): runs that are
    one shorter and longer than one, two and more blocks, one after another, and one that fills half."""
    lens = [15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 1, 95, 96, 97, 127, 128, 129, 2, 191, 192, 193, 255, 257]
    tok, i = [torch.full((n // 2,), 1, device=DEV)], 0
    left = n - n // 2
    while left > 0:
        k = min(left, lens[i % len(lens)])
        tok.append(torch.full((k,), 2 + i, device=DEV))
        left, i = left - k, i + 1
    tok = torch.cat(tok)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(160))
    check_grad(tok[order.to(DEV)], randn(n, 8, seed=161, dtype=dtype), i + 5, 0.5)


# --------------------------------------------------------------------------- autograd

@pytest.mark.parametrize("call", ["lookup", "gradient", "loss", "clip in place", "clip into arenas", "norms", "norm"])
def test_writing_over_what_autograd_saved_is_noticed(call):
    """Buffers that a caller hands over to be written count as changed in place: a backward pass that saved one
    of them fails instead of using what was written over it."""
    x = randn(4, 16, seed=170).requires_grad_()
    y = x.exp()  # its backward needs y itself
    buf = y.detach()
    tok = torch.tensor([1, 0, 3, 2], device=DEV)
    if call == "lookup":
        lm.embed_lookup(tok, randn(4, 16, seed=171), out=buf)
    elif call == "gradient":
        lm.embed_grad(tok, randn(4, 16, seed=172), buf)
    elif call == "loss":
        v = torch.ones(4, device=DEV)
        lm.policy_loss(buf, tok, -v, v, v, dlogits=buf)
    elif call == "clip in place":
        lm.GradSet([[randn(9, seed=173)], [buf]]).clip(0.1)
    elif call == "clip into arenas":
        lm.GradSet([[randn(9, seed=173)]], offsets=[3], arenas=[buf.view(-1)]).clip(0.1)
    else:
        s = lm.GradSet([[randn(9, seed=173 + k)] for k in range(64)])
        s.clip(0.1, out=buf.view(-1)) if call == "norms" else s.norm(out=buf.view(-1))
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()


@pytest.mark.parametrize("in_place", [True, False])
def test_views_of_one_tensor_and_others_are_all_noticed(in_place):
    x = [randn(40, seed=178).requires_grad_() for _ in range(3)]
    y = [t.exp() for t in x]
    bufs = [y[0].detach()[:20], y[0].detach()[20:], y[1].detach(), y[2].detach()[4:24]]
    if in_place:
        lm.GradSet([bufs]).clip(0.1)
    else:
        lm.GradSet([[randn(9, seed=179)]] * 4, offsets=[0], arenas=[b[:20] for b in bufs]).clip(0.1)
    for t in y:
        with pytest.raises(RuntimeError, match="inplace"):
            t.sum().backward()


def test_reading_changes_no_version():
    z, tok = randn(4, 16, seed=175), torch.tensor([1, 0, 3, 2], device=DEV)
    v = torch.ones(4, device=DEV)
    s = lm.GradSet([[z]])
    before = [t._version for t in (z, tok, v)]
    lm.embed_lookup(tok, z)
    lm.token_logprob(z, tok)
    lm.policy_loss(z, tok, -v, v, v)
    lm.embed_grad(tok, z, torch.zeros(4, 16, device=DEV))
    s.norm()
    assert [t._version for t in (z, tok, v)] == before


def test_inference_tensors():
    """Tensors without a version counter."""
    with torch.inference_mode():
        table, tok = randn(6, 8, seed=176), torch.tensor([5, 1], device=DEV)
        out = torch.empty(2, 8, device=DEV)
        assert lm.embed_lookup(tok, table, out=out) is out and torch.equal(out, table[tok])
        g = [[randn(40, seed=177)]]
        assert float(lm.GradSet(g).clip(0.5)[0]) > 0.5
    lm.embed_lookup(tok, table, out=out)
    assert abs(float(lm.GradSet(g).norm()[0]) - 0.5) < 1e-6


# --------------------------------------------------------------------------- memory

def test_a_kept_result_keeps_no_workspace():
    """The four sums of a loss may be kept for as long as one likes: they hold 16 bytes."""
    z, tok = randn(3, 1000, 4, seed=180), torch.zeros(3, 1000, dtype=torch.int64, device=DEV)
    v = torch.ones(3, 1000, device=DEV)
    r = lm.policy_loss(z, tok, -v, v, v)
    assert r.stats.untyped_storage().nbytes() == 16
    assert r.logp.untyped_storage().nbytes() == 4 * 3000 and r.dlogits.untyped_storage().nbytes() == 4 * z.numel()


# --------------------------------------------------------------------------- temperature

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [7, 3000])
def test_scores_at_the_ends_of_the_temperature(dtype, vocab):
    """Any positive finite inverse temperature: the largest leaves the rows' maxima, the smallest all entries alike.
    A product with it may leave the range of binary32, the maximum's own difference (0) may not."""
    z = torch.arange(vocab, device=DEV).remainder(5).to(dtype) * 0.25
    z = torch.stack([z, -z, torch.zeros_like(z)])
    y = torch.tensor([4, 0, 1], device=DEV)
    top = (z.float() == z.float().amax(-1, keepdim=True)).sum(-1)
    for c in (2.0 ** 127 * 1.9, 3e38, 2.3e38, 1e30):
        got = lm.token_logprob(z, y, inv_temp=c).logp.cpu()
        R.within(got, -torch.log(top.double().cpu()), torch.full((3,), 1e-5, dtype=torch.float64), f"logp at {c}")
    for c in (1e-45, 1e-38, 1e-20):
        got = lm.token_logprob(z, y, inv_temp=c).logp.cpu()
        R.within(got, torch.full((3,), vocab, dtype=torch.float64).log().neg(), torch.full((3,), 1e-5, dtype=torch.float64), f"logp at {c}")
    v = torch.ones(3, device=DEV)
    p = lm.policy_loss(z, y, v * 0, v, v, inv_temp=3e38, grad_scale=1e-38)
    assert bool(torch.isfinite(p.stats).all()) and bool(torch.isfinite(p.dlogits).all())


# --------------------------------------------------------------------------- capture

def test_a_set_dropped_or_made_beside_a_capture():
    """A set that goes while a graph is being recorded frees its table and leaves the recording intact; so does one
    that is made on a stream that records nothing."""
    g = [[randn(5000, seed=190)]]
    kept, dropped = lm.GradSet(g), lm.GradSet([[randn(50, seed=191)]])
    out = torch.zeros(1, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept.norm(out=out)
        dropped.close()
        other = lm.GradSet([[g[0][0][:77]]], stream=side)
    graph.replay()
    torch.cuda.synchronize()
    assert float(out[0]) == float(kept.norm()[0]) > 0
    side.synchronize()
    assert abs(float(other.norm()[0]) - float(g[0][0][:77].double().norm())) < 1e-4
