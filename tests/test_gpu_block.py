"""The operators inside a worker's step, against plain 64-bit forms.

Tolerances are the bounds of block_reference, derived from the arithmetic."""
import ctypes
import math

import pytest
import torch

import block_reference as R
from paper_2005_06728_b200 import binding, lm
from test_gpu_lm import BF16, DEV, F16, F32, gen, in_poison, randn

pytestmark = pytest.mark.gpu


def stalled():
    n = ctypes.c_uint(77)
    assert binding.load_library().odsgd_stalled_waits(ctypes.byref(n)) == binding.OK
    return n.value


# --------------------------------------------------------------------------- gated feed-forward block

def block(shape, dim, width, kind, weight_kind, seed=0):
    x = randn(*shape, dim, seed=seed + 1, dtype=kind)
    return x, randn(width, dim, seed=seed + 2, dtype=weight_kind, sigma=dim ** -0.5), randn(width, dim, seed=seed + 3, dtype=weight_kind, sigma=dim ** -0.5)


def check_forward(x, wg, wu, act, **kw):
    ref = R.gated(x, wg, wu, act)
    r = lm.gated_ffn(x, wg, wu, activation=act, save=True, **kw)
    for key, (value, bound) in ref.items():
        R.within(getattr(r, key), value, bound, key)
    return r


def check_backward(x, wg, wu, gate, up, dh, act, **kw):
    old = None
    if kw.get("accumulate"):
        old = kw["dw_gate"].clone(), kw["dw_up"].clone()
    dw_kind = kw["dw_gate"].dtype if "dw_gate" in kw else None
    ref = R.gated_grad(x, wg, wu, gate, up, dh, act, dw_kind, old)
    r = lm.gated_ffn_grad(x, wg, wu, gate, up, dh, activation=act, **kw)
    for key, (value, bound) in ref.items():
        R.within(getattr(r, key), value, bound, key)
    return r


@pytest.mark.parametrize("kind,weight_kind,act", [(BF16, BF16, "silu"), (F16, F16, "gelu"), (BF16, F32, "gelu"), (F16, F32, "silu")])
@pytest.mark.parametrize("shape,dim,width", [((), 8, 8), ((1,), 1, 1), ((3,), 64, 128), ((2, 5), 72, 130), ((130,), 33, 257), ((4, 65), 200, 129),
                                             ((257,), 256, 384), ((3, 2, 50), 1000, 264), ((700,), 65, 63), ((65,), 2051, 7), ((16,), 512, 1000),
                                             ((48,), 264, 2056)])
def test_gated(kind, weight_kind, act, shape, dim, width):
    x, wg, wu = block(shape, dim, width, kind, weight_kind)
    r = check_forward(x, wg, wu, act)
    assert r.h.shape == (*shape, width) and r.h.dtype == kind
    assert torch.equal(lm.gated_ffn(x, wg, wu, activation=act).h, r.h), "the same without keeping"
    dh = randn(*shape, width, seed=9, dtype=kind)
    q = check_backward(x, wg, wu, r.gate, r.up, dh, act)
    again = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, activation=act)
    for a, b in zip(q, again):
        assert torch.equal(a, b), "a repeated call gives the same bits"
    assert stalled() == 0


@pytest.mark.parametrize("n,dim,width", [(1000, 1024, 2048), (2049, 520, 1100), (333, 2304, 5000)])
def test_gated_larger(n, dim, width):
    """Several tiles of rows and columns for each pair of CTAs, uneven ends."""
    x, wg, wu = block((n,), dim, width, BF16, BF16, seed=20)
    r = check_forward(x, wg, wu, "silu")
    check_backward(x, wg, wu, r.gate, r.up, randn(n, width, seed=29, dtype=BF16), "silu")


@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 8), (8, 0), (1, 0), (0, 3), (4, 4)])
@pytest.mark.parametrize("n,width", [(70, 72), (5, 264)])
def test_gated_strides_and_alignment(offset, pad, n, width):
    """Everything at any offset, rows further apart than their width; nothing beside the outputs is written."""
    dim = 48

    def place(t):
        rows = t.shape[:-1].numel()
        whole = torch.zeros(offset + rows * (t.shape[-1] + pad), dtype=t.dtype, device=DEV)
        view = whole[offset:].view(*t.shape[:-1], t.shape[-1] + pad)[..., :t.shape[-1]]
        return view.copy_(t)

    for weight_kind in (BF16, F32):
        x, wg, wu = (place(t) for t in block((2, n), dim, width, BF16, weight_kind, seed=30))
        out, check = in_poison((2, n, width), BF16, offset, pad)
        r = check_forward(x, wg, wu, "silu", out=out)
        assert r.h is out
        check()
        gate, up, dh = place(r.gate), place(r.up), place(randn(2, n, width, seed=31, dtype=BF16))
        for dw_kind, accumulate in ((BF16, False), (F32, False), (F32, True)):
            (dx, check_x), (dwg, check_g), (dwu, check_u) = (in_poison((2, n, dim), BF16, offset, pad), in_poison((width, dim), dw_kind, offset, pad),
                                                             in_poison((width, dim), dw_kind, offset, pad))
            check_backward(x, wg, wu, gate, up, dh, "silu", dx=dx, dw_gate=dwg, dw_up=dwu, accumulate=accumulate)
            check_x(), check_g(), check_u()


def test_gated_shifted_transposed_and_broadcast_rows():
    x, wg, wu = block((6, 9), 64, 96, F16, F16, seed=40)
    for rows in (x[:, 1:], x[1:, :-1], x.transpose(0, 1), x[:, ::2], x[2], x[:1, :1].expand(4, 7, 64)):
        r = check_forward(rows, wg, wu, "gelu")
        lead = rows.shape[:-1]
        dh = randn(*reversed(lead), 96, seed=41, dtype=F16).transpose(0, len(lead) - 1)
        check_backward(rows, wg, wu, r.gate, r.up, dh, "gelu")
    whole = randn(2 * 96, 64, seed=42, dtype=F16, sigma=0.125)  # both weights in one tensor
    check_forward(x, whole[:96], whole[96:], "silu")


def test_gated_parts_and_empty():
    x, wg, wu = block((40,), 64, 128, BF16, BF16, seed=50)
    r = lm.gated_ffn(x, wg, wu, save=True)
    dh = randn(40, 128, seed=51, dtype=BF16)
    both = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh)
    only_x = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, want_dw=False)
    only_w = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, want_dx=False)
    assert only_x.dw_gate is None and only_x.dw_up is None and only_w.dx is None
    assert torch.equal(only_x.dx, both.dx) and torch.equal(only_w.dw_gate, both.dw_gate) and torch.equal(only_w.dw_up, both.dw_up)
    none = lm.gated_ffn(x[:0], wg, wu, save=True)
    assert none.h.shape == (0, 128)
    g = lm.gated_ffn_grad(x[:0], wg, wu, none.gate, none.up, dh[:0])
    assert g.dx.shape == (0, 64) and not bool(g.dw_gate.any()) and not bool(g.dw_up.any())
    dw, check = in_poison((128, 64), F32, 0, 4)
    other = torch.ones(128, 64, device=DEV)
    lm.gated_ffn_grad(x[:0], wg, wu, none.gate, none.up, dh[:0], dw_gate=dw, dw_up=other, accumulate=True)
    assert bool((dw == 777.0).all()) and bool((other == 1).all())
    lm.gated_ffn_grad(x[:0], wg, wu, none.gate, none.up, dh[:0], dw_gate=dw, dw_up=other)
    assert not bool(dw.any()) and not bool(other.any())
    check()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_special_values(act):
    """NaN and infinities stay in their token; huge pre-activations saturate as the formulas do."""
    dim, width = 64, 128
    x, wg, wu = block((8,), dim, width, BF16, BF16, seed=60)
    clean = lm.gated_ffn(x, wg, wu, activation=act).h
    y = x.clone()
    y[2, 5], y[4, 0] = float("nan"), float("inf")
    h = lm.gated_ffn(y, wg, wu, activation=act).h
    assert bool(h[2].isnan().all()) and not bool(h[4].isfinite().any())
    keep = [0, 1, 3, 5, 6, 7]
    assert torch.equal(h[keep], clean[keep])
    big = torch.zeros(4, dim, dtype=BF16, device=DEV)
    big[:, 0] = torch.tensor([200.0, -200.0, 3e38, -3e38])
    one = torch.zeros(width, dim, dtype=BF16, device=DEV)
    one[:, 0] = 1.0
    r = lm.gated_ffn(big, one, one, activation=act, save=True)
    assert bool((r.h[0] == 200.0 * 200.0).all()) or bool(((r.h[0] - 40000).abs() <= 40000 * 2.0 ** -8).all())
    assert bool((r.h[1].abs() <= 1e-30).all()) and bool((r.h[2] == float("inf")).all()) and bool((r.h[3].abs() <= 1e-30).all())
    g = lm.gated_ffn_grad(big, one, one, r.gate, r.up, torch.ones_like(r.h), activation=act)
    assert bool(g.dx[:2].isfinite().all())


def test_gated_gradient_is_that_of_differences():
    """Directional derivatives of sum(h * dh) by central differences, in the 64-bit form around the 16-bit inputs."""
    x, wg, wu = block((12,), 32, 40, F16, F16, seed=70)
    dh = randn(12, 40, seed=71, dtype=F16)
    for act in ("silu", "gelu"):
        r = lm.gated_ffn(x, wg, wu, activation=act, save=True)
        g = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, activation=act)

        def value(a, b, c):
            t = a @ b.T
            return float(((t * torch.sigmoid(t) if act == "silu" else t * torch.special.ndtr(t)) * (a @ c.T) * dh.double()).sum())

        base = [t.double() for t in (x, wg, wu)]
        for k, grad in enumerate(g):
            way = torch.randn(base[k].shape, generator=gen(72 + k), device=DEV, dtype=torch.float64)
            at = [[b + e * way if i == k else b for i, b in enumerate(base)] for e in (1e-5, -1e-5)]
            want = (value(*at[0]) - value(*at[1])) / 2e-5
            got = float((grad.double() * way).sum())
            # gate, up, dg, du and the gradient are rounded to 11 bits: 5 roundings of terms that add up to the sum of magnitudes
            assert abs(got - want) <= 5 * 2.0 ** -11 * float((grad.double() * way).abs().sum()) * 8 + 1e-6, (act, k)


def test_gated_agrees_with_autograd_through_a_chain():
    """lookup -> block -> down projection, gradients by hand against autograd in 64 bits."""
    x, wg, wu = block((30,), 64, 96, BF16, F32, seed=80)
    xd, gd, ud = (t.double().requires_grad_() for t in (x, wg.to(BF16), wu.to(BF16)))
    t = xd @ gd.T
    h = torch.nn.functional.silu(t) * (xd @ ud.T)
    dh = randn(30, 96, seed=81, dtype=BF16)
    h.backward(dh.double())
    r = lm.gated_ffn(x, wg, wu, save=True)
    dwg, dwu = torch.zeros(96, 64, device=DEV), torch.zeros(96, 64, device=DEV)
    g = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, dw_gate=dwg, dw_up=dwu)
    for got, want in ((g.dx, xd.grad), (dwg, gd.grad), (dwu, ud.grad)):
        assert float((got.double() - want).norm() / want.norm()) < 4 * 2.0 ** -8  # four roundings to 8 bits


def test_gated_on_another_stream_and_in_a_graph():
    x, wg, wu = block((300,), 128, 256, BF16, F32, seed=90)
    dh = randn(300, 256, seed=91, dtype=BF16)
    want = lm.gated_ffn(x, wg, wu, save=True)
    grads = lm.gated_ffn_grad(x, wg, wu, want.gate, want.up, dh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lm.gated_ffn(x, wg, wu, save=True, stream=side)
    got_grads = lm.gated_ffn_grad(x, wg, wu, got.gate, got.up, dh, stream=side)
    side.synchronize()
    for a, b in zip((*want, *grads), (*got, *got_grads)):
        assert torch.equal(a, b)
    xs, dhs = x.clone(), dh.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = lm.gated_ffn(xs, wg, wu, save=True)
        g = lm.gated_ffn_grad(xs, wg, wu, r.gate, r.up, dhs)
    for seed in (92, 93):
        xs.copy_(randn(300, 128, seed=seed, dtype=BF16))
        dhs.copy_(randn(300, 256, seed=seed + 10, dtype=BF16))
        graph.replay()
        torch.cuda.synchronize()
        e = lm.gated_ffn(xs, wg, wu, save=True)
        eg = lm.gated_ffn_grad(xs, wg, wu, e.gate, e.up, dhs)
        for a, b in zip((*r, *g), (*e, *eg)):
            assert torch.equal(a, b)


def test_gated_beyond_32_bit_offsets():
    """Tokens whose rows lie more than 2^32 elements apart."""
    dim, width, far = 64, 64, (1 << 32) + 64
    whole = torch.empty(far + dim, dtype=BF16, device=DEV)
    x = whole.as_strided((2, dim), (far, 1))
    x.copy_(randn(2, dim, seed=94, dtype=BF16))
    _, wg, wu = block((1,), dim, width, BF16, BF16, seed=95)
    near = x.contiguous()
    out = whole.as_strided((2, width), (far - 128, 1), 64)
    assert torch.equal(lm.gated_ffn(x, wg, wu).h, lm.gated_ffn(near, wg, wu).h)
    want = lm.gated_ffn(near, wg, wu).h
    del x
    lm.gated_ffn(near, wg, wu, out=out)
    assert torch.equal(out, want)


def test_gated_refusals():
    x, wg, wu = block((4,), 16, 24, BF16, BF16)
    r = lm.gated_ffn(x, wg, wu, save=True)
    dh = torch.ones_like(r.h)
    with pytest.raises(TypeError):
        lm.gated_ffn(x.float(), wg, wu)
    with pytest.raises(TypeError):
        lm.gated_ffn(x, wg.half(), wu.half())
    with pytest.raises(TypeError):
        lm.gated_ffn(x, wg, wu.float())
    with pytest.raises(ValueError):
        lm.gated_ffn(x[:, :8], wg, wu)
    with pytest.raises(ValueError):
        lm.gated_ffn(x, wg, wu[:12])
    with pytest.raises(ValueError):
        lm.gated_ffn(x, wg, wu, activation="relu")
    with pytest.raises(ValueError):
        lm.gated_ffn(x.t().contiguous().t(), wg, wu)
    with pytest.raises(ValueError):
        lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, dw_gate=torch.empty_like(wg))
    with pytest.raises(ValueError):
        lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, accumulate=True)
    with pytest.raises(ValueError):
        lm.gated_ffn_grad(x, wg, wu, r.gate[:2], r.up, dh)
    with pytest.raises(binding.OdsgdError):
        lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, dw_gate=torch.empty_like(wg), dw_up=torch.empty_like(wu), accumulate=True)
    with pytest.raises(binding.OdsgdError):
        lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, dx=x)
    with pytest.raises(binding.OdsgdError):
        lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))
    with pytest.raises(binding.OdsgdError):
        lm.gated_ffn(x, wg.float(), wu.float(), workspace=torch.empty(8, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        lm.gated_ffn(x, wg, wu, workspace=torch.empty(64, dtype=torch.uint8))
    out = torch.empty(4, 24, dtype=BF16, device=DEV)
    before = out._version
    lm.gated_ffn(x, wg, wu, out=out)
    assert out._version > before, "what is written counts as changed"


# --------------------------------------------------------------------------- dropout

@pytest.mark.parametrize("kind,other", [(F32, None), (BF16, None), (F16, None), (BF16, BF16), (BF16, F32), (F16, F32), (F32, F16), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("shape", [(1,), (8,), (7,), (3, 8), (5, 13), (2, 3, 40), (4, 1, 257)])
def test_dropout(kind, other, shape):
    x = randn(*shape, seed=1, dtype=kind)
    r = None if other is None else randn(*shape, seed=2, dtype=other, sigma=3.0)
    for p, seed, offset in ((0.1, 12345, 0), (0.5, (1 << 64) - 3, (1 << 63) + 7), (0.0, 1, 2), (0.999, 5, 1 << 32)):
        got = lm.dropout(x, p, seed, offset=offset, residual=r)
        assert got.dtype == (kind if other is None else other) and got.shape == x.shape
        ref, bound = R.dropout(x, p, seed, offset, r, got.dtype)
        R.within(got, ref, bound, "dropout")
        if p == 0.0 and r is None:
            assert torch.equal(got, x)


@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 8), (8, 16), (1, 0), (0, 3), (4, 4)])
@pytest.mark.parametrize("dim", [24, 29])
def test_dropout_strides_and_alignment(offset, pad, dim):
    def place(t):
        whole = torch.zeros(offset + 10 * (dim + pad), dtype=t.dtype, device=DEV)
        return whole[offset:].view(2, 5, dim + pad)[..., :dim].copy_(t)

    x, r = place(randn(2, 5, dim, seed=3, dtype=BF16)), place(randn(2, 5, dim, seed=4))
    for view, res in ((x, r), (x, None), (x.transpose(0, 1), r.transpose(0, 1)), (x[:, 1:], r[:, 1:]), (x[:1].expand(3, 5, dim), None)):
        out, check = in_poison(tuple(view.shape), F32 if res is not None else BF16, offset, pad)
        lm.dropout(view, 0.3, 77, offset=9, residual=res, out=out)
        ref, bound = R.dropout(view, 0.3, 77, 9, res, out.dtype)
        R.within(out, ref, bound, "dropout")
        check()


def test_dropout_in_place_and_backward():
    x, r = randn(6, 40, seed=5, dtype=BF16), randn(6, 40, seed=6, dtype=BF16)
    want = lm.dropout(x, 0.25, 8, offset=1, residual=r)
    a, b = x.clone(), r.clone()
    assert lm.dropout(x, 0.25, 8, offset=1, residual=b, out=b) is b and torch.equal(b, want)
    lm.dropout(a, 0.25, 8, offset=1, out=a)
    assert torch.equal(a, lm.dropout(x, 0.25, 8, offset=1))
    # the gradient goes through the same mask, whatever the gradient's type and strides
    dy = randn(6, 44, seed=7)[:, 3:43]
    keep = R.kept((6, 40), 0.25, 8, 1).to(DEV)
    dx = lm.dropout(dy, 0.25, 8, offset=1)
    assert torch.equal(dx != 0, keep & (dy != 0)) and torch.equal(want != r, keep & (want != r))
    assert not torch.equal(lm.dropout(x, 0.25, 8, offset=2), lm.dropout(x, 0.25, 8, offset=1))
    assert not torch.equal(lm.dropout(x, 0.25, 9, offset=1), lm.dropout(x, 0.25, 8, offset=1))
    n = randn(4, 16, seed=8)
    n[1] = float("nan")
    n[2] = float("inf")
    keep = R.kept((4, 16), 0.5, 3, 0).to(DEV)
    y = lm.dropout(n, 0.5, 3)
    assert torch.equal(y.isfinite(), n.isfinite() | ~keep) and not bool(y[~keep].any())


def test_dropout_many_elements():
    """Shares of dropped elements, neighbours and calls independent, beyond 2^32 elements."""
    n = (1 << 32) + 4096
    x = torch.ones(n // 4096, 4096, dtype=BF16, device=DEV)
    y = lm.dropout(x, 0.25, 11, out=x)
    share = float((y == 0).sum(dtype=torch.int64)) / n
    assert abs(share - 0.25) < 6 * math.sqrt(0.25 * 0.75 / n)
    tail = y.view(-1)[-4096:].float()
    first = (n - 4096) // 8
    want = [h >= 16384 for b in range(first, first + 512) for w in R.philox(b, 0, 11) for h in (w & 0xFFFF, w >> 16)]
    assert torch.equal(tail != 0, torch.tensor(want, device=DEV))
    keep = y.view(-1)[:1 << 24] != 0
    both = float((keep[1:] & keep[:-1]).double().mean())
    assert abs(both - 0.5625) < 6 * math.sqrt(0.5625 * 0.4375 / (1 << 24)) * 1.5


def test_dropout_counter_and_graph():
    x = randn(50, 64, seed=10, dtype=BF16)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    lm.dropout(x, 0.1, 4, offset=3, counter=step)
    with torch.cuda.graph(graph):
        y = lm.dropout(x, 0.1, 4, offset=3, counter=step)
        step += 1
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, lm.dropout(x, 0.1, 4, offset=3 + k))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z = lm.dropout(x, 0.1, 4, offset=3, stream=side)
    side.synchronize()
    assert torch.equal(z, lm.dropout(x, 0.1, 4, offset=3))


def test_dropout_refusals_and_empty():
    x = randn(4, 16)
    assert lm.dropout(x[:0], 0.1, 1).shape == (0, 16) and lm.dropout(x[:, :0], 0.1, 1).shape == (4, 0)
    for p in (-0.1, 1.0, float("nan"), 0.99999999):
        with pytest.raises(binding.OdsgdError):
            lm.dropout(x, p, 1)
    with pytest.raises(ValueError):
        lm.dropout(x, 0.1, -1)
    with pytest.raises(ValueError):
        lm.dropout(x, 0.1, 1, offset=1 << 64)
    with pytest.raises(ValueError):
        lm.dropout(x, 0.1, 1, residual=x[:2])
    with pytest.raises(ValueError):
        lm.dropout(x.t(), 0.1, 1)
    with pytest.raises(TypeError):
        lm.dropout(x.double(), 0.1, 1)
    with pytest.raises(TypeError):
        lm.dropout(x, 0.1, 1, residual=x, out=torch.empty_like(x, dtype=BF16))
    with pytest.raises(TypeError):
        lm.dropout(x, 0.1, 1, counter=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        lm.dropout(x, 0.1, 1, counter=torch.zeros(2, dtype=torch.int64, device=DEV))
    whole = randn(5, 16)
    with pytest.raises(binding.OdsgdError):
        lm.dropout(whole[:4], 0.1, 1, out=whole[1:])
    with pytest.raises(binding.OdsgdError):
        lm.dropout(x, 0.1, 1, out=torch.empty(1, 16, device=DEV).expand(4, 16))
    with pytest.raises(binding.OdsgdError):
        lm.dropout(x, 0.1, 1, out=x.view(-1).view(BF16)[:64].view(4, 16))
    before = x._version
    lm.dropout(x, 0.1, 1, out=x)
    assert x._version > before


# --------------------------------------------------------------------------- drafted tokens

def drafted(batch, drafts, vocab, kind, seed, with_draft=True, sigma=2.5, int_kind=torch.int64):
    base = randn(batch, drafts + 1, vocab, seed=seed, sigma=sigma)
    target = base.to(kind)
    draft = (base[:, :drafts] + randn(batch, drafts, vocab, seed=seed + 1, sigma=0.6)).to(kind)
    probs = torch.softmax(draft.float() * (1.25 if with_draft else 4.0), -1)
    tok = torch.multinomial(probs.view(-1, vocab), 1, generator=gen(seed + 2)).view(batch, drafts) if drafts else torch.zeros(batch, 0, dtype=torch.int64, device=DEV)
    u = torch.rand(batch, drafts + 1, generator=gen(seed + 3), device=DEV)
    return target, tok.to(int_kind), u, draft if with_draft else None


def check_verify(target, tok, u, draft, inv_temp=1.25, draft_inv_temp=None, **kw):
    """Decisions are equal where the 64-bit form is further than 1e-11 from any border (its own sums are off by 1e-13 or so);
    the seeds of these tests are."""
    r = lm.verify_draft(target, tok, u, draft=draft, inv_temp=inv_temp, draft_inv_temp=draft_inv_temp, **kw)
    accepted, tokens, logp, near = R.verify(target, tok, u, draft, inv_temp, inv_temp if draft_inv_temp is None else draft_inv_temp)
    assert near > 1e-11, "a draw on the border: choose another seed"
    assert torch.equal(r.accepted.cpu().long(), accepted)
    assert torch.equal(r.tokens.cpu().long(), tokens) and r.tokens.dtype == tok.dtype
    # the sum is added in 32 bits in parts, exponentials are off by 2^-21: bound as for a sum of so many terms in a tree
    mag = float((target.double().nan_to_num(0, 0, 0).abs().amax() * inv_temp).clamp(max=1e30))
    bound = torch.full_like(logp, 2.0 ** -19 + mag * 2.0 ** -21)
    R.within(r.logp.cpu(), logp, bound, "logp")
    return r


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("batch,drafts,vocab", [(1, 0, 1), (1, 1, 1), (3, 2, 7), (2, 4, 33), (5, 3, 1000), (4, 2, 4099), (3, 5, 20001), (9, 1, 513),
                                                (2, 9, 64), (40, 0, 100), (2, 3, 70000)])
@pytest.mark.parametrize("with_draft", [True, False])
def test_verify(kind, batch, drafts, vocab, with_draft):
    check_verify(*drafted(batch, drafts, vocab, kind, 100 + vocab + drafts, with_draft, int_kind=torch.int32 if vocab % 2 else torch.int64))


def test_verify_many_sequences_accept_and_refuse():
    r = check_verify(*drafted(300, 4, 50, BF16, 300, sigma=1.0))
    assert len(set(r.accepted.tolist())) == 5, "every number of accepted drafts occurs"
    again = lm.verify_draft(*drafted(300, 4, 50, BF16, 300, sigma=1.0)[:3], draft=drafted(300, 4, 50, BF16, 300, sigma=1.0)[3], inv_temp=1.25)
    for a, b in zip(r, again):
        assert torch.equal(a, b)


def test_verify_most_drafts():
    target, tok, u, _ = drafted(2, 255, 40, F16, 310, False)
    check_verify(target, tok, u * 1e-3, None)  # low numbers: long runs are accepted


def test_verify_strides_and_padding():
    target, tok, u, draft = drafted(4, 3, 1001, BF16, 320)
    tok[1, 2:], tok[2, 0], tok[3] = -1, 1001, -5
    check_verify(target, tok, u, draft)
    wide_t, wide_d = torch.zeros(4, 4, 1010, dtype=BF16, device=DEV), torch.zeros(3, 4, 1003, dtype=BF16, device=DEV).transpose(0, 1)
    wide_t[..., 5:1006], wide_d[..., 1:1002] = target, draft
    check_verify(wide_t[..., 5:1006], tok.t().contiguous().t(), u.t().contiguous().t(), wide_d[..., 1:1002])
    check_verify(target.transpose(0, 1).contiguous().transpose(0, 1), tok, u[:1].expand(4, 4), draft)
    check_verify(target, tok, u, draft, inv_temp=0.7, draft_inv_temp=3.0)


def test_verify_borders():
    """Random numbers on the border itself, decided in 64 bits: u q = p refuses, the next number below accepts."""
    z = torch.zeros(1, 2, 4, device=DEV)  # uniform target: p = 1/4
    tok = torch.tensor([[2]], device=DEV)
    u = torch.tensor([[0.25, 0.0]], device=DEV)
    assert lm.verify_draft(z, tok, u).accepted.tolist() == [0]
    r = lm.verify_draft(z, tok, torch.tensor([[0.25 - 2.0 ** -26, 0.0]], device=DEV))
    assert r.accepted.tolist() == [1] and r.tokens.tolist() == [[2, 0]]
    # what is left of a uniform target without token 2: a third each, drawn at its borders
    for last, want in ((0.0, 0), (0.33, 0), (0.34, 1), (0.66, 1), (0.67, 3), (1.0 - 2.0 ** -24, 3)):
        assert lm.verify_draft(z, tok, torch.tensor([[0.9, last]], device=DEV)).tokens.tolist() == [[want, -1]]
    same = drafted(6, 2, 300, BF16, 330)
    r = lm.verify_draft(same[0], same[1], same[2], draft=same[0][:, :2].contiguous())
    assert r.accepted.tolist() == [2] * 6, "equal distributions accept everything"
    for last, want in ((0.0, 0), (0.25, 1), (0.5, 2), (0.75, 3)):  # cum > u whole: at a border the next one
        assert lm.verify_draft(z[:, :1], tok[:, :0], torch.tensor([[last]], device=DEV)).tokens.tolist() == [[want]]


def test_verify_masked_and_void_rows():
    target, tok, u, draft = drafted(6, 2, 500, F32, 340)
    target[..., 100:] = float("-inf")
    draft[..., 100:] = float("-inf")
    tok.clamp_(max=99)
    tok[0, 0] = 400  # neither gives it a probability
    check_verify(target, tok, u, draft)
    low = target.clone()
    low[..., 100:] = torch.finfo(F32).min
    for a, b in zip(lm.verify_draft(low, tok, u, draft=draft), lm.verify_draft(target, tok, u, draft=draft)):
        assert torch.equal(a, b)
    one = torch.full((1, 1, 300), float("-inf"), device=DEV)
    one[0, 0, 299] = -5.0
    r = lm.verify_draft(one, tok[:1, :0], u[:1, :1])
    assert r.tokens.tolist() == [[299]] and r.logp.tolist() == [[0.0]]
    for bad in (float("nan"), float("inf"), None):
        void = target.clone()
        if bad is None:
            void[2, 0] = float("-inf")
        else:
            void[2, 0, 50] = bad
        r = lm.verify_draft(void, tok, u, draft=draft)
        want = lm.verify_draft(target, tok, u, draft=draft)
        assert r.accepted[2] == 0 and r.tokens[2].tolist() == [-1, -1, -1] and math.isnan(float(r.logp[2, 0]))
        keep = [0, 1, 3, 4, 5]
        for a, b in zip(r, want):
            assert torch.equal(a[keep], b[keep])


def test_verify_masks_at_the_ends():
    """Random numbers of 0 and next to 1 pass over masked tokens at both ends, whatever the mask's value and the temperature."""
    for kind in (F32, BF16, F16):
        for v in (40, 700, 20000):
            for mask in (float("-inf"), torch.finfo(kind).min, -6e4):
                z = torch.full((4, 2, v), mask, dtype=kind, device=DEV)
                lo, hi = v // 3, 2 * v // 3
                z[..., lo:hi] = randn(4, 2, hi - lo, seed=345, dtype=kind)
                q = z[:, :1].clone()
                q[..., lo] += 3  # what is left does not hold the first
                tok = torch.full((4, 1), lo, device=DEV)
                u = torch.tensor([[1 - 2.0 ** -24, 0.0], [1 - 2.0 ** -24, 1 - 2.0 ** -24], [0.0, 0.0], [0.0, 1 - 2.0 ** -24]], device=DEV)
                for c in (1.0, 0.05, 30.0):
                    r = lm.verify_draft(z, tok, u, draft=q, inv_temp=c)
                    t = r.tokens.tolist()
                    # (at 30 the draft's share of token lo may be below what 64 bits hold beside the rest: equal distributions then)
                    first = lo if c == 30.0 else lo + 1
                    assert r.accepted.tolist() == [0, 0, 1, 1] and first <= t[0][0] < hi and first <= t[1][0] < hi, (kind, v, mask, c)
                    assert t[2][1] == lo and lo <= t[3][1] < hi and t[2][0] == t[3][0] == lo


def test_verify_draws_as_the_target_does():
    """Drafts of another distribution, verified: what comes out first is distributed as the target (5 tokens, 200000 sequences)."""
    n, v = 65536, 5
    zt, zq = torch.tensor([0.3, -1.0, 1.2, 0.0, -0.4], device=DEV), torch.tensor([1.5, 0.2, -0.7, 0.1, 0.0], device=DEV)
    counts = torch.zeros(v, device=DEV)
    for k in range(3):
        tok = torch.multinomial(torch.softmax(zq, 0), n, replacement=True, generator=gen(350 + k)).view(n, 1)
        u = torch.rand(n, 2, generator=gen(360 + k), device=DEV)
        r = lm.verify_draft(zt.expand(n, 2, v), tok, u, draft=zq.expand(n, 1, v))
        counts += torch.bincount(r.tokens[:, 0], minlength=v)
    p = torch.softmax(zt, 0)
    off = (counts / (3 * n) - p).abs() / (p * (1 - p) / (3 * n)).sqrt()
    assert float(off.max()) < 5


def test_verify_streams_graphs_and_refusals():
    target, tok, u, draft = drafted(3, 2, 5000, BF16, 370)
    want = lm.verify_draft(target, tok, u, draft=draft)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lm.verify_draft(target, tok, u, draft=draft, stream=side)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    us, graph = u.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = lm.verify_draft(target, tok, us, draft=draft)
    for k in range(3):
        us.copy_(torch.rand(3, 3, generator=gen(380 + k), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(r, lm.verify_draft(target, tok, us, draft=draft)):
            assert torch.equal(a, b)
    assert lm.verify_draft(target[:0], tok[:0], u[:0], draft=draft[:0]).tokens.shape == (0, 3)
    with pytest.raises(TypeError):
        lm.verify_draft(target, tok, u, draft=draft.half())
    with pytest.raises(TypeError):
        lm.verify_draft(target, tok, u.double())
    with pytest.raises(ValueError):
        lm.verify_draft(target, tok[:, :1], u)
    with pytest.raises(ValueError):
        lm.verify_draft(target, tok, u[:, :2])
    with pytest.raises(ValueError):
        lm.verify_draft(target, tok, u, draft=draft[..., :100])
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-31, 1e31):
        with pytest.raises(binding.OdsgdError):
            lm.verify_draft(target, tok, u, inv_temp=t)
    with pytest.raises(binding.OdsgdError):
        lm.verify_draft(target, tok, u, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(binding.OdsgdError):
        lm.verify_draft(randn(1, 258, 4), torch.zeros(1, 257, dtype=torch.int64, device=DEV), torch.zeros(1, 258, device=DEV))


def test_verify_beyond_32_bit_offsets():
    v = 1 << 20
    target = torch.zeros(16, 256, v, dtype=BF16, device=DEV)  # 2^32 elements
    target[15, 255, v - 1] = 60.0
    target[15, :255, 7] = 60.0
    tok = torch.full((16, 255), 7, device=DEV)
    tok[:15] = -1
    u = torch.full((16, 256), 0.5, device=DEV)
    r = lm.verify_draft(target, tok, u)
    assert r.accepted.tolist() == [0] * 15 + [255] and r.tokens[15].tolist() == [7] * 255 + [v - 1]
    assert r.tokens[:15, 0].tolist() == [v // 2] * 15


# --------------------------------------------------------------------------- together, in the token policy

def test_policy_example_with_block_dropout_and_drafts():
    from paper_2005_06728_b200 import policy_example

    for kw in (dict(block=96), dict(block=50, drop=0.2), dict(drafts=3), dict(block=72, drop=0.1, drafts=4, vocab=53, dim=40)):
        a, b = policy_example.train(steps=8, **kw), policy_example.train(steps=8, **kw)
        assert all(math.isfinite(v) for v in a.losses) and bool(a.weights.isfinite().all())
        assert a.rewards == b.rewards and torch.equal(a.weights, b.weights), "a run can be repeated"
    with pytest.raises(ValueError):
        policy_example.train(steps=1, drop=0.1)


def test_policy_example_gradients():
    """lookup, block, dropout, head: the gradients of all tensors against autograd in 64 bits."""
    from paper_2005_06728_b200 import policy_example

    vocab, dim, width, p = 61, 48, 72, 0.25
    model = policy_example.GatedModel(vocab, dim, width, p)
    w = model.views(model.init(5, torch.device(DEV)))
    tokens = torch.randint(0, vocab, (6, 10), generator=gen(400), device=DEV)
    tokens[2, 7:] = -1
    z, kept = model.forward(w, tokens, 9, 4, training=True)
    dz = randn(6, 10, vocab, seed=401, dtype=BF16)
    dz[2, 7:] = 0
    out = model.gradients(torch.device(DEV))
    model.backward(w, tokens, kept, dz, out)
    v = {k: t.double().requires_grad_() for k, t in w.items()}
    x = torch.nn.functional.embedding(tokens.clamp(min=0), v["embedding"]) * math.sqrt(dim) * (tokens >= 0)[..., None]
    t = x @ v["gate"].T
    y = (t * torch.sigmoid(t) * (x @ v["up"].T)) @ v["down"].T
    s = x + torch.where(R.kept((6, 10, dim), p, 9, 4).to(DEV), y / 0.75, torch.zeros((), dtype=torch.float64, device=DEV))
    zz = s @ v["head"].T
    zz.backward(dz.double())
    # along the longest way (embedding) some twelve roundings to 8 bits, each of at most 2^-8 and of either sign
    assert float((z.double() - zz.detach()).norm() / zz.detach().norm()) < 6 * 2.0 ** -8
    for (name, _), got in zip(model.shapes, out):
        want = v[name].grad
        assert float((got.double() - want).norm() / want.norm()) < 12 * 2.0 ** -8, name


def test_drafted_answers_carry_their_scores():
    from paper_2005_06728_b200 import policy_example

    z = randn(9, 14, 37, seed=410, sigma=1.5)
    draft = z + randn(9, 14, 37, seed=411, sigma=0.7)
    counts = torch.arange(14, device=DEV)[None, :] < torch.tensor([14, 1, 7, 13, 2, 14, 5, 9, 3], device=DEV)[:, None]
    for drafts in (1, 3, 20):
        answers, acting = policy_example.drafted_answers(z, draft, counts, drafts, gen(412 + drafts))
        assert bool((answers >= 0).all()) and bool((answers < 37).all())
        want = lm.token_logprob(z, answers).logp
        # both are sums of 37 exponentials in 32 bits
        assert float((acting - want)[counts].abs().max()) < 40 * 2.0 ** -22
        assert not bool(acting[~counts].any())


# --------------------------------------------------------------------------- calls that nothing prepared

FIRST_CALLS_CAPTURED = """
import torch
from paper_2005_06728_b200 import lm
g = torch.Generator(device="cuda").manual_seed(1)
r = lambda *s, k=torch.bfloat16: torch.randn(*s, generator=g, device="cuda").to(k)
x, wg, wu, dh, z, tok = r(40, 72), r(130, 72, k=torch.float32), r(130, 72, k=torch.float32), r(40, 130), r(3, 3, 3000), torch.tensor([[1, 2]] * 3, device="cuda")
big, u = r(2100, 72), torch.full((3, 3), 0.3, device="cuda")
step = torch.zeros(1, dtype=torch.int64, device="cuda")
def run():
    a = lm.gated_ffn(x, wg, wu, save=True)
    return (*a, *lm.gated_ffn_grad(x, wg, wu, a.gate, a.up, dh), lm.gated_ffn(big, wg, wu).h, lm.dropout(x, 0.5, 3, counter=step, residual=x),
            *lm.verify_draft(z, tok, u), *lm.verify_draft(z[..., :500], tok, u))
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    got = run()
graph.replay()
torch.cuda.synchronize()
for a, b in zip(got, run()):
    assert torch.equal(a, b)
print("equal")
"""


def test_first_calls_of_a_process_can_be_captured():
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS_CAPTURED], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "equal", r.stderr[-2000:]


def test_calls_on_two_streams_at_once():
    """Every kernel on two streams with nothing between them but the GPU's own order; each has its own tensors and workspace."""
    streams, sets = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for k in range(2):
        x, wg, wu = block((500 if k else 30,), 264, 400, BF16, F32 if k else BF16, seed=500 + 10 * k)
        sets.append((x, wg, wu, randn(x.shape[0], 400, seed=505 + 10 * k, dtype=BF16), drafted(6, 3, 9000, BF16, 520 + 10 * k)))

    def run(s, stream):
        x, wg, wu, dh, (target, tok, u, draft) = s
        r = lm.gated_ffn(x, wg, wu, save=True, stream=stream)
        g = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, dh, stream=stream)
        return (*r, *g, lm.dropout(x, 0.2, 5, residual=x, stream=stream), *lm.verify_draft(target, tok, u, draft=draft, stream=stream))

    want = [[t.clone() for t in run(s, None)] for s in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k in (0, 1):
            got[k].append(run(sets[k], streams[k]))
    torch.cuda.synchronize()
    for k in (0, 1):
        for outs in got[k]:
            for a, b in zip(outs, want[k]):
                assert torch.equal(a, b)
    assert stalled() == 0


def test_back_to_back_calls_read_what_the_one_ahead_wrote():
    """Grids are scheduled while the one ahead drains: dropout onto h in place, h through the block again, drafts from its result."""
    x, wg, wu = block((600,), 128, 128, BF16, BF16, seed=540)
    tok, u = torch.zeros(600, 0, dtype=torch.int64, device=DEV), torch.full((600, 1), 0.6, device=DEV)

    def run(wait):
        h = x.clone()
        for k in range(4):
            h = lm.gated_ffn(h, wg, wu).h
            wait()
            lm.dropout(h, 0.1, 7, offset=k, out=h)
            h = lm.dropout(h, 0.3, 8, offset=k, residual=x)
            wait()
        return h, *lm.verify_draft(h.view(600, 1, 128), tok, u)

    for a, b in zip(run(lambda: None), run(torch.cuda.synchronize)):
        assert torch.equal(a, b)
