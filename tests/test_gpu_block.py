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
        lm.gated_ffn(x, wg, wu, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        lm.gated_ffn(x, wg, wu, workspace=torch.empty(64, dtype=torch.uint8))
    out = torch.empty(4, 24, dtype=BF16, device=DEV)
    before = out._version
    lm.gated_ffn(x, wg, wu, out=out)
    assert out._version > before, "what is written counts as changed"
