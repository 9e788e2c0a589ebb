"""Activations of the gated block and their slopes at every 16-bit number, relative to their own size."""
import math

import pytest
import torch

import block_reference as R
from lm_reference import TINY, UNIT
from paper_2005_06728_b200 import lm
from test_gpu_lm import BF16, DEV, F16

pytestmark = pytest.mark.gpu


def reference(t, name):
    """Value, slope, and what 32 bits may take from them: the exponential is off by 2^-21 and by its argument's roundings, at most
    three of 2^-24 of t (t^2 / 2), relative; the rest is sixteen roundings of 2^-22 at most.  Nothing cancels in the values; the two terms
    of a slope do, so that its error goes by their sizes."""
    if name == "silu":
        s, r = torch.sigmoid(t), torch.sigmoid(-t)
        rel = (t.abs() + 16) * 2.0 ** -22
        return t * s, s + t * s * r, rel * (t * s).abs(), rel * s * (1 + t.abs())
    cdf = torch.special.log_ndtr(t).exp()
    bell = torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)
    rel = (t * t * (t < 0) + 16) * 2.0 ** -22
    return t * cdf, cdf + t * bell, rel * (t * cdf).abs(), rel * cdf + (t * t + 16) * 2.0 ** -22 * (t * bell).abs()


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activation_of_every_number(kind, act):
    t = torch.arange(-32768, 32768, device=DEV).to(torch.int16).view(kind)
    t = t[t.isfinite() & (t.abs() <= 80)]
    x = torch.zeros(len(t), 8, dtype=kind, device=DEV)
    x[:, 0], x[:, 1] = t, 1
    wg, wu = torch.zeros(2, 1, 8, dtype=kind, device=DEV)
    wg[:, 0], wu[:, 1] = 1, 1
    value, slope, off_v, off_s = reference(t.double(), act)
    # what is below the smallest normal number of 32 bits may be lost (times t)
    off_v, off_s = off_v + t.double().abs() * 2.0 ** -126, off_s + (1 + t.double().abs()) * 2.0 ** -126
    bounds = [off + (ref.abs() + off) * UNIT[kind] * 1.01 + TINY[kind] for ref, off in ((value, off_v), (slope, off_s))]
    for many in (len(t), 1000, 16):  # more than the kernel for few tokens takes, and what it takes
        for at in range(0, len(t), many) if many > 16 else (0, 15008, len(t) - 16):
            part = slice(at, at + many)
            r = lm.gated_ffn(x[part], wg, wu, activation=act, save=True)
            assert torch.equal(r.gate[:, 0], t[part]) and bool((r.up == 1).all())
            R.within(r.h[:, 0], value[part], bounds[0][part], "value")
            g = lm.gated_ffn_grad(x[part], wg, wu, r.gate, r.up, torch.ones_like(r.h), activation=act, want_dw=False)
            R.within(g.dx[:, 0], slope[part], bounds[1][part], "slope")
            R.within(g.dx[:, 1], value[part], bounds[0][part], "value")
