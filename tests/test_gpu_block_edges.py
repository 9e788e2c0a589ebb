"""Calls of the operators inside a worker's step that their documentation allows and test_gpu_block does not make."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2005_06728_b200 import lm
from test_gpu_block import block, drafted
from test_gpu_lm import BF16, DEV, F32, randn

pytestmark = pytest.mark.gpu


def all_calls():
    x, wg, wu = block((2, 20), 72, 130, BF16, F32, seed=700)
    r = lm.gated_ffn(x, wg, wu, save=True)
    g = lm.gated_ffn_grad(x, wg, wu, r.gate, r.up, randn(2, 20, 130, seed=703, dtype=BF16))
    target, tok, u, draft = drafted(3, 2, 3000, BF16, 710)
    return (*r, *g, lm.dropout(x, 0.3, 5, residual=x), *lm.verify_draft(target, tok, u, draft=draft), *lm.token_logprob(target, u.long()))


class Dispatched(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.calls = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.calls.append(str(func))
        return func(*args, **(kwargs or {}))


def test_new_memory_under_modes():
    want = all_calls()
    with Dispatched() as m:
        got = all_calls()
    assert any("empty" in c for c in m.calls)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    try:
        torch.use_deterministic_algorithms(True)
        x = randn(4, 8)
        got = lm.dropout(x, 0.3, 5), lm.dropout(x, 0.3, 5, out=torch.zeros_like(x))
        assert torch.equal(*got) and bool(lm._new(x, (3, 5), F32, None).isnan().all())
    finally:
        torch.use_deterministic_algorithms(False)


def test_stalled_waits_waits_for_every_stream():
    x, wg, wu = block((300,), 264, 400, BF16, F32, seed=720)
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # some tenth of a second
        lm.gated_ffn(x, wg, wu)
        done.record()
    assert not done.query()
    assert lm.stalled_waits() == 0
    assert done.query()
    y = torch.zeros(4, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError):
            lm.stalled_waits()
        y += 1
    graph.replay()
    torch.cuda.synchronize()
    assert y.tolist() == [1.0] * 4, "the capture went on"


def test_a_run_whose_products_were_cut_short_is_void(monkeypatch):
    from paper_2005_06728_b200 import policy_example

    counts = iter((0, 1))
    monkeypatch.setattr(lm, "stalled_waits", lambda: next(counts))
    with pytest.raises(RuntimeError, match="void"):
        policy_example.train(steps=1, block=40)


@pytest.mark.parametrize("shape,dim,width", [((1,), 1, 1), ((2, 9), 33, 65), ((70,), 200, 129), ((300,), 1001, 257), ((9000,), 40, 24)])
def test_what_a_workspace_held_before_has_no_effect(shape, dim, width):
    """Workspaces of NaN (every byte 0xff), larger than needed, against those that a call makes."""
    for weight_kind in (BF16, F32):
        x, wg, wu = block(shape, dim, width, BF16, weight_kind, seed=730)
        dh = randn(*shape, width, seed=733, dtype=BF16)
        ws = torch.full((1 << 26,), 255, dtype=torch.uint8, device=DEV)
        want = lm.gated_ffn(x, wg, wu, save=True)
        grads = lm.gated_ffn_grad(x, wg, wu, want.gate, want.up, dh)
        got = lm.gated_ffn(x, wg, wu, save=True, workspace=ws)
        ws.fill_(255)
        got_grads = lm.gated_ffn_grad(x, wg, wu, want.gate, want.up, dh, workspace=ws)
        for a, b in zip((*want, *grads), (*got, *got_grads)):
            assert torch.equal(a, b)
    for vocab in (40, 5000):
        target, tok, u, draft = drafted(3, 2, vocab, BF16, 740)
        ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV)
        for q in (draft, None):
            for a, b in zip(lm.verify_draft(target, tok, u, draft=q), lm.verify_draft(target, tok, u, draft=q, workspace=ws)):
                assert torch.equal(a, b)
