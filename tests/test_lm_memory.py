"""New memory of lm.py's calls is made by torch's factory functions wherever something looks at what those do.  On the CPU: the short way
is replaced by a record of its calls."""
import pytest
import torch
from torch.overrides import TorchFunctionMode
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2005_06728_b200 import lm

SHAPES = [((2, 3), (3, 1)), ((4, 0, 5), (5, 5, 1)), ((), ()), (7, (1,)), (None, (6, 1))]


class Dispatched(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.calls = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.calls.append(func)
        return func(*args, **(kwargs or {}))


class Functions(TorchFunctionMode):
    def __init__(self):
        super().__init__()
        self.calls = []

    def __torch_function__(self, func, types, args=(), kwargs=None):
        self.calls.append(func)
        return func(*args, **(kwargs or {}))


@pytest.fixture
def short(monkeypatch):
    calls = []

    def record(shape, strides, dtype):
        calls.append((shape, strides, dtype))
        return torch.empty_strided(shape, strides, dtype=dtype)

    monkeypatch.setattr(lm, "_empty_strided", record)
    return calls


@pytest.mark.parametrize("shape,strides", SHAPES)
@pytest.mark.parametrize("dtype", [None, torch.int32])
def test_both_ways_make_the_same(short, monkeypatch, shape, strides, dtype):
    like = torch.zeros(6, 5).t()[:5, :].expand(5, 6) if shape is None else torch.zeros(3)
    a = lm._new(like, shape, dtype, None)
    assert len(short) == 1 and short[0][1] == strides
    monkeypatch.setattr(lm, "_empty_strided", None)
    b = lm._new(like, shape, dtype, None)
    for t in (a, b):
        assert t.shape == ((shape,) if type(shape) is int else like.shape if shape is None else shape)
        assert t.is_contiguous() and t.dtype == (dtype or like.dtype)


@pytest.mark.parametrize("mode", [Dispatched, Functions])
@pytest.mark.parametrize("shape,strides", SHAPES)
def test_modes_see_new_memory(short, mode, shape, strides):
    like = torch.zeros(5, 6)
    with mode() as m:
        lm._new(like, shape, torch.float32, None)
    assert len(m.calls) >= 1 and not short


@pytest.mark.parametrize("shape,strides", SHAPES[:1] + SHAPES[3:])
def test_deterministic_algorithms_fill_new_memory(short, shape, strides):
    before = torch.are_deterministic_algorithms_enabled(), torch.utils.deterministic.fill_uninitialized_memory
    try:
        torch.use_deterministic_algorithms(True)
        torch.utils.deterministic.fill_uninitialized_memory = True
        t = lm._new(torch.zeros(5, 6), shape, torch.float32, None)
        assert bool(t.isnan().all()) and not short
    finally:
        torch.use_deterministic_algorithms(before[0])
        torch.utils.deterministic.fill_uninitialized_memory = before[1]
