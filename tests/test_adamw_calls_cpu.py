"""Calls of one optimizer that overlap: each hands over its own gradients. No GPU: the library's entry is replaced by one that records what it is given."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2501_07145_amd import linear


class Recorder:
    """The library, as far as RfsfAdamW calls it. `before`: called once, before the first step reads what it was given, as another thread would run there."""

    def __init__(self):
        self.before, self.steps = None, []

    def rfsf_adamw_step(self, address, count, config, stream):
        before, self.before = self.before, None
        if before:
            before()
        words = np.ctypeslib.as_array(ctypes.cast(address, ctypes.POINTER(ctypes.c_int64)), (count, 8)).copy()
        self.steps.append(words)
        return 0


@pytest.fixture
def library(monkeypatch):
    recorder = Recorder()
    monkeypatch.setattr(linear, "load_library", lambda: recorder)
    monkeypatch.setattr(linear, "_dev", lambda t, dtype, name: t)
    monkeypatch.setattr(linear, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(linear, "_addresses", lambda tensors, sizes, dtype, name: [t.data_ptr() for t in tensors])
    return recorder


@pytest.mark.parametrize("state_bits", [8, 32])
def test_a_step_that_another_one_overtakes_keeps_its_gradients(library, state_bits):
    params = [torch.zeros(n) for n in (3, 300, 1000)]
    mine, others = [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params]
    optimizer = linear.RfsfAdamW(params, state_bits=state_bits)
    library.before = lambda: optimizer.step(others, 1, 1e-3)
    optimizer.step(mine, 1, 1e-3)
    assert [list(words[:, 1]) for words in library.steps] == [[g.data_ptr() for g in others], [g.data_ptr() for g in mine]]
    state = optimizer.state
    for words in library.steps:
        assert list(words[:, 0]) == [p.data_ptr() for p in params] and list(words[:, 7]) == [3, 300, 1000]
        assert list(words[:, 2]) == [t.data_ptr() for t in state["m"]] and list(words[:, 3]) == [t.data_ptr() for t in state["v"]]


@pytest.mark.parametrize("out", [(), ([torch.zeros(3)],), ([torch.zeros(3)], [torch.zeros(3)], [torch.zeros(3)]), ([torch.zeros(3)], []), ([], [torch.zeros(3)])])
def test_moments_are_written_to_two_lists(library, out):
    """Anything else than two lists of a tensor for each parameter is refused, before the library is called (which has no such entry here)."""
    optimizer = linear.RfsfAdamW([torch.zeros(3)], state_bits=8)
    with pytest.raises(ValueError):
        optimizer.moments(out=out)
