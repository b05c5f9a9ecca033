"""Refusals of the scores with adapters, which come before anything touches the device."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from paper_2501_07145_amd import binding, linear
from tests import adapters_reference as ref

SOME = 256          # a pointer that is not NULL and never read


def _shape(**kw):
    base = dict(K=9, C=5, rank=3, count=4, bf16=0)
    base.update(kw)
    return linear._AdaptersShape(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(K=0), -2), (dict(C=0), -2), (dict(rank=0), -2), (dict(count=0), -2), (dict(K=3500001), -9), (dict(C=3500001), -9), (dict(rank=257), -9), (dict(count=131073), -9),
])
def test_shapes_that_are_refused(kw, code):
    lib, s = binding.load_library(), _shape(**kw)
    at = ctypes.byref(s)
    assert lib.rfsf_adapters_layout_bytes(at, None) == code
    assert lib.rfsf_adapters_set_weights(at, SOME, 1 << 30, SOME, None) == code
    assert lib.rfsf_adapters_set(at, 0, SOME, 1 << 30, SOME, 1 << 30, 1.0, SOME, None) == code
    assert lib.rfsf_adapted_scores_workspace_bytes(at, 4, None, None) == code
    assert lib.rfsf_adapted_scores(at, SOME, SOME, 4, 1 << 30, SOME, SOME, 1 << 30, SOME, 1 << 50, None) == code


def test_arguments_of_laying_out():
    lib, s = binding.load_library(), _shape()
    good = [ctypes.byref(s), SOME, 9, SOME, None]
    for at, value, code in [(0, None, -1), (1, None, -1), (3, None, -1), (2, 8, -4), (3, SOME + 16, -4)]:
        args = list(good)
        args[at] = value
        assert lib.rfsf_adapters_set_weights(*args) == code, (at, value)
    good = [ctypes.byref(s), 0, SOME, 9, SOME, 3, 1.0, SOME, None]
    for at, value, code in [(0, None, -1), (1, -1, -2), (1, 4, -2), (2, None, -1), (3, 8, -4), (4, None, -1), (5, 2, -4), (6, float("nan"), -11), (6, 1e60, -11),
                            (7, None, -1), (7, SOME + 16, -4)]:
        args = list(good)
        args[at] = value
        assert lib.rfsf_adapters_set(*args) == code, (at, value)


def test_arguments_of_scores():
    lib, s = binding.load_library(), _shape()
    mn = ctypes.c_size_t(0)
    assert lib.rfsf_adapted_scores_workspace_bytes(ctypes.byref(s), 7, None, ctypes.byref(mn)) == 0 and mn.value > 0
    good = [ctypes.byref(s), SOME, SOME, 7, 9, SOME, SOME, 5, SOME, 1 << 30, None]
    for at, value, code in [(0, None, -1), (1, None, -1), (2, None, -1), (3, -1, -2), (3, 1 << 31, -9), (4, 8, -4), (5, None, -1), (6, None, -1), (7, 4, -4), (8, None, -1),
                            (9, mn.value - 1, -6), (1, SOME + 16, -4)]:
        args = list(good)
        args[at] = value
        assert lib.rfsf_adapted_scores(*args) == code, (at, value)
    assert lib.rfsf_adapted_scores(ctypes.byref(s), None, None, 0, 9, None, None, 5, None, 0, None) == 0


def test_the_smallest_workspace_is_no_larger_than_the_recommended_one():
    rng = np.random.default_rng(1)
    lib = binding.load_library()
    for _ in range(2000):
        N, K, C, rank, count = (int(np.exp(rng.uniform(0, np.log(top)))) for top in (10 ** 7, 12000, 50000, 257, 1000))
        rec, mn = ctypes.c_size_t(0), ctypes.c_size_t(0)
        s = _shape(K=K, C=C, rank=rank, count=count, bf16=int(rng.integers(2)))
        assert lib.rfsf_adapted_scores_workspace_bytes(ctypes.byref(s), N, ctypes.byref(rec), ctypes.byref(mn)) == 0
        assert 0 < mn.value <= rec.value, (N, K, C, rank, count)


def test_binding_refuses_what_it_cannot_pass_on():
    with pytest.raises(ValueError):
        rfsf.RfsfAdapters(torch.zeros(5, 9), 4, 3)


def test_reference_against_merged_weights():
    rng = np.random.default_rng(2)
    X, W, A, B = rng.standard_normal((6, 9)), rng.standard_normal((5, 9)), rng.standard_normal((3, 2, 9)), rng.standard_normal((3, 5, 2))
    adapters, scale = np.array([0, 2, -1, 2, 3, -5]), np.array([0.5, 1.0, -2.0])
    got = ref.scores(X, W, A, B, scale, adapters)
    for n, a in enumerate(adapters):
        if a >= 3:
            assert np.isnan(got[n]).all()
        else:
            merged = W + (scale[a] * B[a] @ A[a] if a >= 0 else 0.0)
            assert np.allclose(got[n], merged @ X[n], rtol=1e-12, atol=1e-12)
