"""Refusals of the entry points for linear models, which come before anything touches the device, and the formulas that the GPU
tests compare with, against differences."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from paper_2501_07145_amd import binding, linear
from tests.linear_reference import xent

SOME = 256          # a pointer that is not NULL and never read


def _xent_shape(**kw):
    base = dict(N=4, K=9, C=5, ld_phi=9, ld_w=9, ld_dphi=9, ld_dw=9, bf16=0, gradients=3)
    base.update(kw)
    return linear._XentShape(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), -2), (dict(K=0), -2), (dict(C=0), -2), (dict(gradients=4), -2), (dict(ld_phi=8), -4), (dict(ld_w=8), -4),
    (dict(ld_dphi=8), -4), (dict(ld_dw=8), -4), (dict(C=4000001), -9), (dict(K=4000001, ld_phi=4000001, ld_w=4000001, ld_dphi=4000001, ld_dw=4000001), -9),
    (dict(N=1 << 31), -9),
])
def test_xent_shapes_that_are_refused(kw, code):
    lib, shp = binding.load_library(), _xent_shape(**kw)
    assert lib.rfsf_softmax_xent_workspace_bytes(ctypes.byref(shp), None, None) == code
    assert lib.rfsf_softmax_xent(ctypes.byref(shp), SOME, SOME, SOME, None, SOME, SOME, SOME, SOME, 1 << 40, None) == code


def test_xent_strides_of_gradients_that_are_not_asked_for_do_not_matter():
    lib = binding.load_library()
    for gradients in (0, 1, 2):
        shp = _xent_shape(gradients=gradients, ld_dphi=9 if gradients == 1 else 0, ld_dw=9 if gradients == 2 else 0)
        assert lib.rfsf_softmax_xent_workspace_bytes(ctypes.byref(shp), None, None) == 0


@pytest.mark.parametrize("missing", range(8))
def test_xent_pointers(missing):
    lib, shp = binding.load_library(), _xent_shape()
    args = [ctypes.byref(shp), SOME, SOME, SOME, SOME, SOME, SOME, SOME, SOME]
    order = [0, 1, 2, 3, 5, 6, 7, 8]          # all but the weights, which may be NULL
    args[order[missing]] = None
    assert lib.rfsf_softmax_xent(*args, 1 << 40, None) == -1


def test_xent_workspace():
    lib, shp = binding.load_library(), _xent_shape(N=5000, K=1000, C=777, ld_phi=1000, ld_w=1000, ld_dphi=1000, ld_dw=1000)
    rec, mn = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.rfsf_softmax_xent_workspace_bytes(ctypes.byref(shp), ctypes.byref(rec), ctypes.byref(mn)) == 0
    assert 0 < mn.value < rec.value
    assert lib.rfsf_softmax_xent(ctypes.byref(shp), SOME, SOME, SOME, None, SOME, SOME, SOME, SOME, mn.value - 1, None) == -6
    # recommended sizes stay bounded: no room for all scores of a large batch
    assert rfsf.rfsf_softmax_xent_workspace_bytes(1 << 20, 1025, 32768, torch.bfloat16, True, True)[0] < 12 << 30
    # without gradients no scores are held at all
    assert rfsf.rfsf_softmax_xent_workspace_bytes(10000, 65, 50000)[0] < 10000 * 50000


def test_the_smallest_workspace_is_no_larger_than_the_recommended_one():
    rng = np.random.default_rng(1)
    for _ in range(2000):
        N, K, C = (int(np.exp(rng.uniform(0, np.log(top)))) for top in (20000, 12000, 50000))
        rec, least = rfsf.rfsf_softmax_xent_workspace_bytes(N, K, C, (torch.float32, torch.bfloat16)[rng.integers(2)], bool(rng.integers(2)), bool(rng.integers(2)))
        assert 0 < least <= rec, (N, K, C)


def test_no_rows_need_nothing():
    lib = binding.load_library()
    shp = _xent_shape(N=0, gradients=1)
    assert lib.rfsf_softmax_xent(ctypes.byref(shp), None, None, None, None, None, None, None, None, 0, None) == 0
    shp = _xent_shape(N=0, gradients=2)
    assert lib.rfsf_softmax_xent(ctypes.byref(shp), None, None, None, None, None, None, None, None, 0, None) == -1      # dW is cleared


def _config(**kw):
    base = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, state_bits=32, grad_bf16=0)
    base.update(kw)
    return linear._AdamwConfig(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(lr=float("nan")), -11), (dict(lr=-1.0), -11), (dict(beta1=1.0), -11), (dict(beta1=-0.1), -11), (dict(beta2=1.0), -11),
    (dict(eps=-1e-8), -11), (dict(eps=float("inf")), -11), (dict(weight_decay=-0.1), -11), (dict(grad_scale=float("inf")), -11),
    (dict(step=0), -11), (dict(state_bits=16), -9), (dict(state_bits=4), -9),
])
def test_adamw_settings_that_are_refused(kw, code):
    lib, c = binding.load_library(), _config(**kw)
    t = (linear._AdamwTensor * 1)(linear._AdamwTensor(SOME, SOME, SOME, SOME, SOME, SOME, None, 4))
    assert lib.rfsf_adamw_step(ctypes.byref(t), 1, ctypes.byref(c), None) == code


def test_adamw_arguments():
    lib = binding.load_library()
    c32, c8 = _config(), _config(state_bits=8)
    T = linear._AdamwTensor
    assert lib.rfsf_adamw_step(None, 0, None, None) == -1
    assert lib.rfsf_adamw_step(None, 1, ctypes.byref(c32), None) == -1
    assert lib.rfsf_adamw_step(None, -1, ctypes.byref(c32), None) == -2
    assert lib.rfsf_adamw_step(None, 0, ctypes.byref(c32), None) == 0
    for k in range(6):
        fields = [SOME] * 6
        fields[k] = None
        t = (T * 2)(T(None, None, None, None, None, None, None, 0), T(*fields, None, 4))
        assert lib.rfsf_adamw_step(ctypes.byref(t), 2, ctypes.byref(c8), None) == -1
        if k < 4:
            assert lib.rfsf_adamw_step(ctypes.byref(t), 2, ctypes.byref(c32), None) == -1
    t = (T * 1)(T(SOME, SOME, SOME, SOME, SOME, SOME, None, -1))
    assert lib.rfsf_adamw_step(ctypes.byref(t), 1, ctypes.byref(c32), None) == -2
    t[0].n = 1 << 50
    assert lib.rfsf_adamw_step(ctypes.byref(t), 1, ctypes.byref(c32), None) == -9
    t[0].n = 4
    places = (ctypes.c_void_p * 1)(SOME)
    assert lib.rfsf_adamw_moments(ctypes.byref(t), 1, ctypes.byref(places), None, None) == -1
    assert lib.rfsf_adamw_moments(ctypes.byref(t), 1, ctypes.byref(places), ctypes.byref((ctypes.c_void_p * 1)(None)), None) == -1


def test_int8_arguments():
    lib = binding.load_library()
    q, g, w = lib.rfsf_int8_quantize, lib.rfsf_int8_gram, lib.rfsf_int8_gram_workspace_bytes
    assert q(SOME, 0, -1, 9, 9, SOME, 128, SOME, None) == -2
    assert q(SOME, 0, 4, 9, 0, SOME, 128, SOME, None) == -2
    assert q(SOME, 0, 4, 8, 9, SOME, 128, SOME, None) == -4
    assert q(SOME, 0, 4, 9, 9, SOME, 127, SOME, None) == -4
    assert q(SOME, 0, 4, 9, 9, SOME, 136, SOME, None) == -4          # not a multiple of 16
    assert q(SOME, 0, 4, 9, 9, SOME + 8, 128, SOME, None) == -4
    assert q(SOME, 0, 4, 131073, 131073, SOME, 131200, SOME, None) == -9
    for k in (0, 5, 7):
        args = [SOME, 0, 4, 9, 9, SOME, 128, SOME, None]
        args[k] = None
        assert q(*args) == -1
    assert q(None, 0, 0, 9, 9, None, 128, None, None) == 0
    mn = ctypes.c_size_t(0)
    assert w(4, 5, 9, None, ctypes.byref(mn)) == 0
    for kw, code in [((-1, 5, 9), -2), ((4, -5, 9), -2), ((4, 5, 0), -2), ((4, 5, 131073), -9), ((4, 100000001, 9), -9), ((1 << 31, 5, 9), -9)]:
        assert w(*kw, None, None) == code
        assert g(SOME, 0, kw[0], 1 << 20, SOME, SOME, kw[1], 1 << 20, kw[2], SOME, 1 << 30, SOME, 1 << 40, None) == code
    good = [SOME, 0, 4, 9, SOME, SOME, 5, 128, 9, SOME, 5, SOME, 1 << 20, None]
    for at, value, code in [(3, 8, -4), (7, 127, -4), (7, 136, -4), (10, 4, -4), (4, SOME + 4, -4), (0, None, -1), (4, None, -1), (5, None, -1), (9, None, -1),
                            (11, None, -1), (12, mn.value - 1, -6)]:
        args = list(good)
        args[at] = value
        assert g(*args) == code, (at, value)
    for at in (2, 6):
        args = list(good)
        args[at] = 0
        assert g(*args) == 0


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 9)
    with pytest.raises(ValueError):
        rfsf.rfsf_softmax_xent(x, x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        rfsf.rfsf_int8_quantize(x)
    with pytest.raises(ValueError):
        rfsf.RfsfAdamW([x])
    with pytest.raises(ValueError):
        rfsf.RfsfAdamW([], state_bits=16)
    with pytest.raises(ValueError):
        rfsf.rfsf_softmax_xent_workspace_bytes(4, 9, 5, torch.float16)


def test_gradients_of_the_reference_against_differences():
    rng = np.random.default_rng(5)
    N, K, C, h = 6, 4, 5, 1e-6
    x, w, s = rng.standard_normal((N, K)), rng.standard_normal((C, K)), rng.standard_normal(N)
    y = np.array([0, 4, -1, 2, 2, -7])
    total = lambda a, b: float((s * xent(a, b, y, s)["loss"]).sum())          # noqa: E731
    r = xent(x, w, y, s)
    for at in np.ndindex(N, K):
        d = np.zeros_like(x)
        d[at] = h
        assert abs((total(x + d, w) - total(x - d, w)) / (2 * h) - r["dPhi"][at]) < 1e-8
    for at in np.ndindex(C, K):
        d = np.zeros_like(w)
        d[at] = h
        assert abs((total(x, w + d) - total(x, w - d)) / (2 * h) - r["dW"][at]) < 1e-8


@pytest.mark.parametrize("state_bits", [8, 32])
def test_an_optimizer_without_parameters_does_nothing(state_bits):
    optimizer = rfsf.RfsfAdamW([], state_bits=state_bits)
    optimizer.step([], step=1, lr=1e-3)
    assert optimizer.params == [] and optimizer.state["m"] == []
    with pytest.raises(ValueError):
        optimizer.step([torch.zeros(3)], step=2, lr=1e-3)
