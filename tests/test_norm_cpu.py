"""Refusals of layer norm and dropout, which come before anything touches the device, and the formulas that the GPU tests compare
with: published numbers of the generator, gradients against differences."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from paper_2501_07145_amd import binding, linear
from tests import norm_reference as ref

SOME = 256          # a pointer that is not NULL and never read


def test_generator_against_published_numbers():
    # the known answers of the generator's authors for Philox 4x32, 10 rounds
    for counter, key, want in [
        ([0, 0, 0, 0], [0, 0], [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
        ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
        ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]),
    ]:
        assert ref.philox(np.array(counter, dtype=np.uint64), key).tolist() == want


def test_numbers_of_rows_worked_on_in_parts_are_those_of_the_whole():
    whole = ref.numbers(9, 21, seed=77 << 40, offset=5 << 33)
    assert np.array_equal(whole[4:], ref.numbers(5, 21, seed=77 << 40, offset=5 << 33, first_row=4))
    assert np.array_equal(whole[:, :11], ref.numbers(9, 11, seed=77 << 40, offset=5 << 33))
    assert 0 <= whole.min() and whole.max() < 65536


def _mask(**kw):
    base = dict(p=0.5, seed=1, offset=2, offset_on_device=None, first_row=0)
    base.update(kw)
    return linear._DropoutMask(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(p=-0.01), -11), (dict(p=1.01), -11), (dict(p=float("nan")), -11), (dict(first_row=-1), -2), (dict(first_row=(1 << 32) - 3), -9),
])
def test_masks_that_are_refused(kw, code):
    lib, m = binding.load_library(), _mask(**kw)
    assert lib.rfsf_dropout(ctypes.byref(m), SOME, 0, 4, 9, 9, SOME, 9, None) == code
    shape = linear._LayerNormShape(4, 9, 9, 9, 9, 0)
    assert lib.rfsf_layer_norm(ctypes.byref(shape), SOME, None, None, 1e-5, ctypes.byref(m), SOME, SOME, SOME, None) == code
    assert lib.rfsf_layer_norm_backward(ctypes.byref(shape), SOME, SOME, SOME, None, SOME, ctypes.byref(m), SOME, SOME, SOME, SOME, 1 << 30, None) == code


def test_dropout_arguments():
    lib, m = binding.load_library(), _mask()
    good = [ctypes.byref(m), SOME, 0, 4, 9, 9, SOME, 9, None]
    for at, value, code in [(0, None, -1), (1, None, -1), (6, None, -1), (3, -1, -2), (5, 0, -2), (4, 8, -4), (7, 8, -4), (3, 1 << 31, -9)]:
        args = list(good)
        args[at] = value
        assert lib.rfsf_dropout(*args) == code, (at, value)
    args = [ctypes.byref(m), SOME, 0, 4, 3500001, 3500001, SOME, 3500001, None]
    assert lib.rfsf_dropout(*args) == -9
    assert lib.rfsf_dropout(ctypes.byref(m), None, 0, 0, 9, 9, None, 9, None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), -2), (dict(K=0), -2), (dict(ld_x=8), -4), (dict(ld_y=8), -4), (dict(ld_dx=8), -4), (dict(N=1 << 31), -9),
    (dict(K=3500001, ld_x=3500001, ld_y=3500001, ld_dx=3500001), -9),
])
def test_norm_shapes_that_are_refused(kw, code):
    lib = binding.load_library()
    base = dict(N=4, K=9, ld_x=9, ld_y=9, ld_dx=9, bf16=0)
    base.update(kw)
    s = linear._LayerNormShape(**base)
    if "ld_dx" not in kw or len(kw) > 1:
        assert lib.rfsf_layer_norm(ctypes.byref(s), SOME, SOME, SOME, 1e-5, None, SOME, SOME, SOME, None) == code
    assert lib.rfsf_layer_norm_backward_workspace_bytes(ctypes.byref(s), 1, None, None) == code
    assert lib.rfsf_layer_norm_backward(ctypes.byref(s), SOME, SOME, SOME, SOME, SOME, None, SOME, SOME, SOME, SOME, 1 << 40, None) == code


def test_norm_arguments():
    lib = binding.load_library()
    s = linear._LayerNormShape(4, 9, 9, 9, 0, 0)
    for eps in (0.0, -1e-5, float("nan"), float("inf"), 1e-60, 1e60):
        assert lib.rfsf_layer_norm(ctypes.byref(s), SOME, SOME, SOME, eps, None, SOME, SOME, SOME, None) == -11
    for at in (0, 1, 6):
        args = [ctypes.byref(s), SOME, None, None, 1e-5, None, SOME, None, None, None]
        args[at] = None
        assert lib.rfsf_layer_norm(*args) == -1
    s.N = 0
    assert lib.rfsf_layer_norm(ctypes.byref(s), None, None, None, 1e-5, None, None, None, None, None) == 0
    assert lib.rfsf_layer_norm_backward(ctypes.byref(s), None, None, None, None, None, None, None, None, None, None, 0, None) == 0


def test_backward_arguments():
    lib = binding.load_library()
    s = linear._LayerNormShape(4, 9, 9, 9, 9, 0)
    mn = ctypes.c_size_t(0)
    assert lib.rfsf_layer_norm_backward_workspace_bytes(ctypes.byref(s), 1, None, ctypes.byref(mn)) == 0 and mn.value > 0
    good = [ctypes.byref(s), SOME, SOME, SOME, None, SOME, None, SOME, SOME, SOME, SOME, 1 << 20, None]
    for at, value, code in [(0, None, -1), (1, None, -1), (2, None, -1), (3, None, -1), (5, None, -1), (8, None, -1), (9, None, -1), (10, None, -1),
                            (11, mn.value - 1, -6)]:
        args = list(good)
        args[at] = value
        assert lib.rfsf_layer_norm_backward(*args) == code, (at, value)
    # nothing is asked for
    assert lib.rfsf_layer_norm_backward(ctypes.byref(s), None, None, None, None, None, None, None, None, None, None, 0, None) == 0


def test_workspaces_stay_small():
    for N in (1, 100, 10 ** 6, 10 ** 9):
        for K in (1, 65, 1025, 20480, 20481, 1000003):
            for need_dX in (False, True):
                rec, least = rfsf.rfsf_layer_norm_backward_workspace_bytes(N, K, need_dX=need_dX)
                assert 8 * K <= least <= rec <= 8 * ((K + 7) // 8 * 8) * 1024 + 256           # at most 1024 parts, of rows rounded up to eight


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 9)
    with pytest.raises(ValueError):
        rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.5, 1))
    with pytest.raises(ValueError):
        rfsf.rfsf_layer_norm(x)
    with pytest.raises(ValueError):
        rfsf.rfsf_layer_norm_backward(x, x[:, 0], x[:, 0], x)
    with pytest.raises(ValueError):
        rfsf.rfsf_layer_norm_backward_workspace_bytes(4, 9, torch.float16)
    for kw in (dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(seed=-1), dict(seed=1 << 64), dict(offset=-1), dict(offset=1 << 64),
               dict(first_row=-1), dict(first_row=1 << 32), dict(counter=torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(ValueError):
            rfsf.RfsfDropout(**{**dict(p=0.5, seed=1), **kw})


def test_gradients_of_the_reference_against_differences():
    rng = np.random.default_rng(3)
    N, K, h, eps = 5, 7, 1e-6, 1e-3
    X, gain, offset, dY = rng.standard_normal((N, K)), rng.standard_normal(K), rng.standard_normal(K), rng.standard_normal((N, K))
    factor = ref.mask(N, K, 0.4, seed=9)

    def total(x, a, b):
        return float((dY * ref.norm(x, a, b, eps, factor)[2]).sum())

    mean, rstd, _ = ref.norm(X, gain, offset, eps, factor)
    dX, dgain, doffset = ref.back(X, mean, rstd, gain, dY, factor)
    for at in np.ndindex(N, K):
        d = np.zeros_like(X)
        d[at] = h
        assert abs((total(X + d, gain, offset) - total(X - d, gain, offset)) / (2 * h) - dX[at]) < 1e-7
    for k in range(K):
        d = np.zeros(K)
        d[k] = h
        assert abs((total(X, gain + d, offset) - total(X, gain - d, offset)) / (2 * h) - dgain[k]) < 1e-8
        assert abs((total(X, gain, offset + d) - total(X, gain, offset - d)) / (2 * h) - doffset[k]) < 1e-8
