"""Settings of rfsf_adamw_step that the step, which computes in 32 bits, cannot use are refused before anything touches the device; others are not."""
import ctypes

import pytest

from paper_2501_07145_amd import binding, linear

GOOD = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, state_bits=32, grad_bf16=0)


def _step(count=0, **kw):
    config = linear._AdamwConfig(**{**GOOD, **kw})
    return binding.load_library().rfsf_adamw_step(None, count, ctypes.byref(config), None)


@pytest.mark.parametrize("kw", [dict(grad_scale=1e39), dict(grad_scale=-1e39), dict(lr=1e39), dict(eps=1e39), dict(weight_decay=1e39), dict(lr=1e20, weight_decay=1e20),
                                dict(lr=1e38, beta1=0.999), dict(grad_scale=float("-inf")), dict(weight_decay=float("nan")), dict(beta2=float("nan"))])
def test_settings_beyond_32_bits_are_refused(kw):
    assert _step(**kw) == -11


@pytest.mark.parametrize("kw", [dict(lr=0.0), dict(eps=0.0), dict(grad_scale=0.0), dict(grad_scale=-1.0), dict(grad_scale=1e38, lr=1e30, eps=1e38), dict(beta1=0.0, beta2=0.0),
                                dict(step=1 << 62), dict(beta1=1 - 2.0 ** -53, beta2=1 - 2.0 ** -53), dict(lr=1e38, beta1=0.5)])
def test_settings_that_are_used(kw):
    assert _step(**kw) == 0
