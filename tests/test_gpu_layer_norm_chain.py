"""The backward pass behind the forward pass, of rows far from zero, against gradients in 64 bits whose mean and deviation are not rounded: the backward pass forms z from the
mean that it is given, which is rounded to 32 bits, so that z is off by up to 2^-24 |mean| rstd, and nothing else is."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from tests import norm_reference as ref
from tests.test_gpu_layer_norm import TYPES, _np

pytestmark = pytest.mark.gpu
EPS = 1e-3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("far", [0.0, 40.0, 3e4, 1e7])
@pytest.mark.parametrize("N,K", [(64, 300), (300, 65), (2100, 65), (40, 1025), (333, 5121), (5, 20485)])
def test_gradients_of_what_the_forward_pass_returned(dtype, far, N, K):
    gen = torch.Generator().manual_seed(K)
    spread = max(1.0, far / 64) if dtype == "bfloat16" else max(1.0, far / 2.0 ** 18)          # some steps of the type
    X = (far + spread * torch.randn(N, K, generator=gen, dtype=torch.float64)).to(TYPES[dtype])
    gain, dY = 1 + 0.3 * torch.randn(K, generator=gen), torch.randn(N, K, generator=gen).to(TYPES[dtype])
    _, mean, rstd = rfsf.rfsf_layer_norm(X.cuda(), gain.cuda(), eps=EPS)
    got = rfsf.rfsf_layer_norm_backward(X.cuda(), mean, rstd, dY.cuda(), gain=gain.cuda())
    x, a, d, ones = _np(X), _np(gain), _np(dY), np.ones((N, K))
    exact_mean, exact_rstd, _ = ref.norm(x, a, 0.0, EPS, ones)
    want = ref.back(x, exact_mean, exact_rstd, a, d, ones)
    arithmetic = ref.back_bounds(x, _np(mean), _np(rstd), a, d, ones, dtype == "bfloat16")
    # what the rounded mean and the deviation, off by `share` of itself, make of z, and that of the gradients
    share = (ref.norm_bounds(x, a, 0.0, EPS, ones, False)[1] / exact_rstd)[:, None]
    z = np.abs((x - exact_mean[:, None]) * exact_rstd[:, None])
    off = (2.0 ** -24 * np.abs(exact_mean) * exact_rstd)[:, None] * (1 + share) + share * z
    h, g = np.abs(d), np.abs(d * a)
    of_mean = exact_rstd[:, None] * (off * (g * z).mean(1)[:, None] + (z + off) * (g * off).mean(1)[:, None])
    of_rstd = share * exact_rstd[:, None] * (g + g.mean(1)[:, None] + z * (g * z).mean(1)[:, None])
    for name, v, w, t in zip(("dX", "dgain", "doffset"), got, want, (arithmetic[0] + of_mean + of_rstd, arithmetic[1] + (h * off).sum(0), arithmetic[2])):
        excess = np.abs(_np(v) - w) - t
        assert np.all(excess <= 0), (name, float(excess.max()))
