"""Layer norm of finite rows near the end of the range of 32 bits, in every kind of kernel: a row without variance is its offset whatever its size, and one
whose squares are beyond 32 bits has a deviation of infinity (rstd 0), the offset as result and a gradient of zero."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from tests import norm_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
EPS = 1e-5


def _np(t):
    return t.double().cpu().numpy()


def _forward(rows, N):
    """gain, offset, and the results for N rows, those of `rows` again and again."""
    K = rows.shape[1]
    gen = torch.Generator().manual_seed(K)
    gain, offset = 1 + 0.3 * torch.randn(K, generator=gen), 0.3 * torch.randn(K, generator=gen)
    at = torch.arange(N) % len(rows)
    return (gain, offset, at) + rfsf.rfsf_layer_norm(rows.cuda()[at.cuda()], gain.cuda(), offset.cuda(), eps=EPS)


def _no_variance(rows, offset, at, Y, mean, rstd):
    """Rows of one number: mean and result are exact, the deviation is that of eps alone (a root and a quotient, each rounded, and eps itself)."""
    assert torch.equal(mean.cpu(), rows[:, 0].float()[at])
    assert np.all(np.abs(_np(rstd) - EPS ** -0.5) <= 4 * ref.U * EPS ** -0.5)
    assert torch.equal(Y.cpu(), offset.to(Y.dtype).expand(len(at), -1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(9, 8), (9, 64), (9, 1024), (9, 8192), (2100, 8), (2100, 64), (2100, 128), (2100, 1024), (2061, 4096), (2061, 16384), (5, 32768)])
def test_sums_of_large_numbers(dtype, N, K):
    """Numbers that fit, whose sums would not (K is a power of two, so that means are exact)."""
    values = [2.0 ** 125, -2.0 ** 126, float(torch.finfo(TYPES[dtype]).max), 2.0 ** 64, 1.0]
    rows = torch.tensor(values, dtype=torch.float64)[:, None].expand(-1, K).to(TYPES[dtype])
    gain, offset, at, *out = _forward(rows, N)
    _no_variance(rows, offset, at, *out)
    if K > 8:           # the sum of the first eight is 2^128
        rows = torch.zeros(2, K, dtype=TYPES[dtype])
        rows[0, :8], rows[1, -8:] = 2.0 ** 125, -2.0 ** 125
        gain, offset, at, Y, mean, rstd = _forward(rows, N)
        assert torch.equal(mean.cpu(), torch.tensor([2.0 ** 128 / K, -2.0 ** 128 / K])[at])
        assert not rstd.any() and torch.equal(Y.cpu(), offset.to(Y.dtype).expand(N, -1))
