"""Every form of the layer norm's kernels (tests/norm_forms.py) against the formulas in 64 bits: rows apart, shifted, in place, far from zero, without variance."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from tests import norm_reference as ref
from tests.norm_forms import BACK, FEW, MANY, MANY_BF16, MANY_ROWS
from tests.test_gpu_layer_norm import TYPES, _beyond, _inputs, _np, _place

pytestmark = pytest.mark.gpu

FORWARD = [(N, K, t) for t in TYPES for N, K in FEW + [(MANY_ROWS, K) for K in MANY + (MANY_BF16 if t == "bfloat16" else [])]]


def _rows(N):
    """The rows that are looked at."""
    return np.unique(np.concatenate([[0, 1, 2, N // 3, N - 2, N - 1], np.random.default_rng(N).integers(0, N, 14)]).clip(0, N - 1))


@pytest.mark.parametrize("far", [0.0, 3e4])
@pytest.mark.parametrize("N,K,dtype", FORWARD)
def test_forward(N, K, dtype, far):
    bf16 = dtype == "bfloat16"
    gen = torch.Generator(device="cuda").manual_seed(N + 7 * K)
    # (numbers of bfloat16 near 3e4 are 128 or more apart)
    x = (torch.randn(N, K, generator=gen, device="cuda") * (1000.0 if bf16 and far else 1.0) + far).to(TYPES[dtype])
    x[N // 3] = far - 123.25
    gain, offset = 1 + 0.3 * torch.randn(K, generator=gen, device="cuda"), 0.3 * torch.randn(K, generator=gen, device="cuda")
    rows = _rows(N)
    x64 = _np(x[rows])
    for p, ld, shift in ((0.0, K, 0), (0.3, K + 3, 1)):
        X, out = _place(x, TYPES[dtype], ld, shift), _place(x, TYPES[dtype], ld + 2)
        drop = rfsf.RfsfDropout(p, seed=K, offset=5, first_row=2) if p else None
        Y, mean, rstd = rfsf.rfsf_layer_norm(X, gain, offset, eps=1e-3, dropout=drop, out=out)
        factor = np.concatenate([ref.mask(1, K, p, K, 5, 2 + int(n)) for n in rows]) if p else np.ones((len(rows), K))
        want = ref.norm(x64, _np(gain), _np(offset), 1e-3, factor)
        bounds = ref.norm_bounds(x64, _np(gain), _np(offset), 1e-3, factor, bf16)
        for name, g, w, t in zip(("mean", "rstd", "Y"), (mean, rstd, Y), want, bounds):
            excess = np.abs(_np(g[rows]) - w) - t
            assert np.all(excess <= 0), (name, p, float(excess.max()))
        assert torch.all(_beyond(Y, ld + 2) == -7.0)
        again = rfsf.rfsf_layer_norm(X, gain, offset, eps=1e-3, dropout=drop, out=X)
        assert again[0] is X and torch.equal(X, Y) and torch.equal(again[1], mean) and torch.equal(again[2], rstd)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", BACK)
def test_backward(dtype, N, K):
    x, gain, _, dy = _inputs(N, K, TYPES[dtype], seed=11)
    for p, ld, shift in ((0.0, K, 0), (0.3, K + 3, 1)):
        X, dY = _place(x, TYPES[dtype], ld, shift), _place(dy, TYPES[dtype], ld, shift)
        drop = rfsf.RfsfDropout(p, seed=K, offset=5, first_row=2) if p else None
        _, mean, rstd = rfsf.rfsf_layer_norm(X, eps=1e-3)
        factor = ref.mask(N, K, p, K, 5, 2) if p else np.ones((N, K))
        args = (_np(x), _np(mean), _np(rstd), _np(gain), _np(dy), factor)
        want, bounds = ref.back(*args), ref.back_bounds(*args, dtype == "bfloat16")
        for need_dX, need_gains in ((True, True), (True, False), (False, True)):
            out = _place(x, TYPES[dtype], ld + 2)
            got = rfsf.rfsf_layer_norm_backward(X, mean, rstd, dY, gain=gain.cuda(), dropout=drop, need_dX=need_dX, need_gains=need_gains, dX=out if need_dX else None)
            for name, g, w, t in zip(("dX", "dgain", "doffset"), got, want, bounds):
                if g is not None:
                    excess = np.abs(_np(g) - w) - t
                    assert np.all(excess <= 0), (name, p, need_dX, need_gains, float(excess.max()))
            if need_dX:
                assert torch.all(_beyond(out, ld + 2) == -7.0)
                for name in ("X", "dY"):
                    a, b = _place(x, TYPES[dtype], ld, shift), _place(dy, TYPES[dtype], ld, shift)
                    again = rfsf.rfsf_layer_norm_backward(a, mean, rstd, b, gain=gain.cuda(), dropout=drop, need_gains=need_gains, dX=a if name == "X" else b)
                    assert all(g is None and w is None or torch.equal(g, w) for g, w in zip(again, got)), name
                    assert torch.all(_beyond(again[0], ld) == -7.0)
