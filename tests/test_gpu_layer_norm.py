"""Layer norm with dropout and its backward pass against the formulas in 64 bits, within bounds that follow from the arithmetic."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from tests import norm_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
SHAPES = [(1, 1), (1, 2), (3, 7), (5, 64), (2, 65), (4, 128), (4, 129), (3, 256), (3, 257), (5, 512), (9, 513), (6, 1024), (7, 1025), (3, 2049), (5, 4097), (3, 6145),
          (2, 8193), (3, 12289), (2, 16385), (2, 20480), (2, 20481), (1, 50001), (1500, 65), (300, 193), (40, 1001), (2100, 129), (1300, 300), (1030, 2051), (300, 5121), (700, 9003), (2049, 4099), (5000, 3), (9000, 1), (4000, 7)]


def _place(x, dtype, ld, shift=0):
    N, K = x.shape
    buf = torch.full((shift + N * ld + 8,), -7.0, dtype=dtype, device="cuda")
    view = buf[shift:shift + N * ld].view(N, ld)[:, :K]
    view.copy_(x)
    return view


def _beyond(view, ld):
    """What lies between and around the rows."""
    N, K = view.shape
    rows = view._base[view.storage_offset():view.storage_offset() + N * ld].view(N, ld)
    return torch.cat([rows[:, K:].flatten(), view._base[:view.storage_offset()], view._base[view.storage_offset() + N * ld:]])


def _inputs(N, K, dtype, seed=0, far=0.0):
    gen = torch.Generator().manual_seed(1000 * seed + 31 * N + K)
    x = torch.randn(N, K, generator=gen, dtype=torch.float64) * 10 ** torch.randn(N, 1, generator=gen, dtype=torch.float64) + far
    gain = 1 + 0.3 * torch.randn(K, generator=gen)
    offset = 0.3 * torch.randn(K, generator=gen)
    dy = torch.randn(N, K, generator=gen)
    return x.to(dtype), gain, offset, dy.to(dtype)


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", SHAPES)
def test_forward(dtype, N, K):
    bf16 = dtype == "bfloat16"
    x, gain, offset, _ = _inputs(N, K, TYPES[dtype])
    for ld, shift, p, affine in ((K, 0, 0.0, True), (K + 3, 1, 0.3, True), ((K + 7) // 8 * 8, 0, 0.2, False)):
        X, out = _place(x, TYPES[dtype], ld, shift), _place(x, TYPES[dtype], ld + 2)
        drop = rfsf.RfsfDropout(p, seed=K, offset=5, first_row=2) if p else None
        Y, mean, rstd = rfsf.rfsf_layer_norm(X, gain.cuda() if affine else None, offset.cuda() if affine else None, eps=1e-3, dropout=drop, out=out)
        factor = ref.mask(N, K, p, K, 5, 2) if p else np.ones((N, K))
        a, b = (_np(gain), _np(offset)) if affine else (1.0, 0.0)
        want = ref.norm(_np(x), a, b, 1e-3, factor)
        bounds = ref.norm_bounds(_np(x), a, b, 1e-3, factor, bf16)
        for name, g, w, t in zip(("mean", "rstd", "Y"), (mean, rstd, Y), want, bounds):
            excess = np.abs(_np(g) - w) - t
            assert np.all(excess <= 0), (name, ld, float(excess.max()))
        assert torch.all(_beyond(Y, ld + 2) == -7.0) and np.all(_np(Y)[factor == 0] == 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [5130, 7171, 8192, 10239, 10300, 12289, 13001, 14336, 14343, 15361, 16384, 16391, 16400])
def test_forward_of_many_long_rows(dtype, K):
    """Some of the rows against the formula, for every number of columns that lanes hold."""
    x, gain, offset, _ = _inputs(5, K, TYPES[dtype])
    rows = [0, 1, 777, 2047, 2052]
    X = torch.zeros(2053, K, dtype=TYPES[dtype], device="cuda")
    X[rows] = x.cuda()
    Y, mean, rstd = rfsf.rfsf_layer_norm(X, gain.cuda(), offset.cuda(), eps=1e-3, dropout=rfsf.RfsfDropout(0.3, seed=K, offset=7, first_row=3))
    factor = np.concatenate([ref.mask(1, K, 0.3, K, 7, 3 + n) for n in rows])
    want = ref.norm(_np(x), _np(gain), _np(offset), 1e-3, factor)
    bounds = ref.norm_bounds(_np(x), _np(gain), _np(offset), 1e-3, factor, dtype == "bfloat16")
    for name, g, w, t in zip(("mean", "rstd", "Y"), (mean, rstd, Y), want, bounds):
        excess = np.abs(_np(g[rows]) - w) - t
        assert np.all(excess <= 0), (name, float(excess.max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", SHAPES)
def test_backward(dtype, N, K):
    bf16 = dtype == "bfloat16"
    x, gain, offset, dy = _inputs(N, K, TYPES[dtype], seed=1)
    for ld, shift, p, affine, need_dX, need_gains in ((K, 0, 0.0, True, True, True), (K + 3, 1, 0.3, True, True, True), ((K + 7) // 8 * 8, 0, 0.2, True, False, True),
                                                     (K, 0, 0.0, False, False, True), (K + 1, 0, 0.25, False, True, False), (K, 0, 0.0, True, True, False)):
        X, dY, out = _place(x, TYPES[dtype], ld, shift), _place(dy, TYPES[dtype], ld + 1), _place(x, TYPES[dtype], ld + 2)
        drop = rfsf.RfsfDropout(p, seed=K, offset=5, first_row=2) if p else None
        gain_ = gain.cuda() if affine else None
        _, mean, rstd = rfsf.rfsf_layer_norm(X, gain_, None, eps=1e-3, dropout=drop)
        got = rfsf.rfsf_layer_norm_backward(X, mean, rstd, dY, gain=gain_, dropout=drop, need_dX=need_dX, need_gains=need_gains, dX=out if need_dX else None)
        factor = ref.mask(N, K, p, K, 5, 2) if p else np.ones((N, K))
        a = _np(gain) if affine else 1.0
        want = ref.back(_np(x), _np(mean), _np(rstd), a, _np(dy), factor)
        bounds = ref.back_bounds(_np(x), _np(mean), _np(rstd), a, _np(dy), factor, bf16)
        assert (got[0] is None) == (not need_dX) and (got[1] is None) == (got[2] is None) == (not need_gains)
        for name, g, w, t in zip(("dX", "dgain", "doffset"), got, want, bounds):
            if g is not None:
                excess = np.abs(_np(g) - w) - t
                assert np.all(excess <= 0), (name, ld, p, float(excess.max()))
        if need_dX:
            assert torch.all(_beyond(out, ld + 2) == -7.0)


@pytest.mark.parametrize("K", [1, 5, 65, 300, 1025, 9001, 20485])
def test_rows_far_from_zero_and_rows_without_variance(K):
    x, gain, offset, _ = _inputs(6, K, torch.float32, seed=2, far=3e4)
    x[4], x[5] = 123.25, 0.0
    Y, mean, rstd = rfsf.rfsf_layer_norm(x.cuda(), gain.cuda(), offset.cuda(), eps=1e-5)
    want, bounds = ref.norm(_np(x), _np(gain), _np(offset), 1e-5, np.ones((6, K))), ref.norm_bounds(_np(x), _np(gain), _np(offset), 1e-5, np.ones((6, K)), False)
    for g, w, t in zip((mean, rstd, Y), want, bounds):
        assert np.all(np.abs(_np(g) - w) <= t)
    assert torch.equal(Y[5].cpu(), offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [9, 300, 1025, 9001, 20485])
def test_infinities_and_nan_stay_in_their_rows(dtype, K):
    x, gain, offset, dy = _inputs(7, K, TYPES[dtype], seed=3)
    X, dY, gain, offset = x.cuda(), dy.cuda(), gain.cuda(), offset.cuda()
    drop = rfsf.RfsfDropout(0.5, 11)
    good = rfsf.rfsf_layer_norm(X, gain, offset, dropout=drop)
    good_dX = rfsf.rfsf_layer_norm_backward(X, good[1], good[2], dY, gain=gain, dropout=drop)[0]
    bad = X.clone()
    bad[2, K // 2], bad[5, 0] = float("inf"), float("nan")
    Y, mean, rstd = rfsf.rfsf_layer_norm(bad, gain, offset, dropout=drop)
    dX, dgain, doffset = rfsf.rfsf_layer_norm_backward(bad, mean, rstd, dY, gain=gain, dropout=drop)
    kept = torch.from_numpy(ref.mask(7, K, 0.5, 11) != 0).cuda()
    for n in range(7):
        if n in (2, 5):
            assert torch.equal(Y[n].isnan(), kept[n]) and bool(dX[n].isnan().all())
        else:
            assert torch.equal(Y[n], good[0][n]) and torch.equal(dX[n], good_dX[n]) and torch.equal(mean[n], good[1][n])
    assert bool(dgain.isnan().all()) and not bool(doffset.isnan().any())
    # gradients of what dropout left out do not matter
    holes = torch.where(kept, dY, torch.full_like(dY, float("nan")))
    assert torch.equal(rfsf.rfsf_layer_norm_backward(X, good[1], good[2], holes, gain=gain, dropout=drop)[0], good_dX)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [7, 2100])
@pytest.mark.parametrize("K", [3, 65, 1025, 20485])
def test_statistics_of_rows_with_infinities_and_nan(dtype, N, K):
    """The mean is what the sum gives, the deviation is NaN and not that of a row without variance; the other rows have theirs."""
    if N * K > 1 << 22:
        N = 2050
    x = torch.ones(N, K, dtype=TYPES[dtype], device="cuda")
    x[:, 0] = 5.0
    x[1, 1], x[2, K - 1], x[4, 0] = float("inf"), float("nan"), -float("inf")
    _, mean, rstd = rfsf.rfsf_layer_norm(x)
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[[1, 2, 4]] = True
    assert torch.equal(rstd.isnan(), bad) and torch.equal(mean.isfinite(), ~bad)
    assert mean[1] == float("inf") and mean[4] == -float("inf") and mean[2].isnan()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(30, 65), (9, 1025), (7, 10241), (5, 20489)])
def test_in_place(dtype, N, K):
    x, gain, offset, dy = (t.cuda() for t in _inputs(N, K, TYPES[dtype], seed=4))
    drop = rfsf.RfsfDropout(0.2, 3)
    Y, mean, rstd = rfsf.rfsf_layer_norm(x, gain, offset, dropout=drop)
    y = x.clone()
    assert torch.equal(rfsf.rfsf_layer_norm(y, gain, offset, dropout=drop, out=y)[0], Y) and torch.equal(y, Y)
    want = rfsf.rfsf_layer_norm_backward(x, mean, rstd, dy, gain=gain, dropout=drop)
    for name in ("X", "dY"):
        a, b = x.clone(), dy.clone()
        got = rfsf.rfsf_layer_norm_backward(a, mean, rstd, b, gain=gain, dropout=drop, dX=a if name == "X" else b)
        assert all(torch.equal(g, w) for g, w in zip(got, want)), name


def test_no_rows():
    x = torch.zeros(0, 17, device="cuda")
    Y, mean, rstd = rfsf.rfsf_layer_norm(x)
    assert Y.shape == (0, 17) and mean.shape == rstd.shape == (0,)
    dgain, doffset = torch.ones(17, device="cuda"), torch.ones(17, device="cuda")
    rfsf.rfsf_layer_norm_backward(x, mean, rstd, x, dgain=dgain, doffset=doffset)
    assert not dgain.any() and not doffset.any()


def test_equal_calls_give_equal_bits_and_graphs_replay():
    x, gain, offset, dy = (t.cuda() for t in _inputs(700, 1025, torch.float32, seed=5))
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = rfsf.RfsfDropout(0.3, 17, counter=counter)
    need = rfsf.rfsf_layer_norm_backward_workspace_bytes(700, 1025)[0]
    spaces = [torch.empty(need + 17, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out, mean, rstd = torch.empty_like(x), torch.empty(700, device="cuda"), torch.empty(700, device="cuda")
    dX, dgain, doffset = torch.empty_like(x), torch.empty(1025, device="cuda"), torch.empty(1025, device="cuda")

    def both(space, d):
        rfsf.rfsf_layer_norm(x, gain, offset, dropout=d, out=out, mean=mean, rstd=rstd)
        rfsf.rfsf_layer_norm_backward(x, mean, rstd, dy, gain=gain, dropout=d, dX=dX, dgain=dgain, doffset=doffset, workspace=space)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(spaces[0], drop)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(spaces[0], drop)
        counter.add_(1)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        results = [t.clone() for t in (out, mean, rstd, dX, dgain, doffset)]
        for t in (out, mean, rstd, dX, dgain, doffset):
            t.zero_()
        both(spaces[1][17:], rfsf.RfsfDropout(0.3, 17, offset=step))          # (a workspace that is not aligned)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, (out, mean, rstd, dX, dgain, doffset)))


def test_many_rows_beyond_two_to_the_31_numbers():
    N, K = 140000, 16001
    x = torch.empty(N, K, dtype=torch.bfloat16, device="cuda").normal_()
    Y, mean, rstd = rfsf.rfsf_layer_norm(x)
    dX, dgain, doffset = rfsf.rfsf_layer_norm_backward(x, mean, rstd, Y, need_dX=False)
    assert dX is None
    at = [0, 1, N // 2, N - 1]
    want, bounds = ref.norm(_np(x[at]), 1.0, 0.0, 1e-5, 1.0), ref.norm_bounds(_np(x[at]), 1.0, 0.0, 1e-5, np.ones((4, K)), True)
    for g, w, t in zip((mean[at], rstd[at], Y[at]), want, bounds):
        assert np.all(np.abs(_np(g) - w) <= t)
    columns = [0, 8000, K - 1]
    z = (x[:, columns].double() - mean.double()[:, None]) * rstd.double()[:, None]
    h = Y[:, columns].double()
    bound = (128 + N // 128 + 6) * ref.U
    assert bool(((dgain[columns] - (h * z).sum(0)).abs() <= bound * (h * z).abs().sum(0)).all())
    assert bool(((doffset[columns] - h.sum(0)).abs() <= bound * h.abs().sum(0)).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_a_graph_whose_first_call_is_captured(dtype):
    # columns whose gains and offsets need more LDS than a kernel may have without being allowed to
    x, gain, offset, dy = (t.cuda() for t in _inputs(2050, 9217, TYPES[dtype], seed=6))
    Y, mean, rstd = torch.empty_like(x), torch.empty(2050, device="cuda"), torch.empty(2050, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rfsf.rfsf_layer_norm(x, gain, offset, dropout=rfsf.RfsfDropout(0.1, 4), out=Y, mean=mean, rstd=rstd)
    for _ in range(3):
        Y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = rfsf.rfsf_layer_norm(x, gain, offset, dropout=rfsf.RfsfDropout(0.1, 4))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((Y, mean, rstd), eager))


def test_everything_left_out():
    x, gain, offset, dy = (t.cuda() for t in _inputs(40, 300, torch.float32, seed=7))
    drop = rfsf.RfsfDropout(1.0, 4)
    Y, mean, rstd = rfsf.rfsf_layer_norm(x, gain, offset, dropout=drop)
    assert not Y.any() and bool(rstd.isfinite().all())
    assert all(not g.any() for g in rfsf.rfsf_layer_norm_backward(x, mean, rstd, dy, gain=gain, dropout=drop))


def test_two_streams_at_once():
    inputs = [[t.cuda() for t in _inputs(N, 1025, torch.float32, seed=8)] for N in (500, 3000)]
    want = []
    for x, gain, offset, dy in inputs:
        Y, mean, rstd = rfsf.rfsf_layer_norm(x, gain, offset)
        want.append((mean, rstd, rfsf.rfsf_layer_norm_backward(x, mean, rstd, dy, gain=gain)))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[rfsf.rfsf_layer_norm_backward(x, mean, rstd, dy, gain=gain, stream=s) for _ in range(5)]
           for (x, gain, offset, dy), (mean, rstd, _), s in zip(inputs, want, streams)]
    torch.cuda.synchronize()
    for (_, _, w), results in zip(want, got):
        assert all(torch.equal(a, b) for r in results for a, b in zip(r, w))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("need_dX", [True, False])
@pytest.mark.parametrize("N,K", [(1, 5), (16, 193), (70, 9), (300, 129), (1000, 257), (333, 5121), (90, 10241), (2000, 2049), (40, 20485), (5000, 65)])
def test_nothing_is_written_beyond_the_workspace(dtype, need_dX, N, K):
    x, gain, _, dy = (t.cuda() for t in _inputs(N, K, TYPES[dtype], seed=9))
    _, mean, rstd = rfsf.rfsf_layer_norm(x, gain)
    size = rfsf.rfsf_layer_norm_backward_workspace_bytes(N, K, TYPES[dtype], need_dX)[1]
    for shift in (0, 9):
        space = torch.full((size + shift + 4096,), 77, dtype=torch.uint8, device="cuda")
        got = rfsf.rfsf_layer_norm_backward(x, mean, rstd, dy, gain=gain, need_dX=need_dX, workspace=space[shift:shift + size])
        assert torch.all(space[shift + size:] == 77) and torch.all(space[:shift] == 77)
        assert all(g is None or bool(g.isfinite().all()) for g in got)


def test_binding_refuses_shapes_that_do_not_fit():
    x = torch.zeros(4, 9, device="cuda")
    v = torch.zeros(9, device="cuda")
    n = torch.zeros(4, device="cuda")
    for kw in (dict(gain=v[:8]), dict(offset=v.double()), dict(out=x[:3]), dict(out=x.bfloat16()), dict(mean=v), dict(rstd=n.double())):
        with pytest.raises(ValueError):
            rfsf.rfsf_layer_norm(x, **kw)
    for kw in (dict(gain=v[:8]), dict(dX=x[:, :8]), dict(dgain=n), dict(doffset=v.bfloat16()), dict(workspace=v)):
        with pytest.raises(ValueError):
            rfsf.rfsf_layer_norm_backward(x, n, n, x, **kw)
    with pytest.raises(ValueError):
        rfsf.rfsf_layer_norm_backward(x, n, n, x.bfloat16())
    with pytest.raises(ValueError):
        rfsf.rfsf_layer_norm_backward(x, None, n, x)
