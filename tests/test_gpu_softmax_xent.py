"""Softmax cross entropy and its gradients on the GPU against 64 bits, elementwise, within the bounds of the stated arithmetic."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from paper_2501_07145_amd import workloads as wl
from tests.linear_reference import xent, xent_bounds

pytestmark = pytest.mark.gpu


def _inputs(N, K, C, bf16, seed=0, left=0.2, pad=3):
    gen = torch.Generator().manual_seed(seed)
    dtype = torch.bfloat16 if bf16 else torch.float32
    phi = (torch.randn(N, K + pad, generator=gen) / K ** 0.5).to(dtype)
    w = (torch.randn(C, K + pad, generator=gen) * 2).to(dtype)
    y = torch.randint(0, C, (N,), generator=gen)
    y[torch.rand(N, generator=gen) < left] = -1
    s = torch.randn(N, generator=gen)
    return phi.cuda()[:, :K], w.cuda()[:, :K], y.cuda(), s.cuda()


def _np(t):
    return t.detach().double().cpu().numpy()


def _scale(y, s):
    return _np(s) if s is not None else np.full(len(y), 1.0 / max(1, int((y >= 0).sum())))


def _check(phi, w, y, s, got):
    bf16 = phi.dtype == torch.bfloat16
    clean = torch.where((y >= 0)[:, None], phi, torch.zeros((), dtype=phi.dtype, device=phi.device))
    scale = _scale(y, None if s is None else torch.where(y >= 0, s, torch.zeros_like(s)))
    r = xent(_np(clean), _np(w), _np(y).astype(np.int64), scale)
    for name, have, bound in zip(("loss", "dPhi", "dW"), got, xent_bounds(r, bf16)):
        if have is not None:
            off = np.abs(_np(have) - r[name])
            assert np.all(off <= bound), (name, float(np.nanmax(off / bound)), int(np.isnan(off).sum()))


SIZES = [(1, 1, 1), (1, 5, 2), (3, 33, 7), (16, 193, 10), (64, 64, 64), (65, 65, 65), (40, 31, 129), (129, 127, 300), (257, 300, 1000),
         (300, 70, 4097), (1000, 129, 31), (2, 2049, 513), (700, 50, 32), (130, 1001, 10), (1, 1000, 33), (513, 64, 16),
         # every way of making the scores and the gradients: few rows, few classes, a long sum cut, many classes, packed operands
         (5, 70, 9000), (16, 300, 17), (17, 300, 17), (9, 131, 9), (3000, 66, 16), (40, 2051, 40), (33, 2100, 70), (20, 5000, 63), (2100, 40, 50), (40, 33, 9000), (19, 20, 30000),
         (620, 300, 600), (530, 291, 777)]
# rows, columns, classes: by the ways above, the last one packed
WAYS = [(90, 40, 20), (90, 40, 300), (12, 40, 300), (300, 40, 7), (620, 300, 600)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,K,C", SIZES)
def test_against_64_bits(N, K, C, bf16):
    phi, w, y, s = _inputs(N, K, C, bf16)
    _check(phi, w, y, s, rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True))
    _check(phi, w, y, None, rfsf.rfsf_softmax_xent(phi, w, y, need_dPhi=True, need_dW=True))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("need_dPhi,need_dW", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("N,K,C", [(150, 70, 10), (150, 70, 200), (15, 70, 200), (620, 300, 600)])
def test_what_is_not_asked_for(N, K, C, bf16, need_dPhi, need_dW):
    phi, w, y, s = _inputs(N, K, C, bf16)
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=need_dPhi, need_dW=need_dW)
    assert (dPhi is not None) == need_dPhi and (dW is not None) == need_dW
    _check(phi, w, y, s, (loss, dPhi, dW))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,K,C", [(700, 1, 900), (700, 64, 901), (701, 1023, 900), (900, 1024, 701), (600, 1025, 702), (330, 4096, 600), (331, 4097, 601), (300, 12288, 500),
                                   (301, 12289, 500)])
def test_losses_of_packed_operands(N, K, C, bf16):
    """Widths around those that are packed in each way; rows that are left out hold anything."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    phi[y < 0] = float("nan")
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s)
    assert dPhi is None and dW is None
    _check(phi, w, y, s, (loss, None, None))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("need_dPhi,need_dW", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("N,K,C", [(1, 4, 1), (2, 5, 3), (7, 3, 2), (17, 255, 4), (130, 256, 5), (129, 257, 8), (701, 514, 9), (2100, 1025, 16), (300, 2047, 16),
                                   (301, 2048, 4), (300, 2049, 16), (9001, 67, 3), (8193, 130, 12), (5000, 1001, 10)])
def test_few_classes(N, K, C, need_dPhi, need_dW, weighted, bf16):
    """Widths around those that one, two, four and eight wavefronts share, rows that are counted in each way."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    s = s if weighted else None
    _check(phi, w, y, s, rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=need_dPhi, need_dW=need_dW))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("N,K,C", [(200, 40, 20), (450, 70, 300), (620, 300, 600), (1500, 170, 900)])
def test_the_smallest_workspace(N, K, C, bf16, weighted):
    """Blocks of 64 rows: dW is added up over them."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    s = s if weighted else None
    _, least = rfsf.rfsf_softmax_xent_workspace_bytes(N, K, C, phi.dtype, True, True)
    workspace = torch.full((least,), 255, dtype=torch.uint8, device="cuda")
    _check(phi, w, y, s, rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True, workspace=workspace))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("need_dPhi,need_dW", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("N,K,C", [(3000, 130, 150), (150, 130, 3000), (2501, 259, 210), (5000, 67, 1300)])
@pytest.mark.parametrize("share", [1.0, 0.4])
def test_long_sums_of_few_tiles(N, K, C, share, need_dPhi, need_dW, bf16):
    """Gradients whose sums are cut into parts; with less workspace, of blocks of rows that add to those before."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    most, least = rfsf.rfsf_softmax_xent_workspace_bytes(N, K, C, phi.dtype, need_dPhi, need_dW)
    size = max(least, int(share * most))
    guard = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    _check(phi, w, y, s, rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=need_dPhi, need_dW=need_dW, workspace=guard[:size]))
    assert torch.all(guard[size:] == 255)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,K,C", [(130, 40, 20), (130, 40, 300), (14, 40, 300), (300, 40, 7), (620, 300, 600)])
def test_rows_left_out_may_hold_anything(N, K, C, bf16):
    phi, w, y, s = _inputs(N, K, C, bf16, left=0.5)
    phi[y < 0] = float("nan")
    phi[torch.nonzero(y < 0)[0]] = float("inf")
    s[y < 0] = float("nan")
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True)
    _check(phi, w, y, s, (loss, dPhi, dW))
    assert torch.all(loss[y < 0] == 0) and torch.all(dPhi[y < 0] == 0)


@pytest.mark.parametrize("N,K,C", WAYS)
@pytest.mark.parametrize("weighted", [False, True])
def test_no_row_counts(N, K, C, weighted):
    phi, w, y, s = _inputs(N, K, C, False, left=2.0)
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s if weighted else None, need_dPhi=True, need_dW=True)
    assert torch.all(loss == 0) and torch.all(dPhi == 0) and torch.all(dW == 0)


def test_no_rows():
    w = torch.randn(5, 9, device="cuda")
    dW = torch.full((5, 12), 7.0, device="cuda")
    loss, dPhi, got = rfsf.rfsf_softmax_xent(torch.empty(0, 9, device="cuda"), w, torch.empty(0, dtype=torch.int64, device="cuda"), need_dPhi=True,
                                             need_dW=True, dW=dW[:, :9])
    assert loss.numel() == 0 and dPhi.shape == (0, 9) and torch.all(got == 0) and torch.all(dW[:, 9:] == 7)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("off", [-1e9, -1e30, -3.3e38])
@pytest.mark.parametrize("N,K,C", WAYS)
def test_classes_shut_off_by_their_offset(N, K, C, off, bf16):
    """Column 0 of features is constant; a huge negative weight there takes a class out. The others lose nothing by it."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    phi[:, 0] = 0.5
    w[3::4, 0] = off
    y[y % 4 == 3] -= 1
    got = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True)
    _check(phi, w, y, s, got)
    assert torch.all(got[2][3::4] == 0)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("off", [-400.0, 400.0])
@pytest.mark.parametrize("N,K,C", WAYS + [(600, 70, 1000)])
def test_scores_far_from_zero(N, K, C, off, bf16):
    """All scores shifted by -200 or 200, which changes nothing but their rounding."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    phi[:, 0] = 0.5
    w[:, 0] = off
    _check(phi, w, y, s, rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("off", [-1e30, 1e30])
@pytest.mark.parametrize("N,K,C", WAYS)
def test_scores_whose_differences_are_lost(N, K, C, off, bf16):
    """Scores near 1e30: equal to 32 bits, so that every class has its share, and nothing overflows."""
    phi, w, y, s = _inputs(N, K, C, bf16, left=0.0)
    phi[:, 0] = 0.5
    w[:, 0] = off
    phi[:, 1:] *= 2.0 ** -30
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True)
    g = (torch.full((N, C), 1.0 / C, device="cuda", dtype=torch.float64) - torch.nn.functional.one_hot(y, C)) * s.double()[:, None]
    assert torch.all((loss.double() - torch.log(torch.tensor(float(C)))).abs() < 1e-5)
    assert torch.isfinite(dPhi).all() and torch.isfinite(dW).all()
    # column 0 alone, the largest of its rows: the others lie so far below it that packing leaves them a few bits
    want, size, dW = g.T @ phi[:, :1].double(), g.abs().T @ phi[:, :1].double().abs(), dW[:, :1]
    assert torch.all((dW.double() - want).abs() <= ((2.0 ** -11 if bf16 else 2.0 ** -20) + 4 * N * 2.0 ** -24) * size + 2.0 ** -8 * want.abs() * bf16 + 1e-30)


@pytest.mark.parametrize("N,K,C", WAYS)
@pytest.mark.parametrize("off", [-3.4028234663852886e38, -3.0e38])
def test_offsets_of_the_lowest_value(N, K, C, off):
    phi, w, y, s = _inputs(N, K, C, False)
    phi[:, 0] = 0.5
    w[3::4, 0] = off
    y[y % 4 == 3] -= 1
    got = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True)
    _check(phi, w, y, s, got)
    assert torch.all(got[2][3::4] == 0)


@pytest.mark.parametrize("N,K,C,bf16", [(700, 513, 2000, False), (700, 513, 2000, True), (3100, 270, 4097, True), (3100, 270, 4097, False),
                                        (4200, 2060, 4097, True), (4200, 2060, 4097, False), (2000, 6164, 40, True)])
def test_large_tiles(N, K, C, bf16):
    """Tiles of all sizes, with and without a 33rd block of rows, against 64 bits on the GPU: each entry within the worst case of its sum, (a + n 2^-24) of
    the sum of magnitudes with a of the operands' rounding."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    dtype = torch.bfloat16 if bf16 else torch.float32
    phi = (torch.randn(N, K, generator=gen, device="cuda") / K ** 0.5).to(dtype)
    w = (torch.randn(C, K, generator=gen, device="cuda") * 2).to(dtype)
    y = torch.randint(0, C, (N,), generator=gen, device="cuda")
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, need_dPhi=True, need_dW=True)
    x, v = phi.double(), w.double()
    l = x @ v.T
    lse = l.logsumexp(1)
    g = (l - lse[:, None]).exp()
    g[torch.arange(N, device="cuda"), y] -= 1
    u = 2.0 ** -24
    dl = ((3 * 2.0 ** -22 + 3 * (K + 4) * u) * (x.abs() @ v.abs().T)).amax(1) + 1e-5
    assert torch.all((loss.double() - (lse - l.gather(1, y[:, None])[:, 0])).abs() <= 2 * dl + 1e-5)
    rough = (2.0 ** -11 if bf16 else 2.0 ** -20) + 2 * dl.max().item()
    out = 2.0 ** -8 if bf16 else 2 * u
    for have, want, size, n in ((dPhi, g @ v / N, g.abs() @ v.abs() / N, C), (dW, g.T @ x / N, g.abs().T @ x.abs() / N, N)):
        assert torch.all((have.double() - want).abs() <= (rough + 3 * (n + 4) * u) * size + out * want.abs() + 1e-12)


@pytest.mark.parametrize("N,K,C", WAYS)
def test_rows_of_all_magnitudes(N, K, C):
    """Rows of Phi from 2^-60 to 2^6, weights of the rows from 2^-30 to 2^30."""
    phi, w, y, s = _inputs(N, K, C, False)
    phi *= torch.pow(2.0, torch.arange(N, device="cuda") % 67 - 60)[:, None]
    s *= torch.pow(2.0, (torch.arange(N, device="cuda") * 7) % 61 - 30)
    _check(phi, w, y, s, rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True))


@pytest.mark.parametrize("N,K,C", WAYS)
def test_infinities_nan_and_labels_beyond_the_classes_show(N, K, C):
    phi, w, y, s = _inputs(N, K, C, False, left=0.0)
    phi[7, 3] = float("nan")
    phi[9, 2] = float("inf")
    y[11] = C
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True)
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[[7, 9, 11]] = True
    assert torch.equal(torch.isnan(loss), bad)
    assert torch.all(torch.isnan(dPhi[bad])) and torch.isfinite(dPhi[~bad]).all() and torch.all(torch.isnan(dW))


@pytest.mark.parametrize("N,K,C", [(60, 20, 9), (200, 90, 150)])
def test_gradients_against_differences(N, K, C):
    """Central differences of the losses along a direction. With scores that move by at most `a` along it, the third derivative of a row's loss
    is at most 8 a^3 (the third central moment of a variable within 2a), so the difference is off by 8 a^3 h^2 / 6; the losses' own errors
    add 2 bound / (2 h)."""
    phi, w, y, s = _inputs(N, K, C, False, seed=3)
    _, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True)
    gen = torch.Generator().manual_seed(9)
    for which in (0, 1):
        d = torch.randn(*(phi if which == 0 else w).shape, generator=gen).cuda()
        d /= d.norm(dim=1, keepdim=True) * (8.0 if which == 0 else 1.0)
        h = 2.0 ** -7
        total, bound = [], 0.0
        for sign in (1, -1):
            a, b = (phi + sign * h * d, w) if which == 0 else (phi, w + sign * h * d)
            loss, _, _ = rfsf.rfsf_softmax_xent(a, b, y)
            r = xent(_np(a), _np(b), _np(y).astype(np.int64), _np(s))
            total.append(float((_np(s) * _np(loss)).sum()))
            bound += float((np.abs(r["s"]) * xent_bounds(r, False)[0]).sum())
        step = (_np(d) @ _np(w).T) if which == 0 else (_np(phi) @ _np(d).T)
        third = 8 * np.abs(step).max(1) ** 3
        grad = (_np(dPhi) * _np(d)).sum() if which == 0 else (_np(dW) * _np(d)).sum()
        difference = (total[0] - total[1]) / (2 * h)
        # the moved operand is rounded to 32 bits: 2^-24 of each number, times the gradient
        moved = 2.0 ** -24 * (np.abs(_np(dPhi) * _np(phi)).sum() if which == 0 else np.abs(_np(dW) * _np(w)).sum()) / h
        assert abs(difference - grad) <= float((np.abs(_np(s)) * third).sum()) * h * h / 6 + bound / (2 * h) + 2 * moved + 1e-5 * abs(grad)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,K,C", [(77, 45, 83)] + WAYS)
def test_padding_of_results_and_odd_strides(N, K, C, bf16):
    phi, w, y, s = _inputs(N, K, C, bf16, pad=5)
    bufs = torch.full((N, K + 5), 9.0, device="cuda", dtype=phi.dtype), torch.full((C, K + 2), 9.0, device="cuda", dtype=phi.dtype)
    got = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True, dPhi=bufs[0][:, 1:K + 1], dW=bufs[1][:, 1:K + 1])
    _check(phi, w, y, s, got)
    assert all(torch.all(b[:, 0] == 9) and torch.all(b[:, K + 1:] == 9) for b in bufs)


@pytest.mark.parametrize("N,K,C", [(40000, 5, 3), (33000, 9, 20)])
def test_many_rows_of_few_columns(N, K, C):
    phi, w, y, _ = _inputs(N, K, C, False)
    _check(phi, w, y, None, rfsf.rfsf_softmax_xent(phi, w, y, need_dPhi=True, need_dW=True))


@pytest.mark.parametrize("N,K,C", WAYS)
def test_equal_calls_give_equal_bits_on_any_stream(N, K, C):
    phi, w, y, s = _inputs(N, K, C, False)
    first = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("N,K,C", WAYS)
def test_in_a_graph(N, K, C):
    phi, w, y, s = _inputs(N, K, C, False)
    rec, _ = rfsf.rfsf_softmax_xent_workspace_bytes(N, K, C, torch.float32, True, True)
    keep = dict(loss=torch.empty(N, device="cuda"), dPhi=torch.empty(N, K, device="cuda"), dW=torch.empty(C, K, device="cuda"),
                workspace=torch.empty(rec, dtype=torch.uint8, device="cuda"))
    call = lambda **kw: rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=True, **kw)          # noqa: E731
    call(**keep)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(**keep)
    for k in range(4):
        phi.mul_(1.25)
        y.add_(1).remainder_(C)
        for t in ("loss", "dPhi", "dW"):
            keep[t].zero_()
        keep["workspace"].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for have, want in zip((keep["loss"], keep["dPhi"], keep["dW"]), call()):
            assert torch.equal(have, want)


def test_features_of_the_library(oracle):
    """Features of the "tiny" configuration, as the library lays them out, into the loss."""
    t = wl.WORKLOADS["tiny"]
    inp = wl.make_inputs(t, 0)
    dev = {k: torch.from_numpy(v).cuda() for k, v in inp.items() if isinstance(v, np.ndarray)}
    phi = rfsf.rfsf_ts_features(dev["X"], dev["W"], dev["hash"], dev["sign"], inp["lengthscale"], t.D)
    rfsf.rfsf_ts_normalize_features(phi, t.M, t.D)
    gen = torch.Generator().manual_seed(1)
    w = torch.randn(4, t.ncols, generator=gen).cuda()
    y = torch.randint(0, 4, (t.N,), generator=gen).cuda()
    _check(phi, w, y, None, rfsf.rfsf_softmax_xent(phi, w, y, need_dPhi=True, need_dW=True))
