"""Softmax cross entropy on the GPU: rows whose label says something other than a class."""
import pytest
import torch

import paper_2501_07145_amd as rfsf

pytestmark = pytest.mark.gpu


def _inputs(N, K, C, bf16, seed=0):
    gen = torch.Generator().manual_seed(seed)
    dtype = torch.bfloat16 if bf16 else torch.float32
    phi = (torch.randn(N, K, generator=gen) / K ** 0.5).to(dtype)
    w = (torch.randn(C, K, generator=gen) * 2).to(dtype)
    return phi.cuda(), w.cuda(), torch.randint(0, C, (N,), generator=gen).cuda(), torch.rand(N, generator=gen).cuda()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("need_dPhi,need_dW", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("N,K,C", [(300, 40, 1), (300, 40, 3), (300, 300, 5), (260, 600, 10), (140, 1100, 13), (200, 2100, 10), (90, 40, 33), (12, 40, 300), (620, 300, 600)])
def test_labels_beyond_the_classes(N, K, C, need_dPhi, need_dW, weighted, bf16):
    """C itself, which shares a group of four with classes that exist, the next ones, and far ones: their rows' losses and gradients are NaN, the others' are not."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    beyond = torch.arange(N, device="cuda") % 3 == 1
    y[beyond] = C + torch.arange(int(beyond.sum()), device="cuda") % 4
    y[torch.nonzero(beyond)[-2:, 0]] = torch.tensor([1 << 31, (1 << 63) - 1], device="cuda")
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s if weighted else None, need_dPhi=need_dPhi, need_dW=need_dW)
    assert torch.equal(torch.isnan(loss), beyond) and torch.isfinite(loss[~beyond]).all()
    if need_dPhi:
        assert torch.isnan(dPhi[beyond]).all() and torch.isfinite(dPhi[~beyond]).all()
    if need_dW:
        assert torch.isnan(dW).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("need_dW", [True, False])
@pytest.mark.parametrize("N,K,C", [(300, 40, 7), (7, 3, 2), (9000, 300, 16), (200, 2100, 10), (12, 40, 300), (5, 700, 9000), (90, 40, 33), (90, 40, 300), (40, 33, 9000), (620, 300, 600),
                                   (150, 130, 3000)])
def test_rows_left_out_have_no_gradient_whatever_the_weights_hold(N, K, C, need_dW, value, bf16):
    """One number of W is not finite: loss and dPhi of the rows that are left out are 0 all the same."""
    phi, w, y, s = _inputs(N, K, C, bf16)
    w[C // 2, K // 2] = value
    y[torch.arange(N, device="cuda") % 2 == 1] = -1
    phi[1] = float("nan")
    loss, dPhi, _ = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=True, need_dW=need_dW)
    assert torch.all(loss[y < 0] == 0) and torch.all(dPhi[y < 0] == 0) and torch.isnan(dPhi[y >= 0]).any()
