"""The accuracy of softmax cross entropies of packed operands, tiles of every size: loss and gradients of the GPU against 64 bits."""
import pytest
import torch

import paper_2501_07145_amd as rfsf
from tests.xent_accuracy import CASES, MEAN, MEAN_BF16, SINGLE

pytestmark = pytest.mark.gpu


def _mean_error(have, want):
    return float((have - want).norm() / want.norm())


@pytest.mark.parametrize("N,K,C,bf16", [c[:4] for c in CASES])
@pytest.mark.parametrize("gradients,share", [(True, 1.0), (True, 0.3), (False, 1.0)])
def test_errors_are_those_of_22_bits(N, K, C, bf16, gradients, share):
    gen = torch.Generator(device="cuda").manual_seed(2)
    dtype = torch.bfloat16 if bf16 else torch.float32
    phi = (torch.randn(N, K, generator=gen, device="cuda") / K ** 0.5).to(dtype)
    w = (torch.randn(C, K, generator=gen, device="cuda") * 2).to(dtype)
    y = torch.randint(0, C, (N,), generator=gen, device="cuda")
    s = 0.5 + torch.rand(N, generator=gen, device="cuda")
    most, least = rfsf.rfsf_softmax_xent_workspace_bytes(N, K, C, dtype, gradients, gradients)
    workspace = torch.empty(max(least, int(share * most)), dtype=torch.uint8, device="cuda")
    loss, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=s, need_dPhi=gradients, need_dW=gradients, workspace=workspace)
    x, v = phi.double(), w.double()
    l = x @ v.T
    lse = l.logsumexp(1)
    want = lse - l.gather(1, y[:, None])[:, 0]
    assert _mean_error(loss.double(), want) <= MEAN
    assert torch.all((loss.double() - want).abs() <= SINGLE * 8)                       # (scores of about 2, losses of about 10)
    if not gradients:
        return
    g = (l - lse[:, None]).exp()
    g[torch.arange(N, device="cuda"), y] -= 1
    g *= s.double()[:, None]
    for have, want, size in ((dPhi, g @ v, (g.square() @ v.square()).sqrt()), (dW, g.T @ x, (g.square().T @ x.square()).sqrt())):
        if bf16:
            assert _mean_error(have.double(), want.to(dtype).double()) <= MEAN_BF16
            assert torch.all((have.double() - want).abs() <= SINGLE * size + 2.0 ** -8 * want.abs())
        else:
            assert _mean_error(have.double(), want) <= MEAN
            assert torch.all((have.double() - want).abs() <= SINGLE * size)
