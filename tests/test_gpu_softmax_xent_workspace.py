"""Softmax cross entropy on the GPU in exactly the workspace that it asks for: nothing behind it or before it is written, and what it held does not count."""
import pytest
import torch

import paper_2501_07145_amd as rfsf

pytestmark = pytest.mark.gpu

GUARD = 8192


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("need_dPhi,need_dW", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("N,K,C", [(1, 1, 1), (7, 3, 2), (300, 70, 7), (9001, 67, 3), (40000, 5, 3), (5000, 300, 16), (200, 2100, 10), (3000, 66, 64), (33, 2100, 40), (12, 40, 30),
                                   (12, 40, 300), (16, 300, 9000), (5, 70, 20000), (90, 40, 33), (90, 40, 300), (20, 5000, 300), (2100, 40, 50), (40, 33, 9000), (620, 300, 600)])
def test_only_the_workspace_is_written(N, K, C, need_dPhi, need_dW, bf16):
    gen = torch.Generator().manual_seed(4)
    dtype = torch.bfloat16 if bf16 else torch.float32
    phi, w = (torch.randn(N, K, generator=gen) / K ** 0.5).to(dtype).cuda(), torch.randn(C, K, generator=gen).to(dtype).cuda()
    y = (torch.randint(0, C + 1, (N,), generator=gen) - 1).cuda()
    recommended, least = rfsf.rfsf_softmax_xent_workspace_bytes(N, K, C, dtype, need_dPhi, need_dW)
    results = []
    for size, fill in ((recommended, 255), (least, 0), (recommended, 60)):
        room = torch.full((size + 2 * GUARD,), fill, dtype=torch.uint8, device="cuda")
        got = rfsf.rfsf_softmax_xent(phi, w, y, need_dPhi=need_dPhi, need_dW=need_dW, workspace=room[GUARD:GUARD + size])
        assert torch.all(room[:GUARD] == fill) and torch.all(room[GUARD + size:] == fill)
        results.append([t for t in got if t is not None])
    assert all(torch.equal(a, b) for a, b in zip(results[0], results[2])) and all(torch.isfinite(t).all() for r in results for t in r)
