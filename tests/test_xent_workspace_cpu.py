"""The workspace of softmax cross entropies that are worked on straight from the matrices: room for what is written there, and for nothing else."""
import pytest
import torch

import paper_2501_07145_amd as rfsf

MB = 1 << 20


@pytest.mark.parametrize("N,K,C,need_dPhi,need_dW,most", [
    # up to 64 classes, losses alone: the scores stay in registers
    (1 << 22, 65, 16, False, False, MB), (1 << 26, 65, 1, False, False, MB), (60000, 1025, 64, False, False, MB),
    # one pass: parts of dW, 256 at most
    (1 << 22, 65, 16, True, True, 256 * 16 * 65 * 4 + MB), (1 << 22, 65, 16, False, True, 256 * 16 * 65 * 4 + MB), (4096, 1025, 16, True, False, MB),
    # few rows, losses alone: the scores once, no G
    (16, 65, 1000000, False, False, 16 * 1000000 * 4 + 16 * 62500 * 8 + MB),
    # few rows with gradients: the scores and G
    (16, 65, 100000, True, True, 2 * 16 * 100000 * 4 + 16 * 6252 * 8 + 128 * 16 * 65 * 4 + MB),
])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nothing_is_asked_for_that_is_not_used(N, K, C, need_dPhi, need_dW, most, dtype):
    recommended, least = rfsf.rfsf_softmax_xent_workspace_bytes(N, K, C, dtype, need_dPhi, need_dW)
    assert 0 < least <= recommended <= most
