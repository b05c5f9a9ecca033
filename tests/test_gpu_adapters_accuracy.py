"""The accuracy of scores with adapters, worked on in every way: those of the GPU against 64 bits."""
import pytest
import torch

import paper_2501_07145_amd as rfsf
from tests.adapters_accuracy import CASES, MEAN, SINGLE, errors, problem, scores
from tests.test_gpu_adapters import CASES as OTHER_CASES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K,C,rank,count,bf16", [c[:6] for c in CASES] + [c + (bf16,) for c in OTHER_CASES for bf16 in (False, True)])
def test_errors_are_those_of_22_bits(N, K, C, rank, count, bf16):
    X, W, A, B, scale, adapters = problem(N, K, C, rank, count, bf16, "cuda")
    dtype = torch.bfloat16 if bf16 else torch.float32
    h = rfsf.RfsfAdapters(W.to(dtype), count, rank)
    for e in range(count):
        h.set(e, A[e].to(dtype), B[e].to(dtype), float(scale[e]))
    got = h.scores(X.to(dtype), adapters)
    mean, most = errors(got, *scores(X, W, A, B, scale, adapters))
    assert mean <= MEAN and most <= SINGLE
