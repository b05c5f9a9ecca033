"""Calls of layer norm and of scores with adapters that the header allows: statistics that nobody wants, graphs that share a workspace, gains or offsets alone."""
import ctypes

import pytest
import torch

import paper_2501_07145_amd as rfsf
from paper_2501_07145_amd import binding, linear

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(7, 65), (2100, 65), (2100, 1025), (3, 20485)])
def test_statistics_that_are_not_wanted(dtype, N, K):
    x = torch.randn(N, K, device="cuda").to(TYPES[dtype])
    want, mean, rstd = rfsf.rfsf_layer_norm(x)
    shape = linear._LayerNormShape(N, K, K, K, K, int(dtype == "bfloat16"))
    for at in ((), (0,), (1,)):
        out, stats = torch.empty_like(x), [torch.full((N,), -7.0, device="cuda") for _ in range(2)]
        pointers = [s.data_ptr() if i in at else None for i, s in enumerate(stats)]
        rc = binding.load_library().rfsf_layer_norm(ctypes.byref(shape), x.data_ptr(), None, None, 1e-5, None, out.data_ptr(), *pointers, binding._stream_ptr(None))
        assert rc == 0 and torch.equal(out, want)
        for i, (s, w) in enumerate(zip(stats, (mean, rstd))):
            assert torch.equal(s, w) if i in at else bool((s == -7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(7, 65), (2100, 1025), (3, 20485)])
def test_gains_or_offsets_alone(dtype, N, K):
    x = torch.randn(N, K, device="cuda").to(TYPES[dtype])
    gain, offset = torch.rand(K, device="cuda"), torch.rand(K, device="cuda")
    one, zero = torch.ones(K, device="cuda"), torch.zeros(K, device="cuda")
    for have, same in (((gain, None), (gain, zero)), ((None, offset), (one, offset)), ((None, None), (one, zero))):
        assert torch.equal(rfsf.rfsf_layer_norm(x, *have)[0], rfsf.rfsf_layer_norm(x, *same)[0])


def test_graphs_that_share_a_workspace():
    x, dy, gain = torch.randn(700, 1025, device="cuda"), torch.randn(700, 1025, device="cuda"), torch.rand(1025, device="cuda")
    _, mean, rstd = rfsf.rfsf_layer_norm(x, gain)
    W, A, B = torch.randn(900, 1025, device="cuda"), torch.randn(5, 8, 1025, device="cuda"), torch.randn(5, 900, 8, device="cuda")
    h = rfsf.RfsfAdapters(W, 5, 8)
    for e in range(5):
        h.set(e, A[e], B[e])
    who = [torch.randint(-1, 5, (n,), device="cuda") for n in (700, 40)]
    need = max(rfsf.rfsf_layer_norm_backward_workspace_bytes(700, 1025)[0], *(h.workspace_bytes(n)[0] for n in (700, 40)))
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = [torch.empty(1025, device="cuda"), torch.empty(1025, device="cuda"), torch.empty_like(x), torch.empty(700, 900, device="cuda"), torch.empty(40, 900, device="cuda")]

    def back():
        rfsf.rfsf_layer_norm_backward(x, mean, rstd, dy, gain=gain, dX=out[2], dgain=out[0], doffset=out[1], workspace=space)

    def scores(i):
        h.scores(x[:len(who[i])], who[i], out=out[3 + i], workspace=space)

    calls = [back, lambda: scores(0), lambda: scores(1)]
    for call in calls:
        call()
    want = [t.clone() for t in out]
    torch.cuda.synchronize()
    graphs = []
    for call in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for order in ((0, 1, 2), (2, 0, 1), (1, 2, 0), (0, 0, 2, 1)):
        for t in out:
            t.fill_(-7.0)
        space.fill_(255)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), order
