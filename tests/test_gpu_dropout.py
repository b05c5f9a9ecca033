"""Dropout against the generator's numbers: the same places are kept, whatever the type, the size, the strides and the way rows are
cut, and what is kept is scaled."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf
from tests import norm_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


def _rows(N, K, dtype, ld, seed, shift=0):
    """Rows ld numbers apart, `shift` numbers into their memory, with something else around them."""
    gen = torch.Generator().manual_seed(seed)
    buf = torch.full((shift + N * ld + 8,), -7.0, dtype=dtype)
    x = buf[shift:shift + N * ld].view(N, ld)[:, :K]
    x.copy_(torch.randn(N, K, generator=gen))
    return buf.cuda()[shift:shift + N * ld].view(N, ld)[:, :K]


def _check(out, x, factor, bf16):
    want = x.double().cpu().numpy() * factor
    got = out.double().cpu().numpy()
    assert np.array_equal(got == 0, want == 0)
    # the factor, the product and, with bfloat16, the result are rounded
    tol = (2 * ref.U + ref.BF16 * (1 + 2 * ref.U)) if bf16 else 2 * ref.U
    assert np.all(np.abs(got - want) <= tol * np.abs(want) + 2.0 ** -133)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K,p", [(1, 1, 0.5), (1, 7, 0.3), (3, 8, 0.1), (5, 9, 0.9), (17, 65, 0.25), (300, 65, 0.2), (9, 257, 0.5), (4, 512, 0.01), (6, 1025, 0.6),
                                   (2, 4097, 0.1), (3, 10241, 0.35), (1, 70001, 0.5), (2000, 33, 0.7), (70000, 1, 0.4), (3001, 9, 0.3), (517, 129, 0.3)])
def test_places_and_values(dtype, N, K, p):
    bf16 = dtype == "bfloat16"
    for ld, shift in ((K, 0), ((K + 7) // 8 * 8, 0), (K + 3, 1)):
        x = _rows(N, K, TYPES[dtype], ld, seed=K, shift=shift)
        out = _rows(N, K, TYPES[dtype], ld + 2, seed=1)
        got = rfsf.rfsf_dropout(x, rfsf.RfsfDropout(p, seed=123456789012345678, offset=1 << 40, first_row=3), out=out)
        assert got is out
        _check(got, x, ref.mask(N, K, p, 123456789012345678, 1 << 40, 3), bf16)
        assert torch.all(out._base[:N * (ld + 2)].view(N, ld + 2)[:, K:] == -7.0) and torch.all(out._base[N * (ld + 2):] == -7.0)    # what is beyond stays as it was


@pytest.mark.parametrize("dtype", TYPES)
def test_probabilities_at_the_ends(dtype):
    x = _rows(11, 77, TYPES[dtype], 77, seed=2)
    assert torch.equal(rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.0, 5)), x)
    assert torch.equal(rfsf.rfsf_dropout(x, rfsf.RfsfDropout(2.0 ** -18, 5)), x)               # rounds to none
    assert torch.all(rfsf.rfsf_dropout(x, rfsf.RfsfDropout(1.0, 5)) == 0)
    _check(rfsf.rfsf_dropout(x, rfsf.RfsfDropout(65535 / 65536, 5)), x, ref.mask(11, 77, 65535 / 65536, 5), dtype == "bfloat16")


def test_settings_at_the_ends_of_their_range():
    x = torch.ones(6, 40, device="cuda")
    for kw in (dict(seed=(1 << 64) - 1), dict(seed=1 << 32), dict(seed=7, offset=(1 << 64) - 1), dict(seed=7, first_row=(1 << 32) - 6), dict(seed=7, offset=1 << 32)):
        got = rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.5, **kw))
        assert np.array_equal(got.cpu().numpy() != 0, ref.mask(6, 40, 0.5, **kw) != 0), kw


def test_rows_worked_on_in_parts_and_in_place():
    x = _rows(50, 333, torch.float32, 336, seed=4)
    whole = rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.4, 99, offset=3))
    parts = [rfsf.rfsf_dropout(x[a:b], rfsf.RfsfDropout(0.4, 99, offset=3, first_row=a)) for a, b in ((0, 1), (1, 30), (30, 50))]
    assert torch.equal(whole, torch.cat(parts))
    y = x.clone()
    assert rfsf.rfsf_dropout(y, rfsf.RfsfDropout(0.4, 99, offset=3), out=y) is y
    assert torch.equal(y, whole)
    assert rfsf.rfsf_dropout(x[:0], rfsf.RfsfDropout(0.4, 99)).shape == (0, 333)


def test_what_is_left_out_is_zero_whatever_it_was():
    factor = ref.mask(8, 100, 0.5, 1)
    x = torch.ones(8, 100, device="cuda")
    dropped = torch.from_numpy(factor == 0).cuda()
    x[dropped] = float("nan")
    x[3][dropped[3]] = float("inf")
    got = rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.5, 1))
    assert torch.equal(got, torch.from_numpy(factor).float().cuda())


def test_a_counter_on_the_device_and_a_captured_graph():
    x = torch.randn(30, 129, device="cuda")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    settings = rfsf.RfsfDropout(0.3, 42, offset=1000, counter=counter)
    out = torch.empty_like(x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        rfsf.rfsf_dropout(x, settings, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rfsf.rfsf_dropout(x, settings, out=out)
        counter.add_(1)
    for step in range(4):
        assert int(counter) == step
        graph.replay()
        eager = rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.3, 42, offset=1000 + step))
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_another_stream():
    x = torch.randn(200, 1025, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.3, 42), stream=stream)
    stream.synchronize()
    assert torch.equal(got, rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.3, 42)))


def test_rows_beyond_two_to_the_31_numbers():
    N, K = 33000, 65537
    x = torch.ones(N, K, dtype=torch.bfloat16, device="cuda")
    rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.5, 8), out=x)
    want = ref.mask(N, K // 2000, 0.5, 8)
    assert np.array_equal(x[:, :K // 2000].float().cpu().numpy(), want)
    groups = ref.mask(2, K, 0.5, 8, first_row=N - 2)
    assert np.array_equal(x[N - 2:].float().cpu().numpy(), groups)


def test_share_of_places_and_independence_of_rows():
    # 4e6 places kept with probability 3/4: five standard deviations are 0.11 %; two rows agree in a share of 10/16 of the places
    x = torch.ones(400, 10000, device="cuda")
    kept = rfsf.rfsf_dropout(x, rfsf.RfsfDropout(0.25, 31)) != 0
    assert abs(float(kept.float().mean()) - 0.75) < 5 * (0.75 * 0.25 / 4e6) ** 0.5
    agree = (kept[1:] == kept[:-1]).float().mean()
    assert abs(float(agree) - 0.625) < 5 * (0.625 * 0.375 / 3.99e6) ** 0.5 * 1.5
