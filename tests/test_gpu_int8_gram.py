"""Rows as 8-bit integers and the Gram against them on the GPU: codes to the bit, sums against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _rows(N, K, seed, bf16=False, pad=1):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(N, K + pad, generator=gen) * torch.exp(2 * torch.randn(N, 1, generator=gen))
    return x.to(torch.bfloat16 if bf16 else torch.float32).cuda()[:, :K]


def _codes(x):
    """The definition, with numpy's 32-bit operations."""
    x = x.float().cpu().numpy()
    top = np.abs(x).max(1)
    with np.errstate(divide="ignore"):
        inverse = np.where(top < np.float32(2.0 ** -119), np.float32(0), (np.float32(1) / top) * np.float32(127)).astype(np.float32)
    return np.rint(x * inverse[:, None]).astype(np.int64), (top * np.float32(1.0 / 127.0)).astype(np.float32)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 5), (2, 127), (2, 128), (5, 129), (70, 1025), (3, 10241)])
def test_codes_are_the_definition_and_the_room_is_cleared(N, K, bf16):
    x = _rows(N, K, 0, bf16)
    x[0] = 0
    if N > 2:
        x[2] *= 2.0 ** -125
    room = (K + 127) // 128 * 128
    buf = torch.full((N, room + 16), 77, dtype=torch.int8, device="cuda")
    codes, scales = rfsf.rfsf_int8_quantize(x, codes=buf[:, :K])
    want, want_scales = _codes(x)
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), want_scales)
    assert torch.all(buf[:, K:room] == 0) and torch.all(buf[:, room:] == 77)
    again, _ = rfsf.rfsf_int8_quantize(x)
    assert torch.equal(again, codes) and again.stride(0) % 128 == 0


def test_more_rows_than_a_launch_has():
    """2^23 + 9 rows of three columns: every one is quantised, the ones about the launches' ends too."""
    N = (1 << 23) + 9
    x = (torch.arange(3 * N, device="cuda", dtype=torch.float32).reshape(N, 3) % 251) - 125
    codes, scales = rfsf.rfsf_int8_quantize(x)
    top = x.abs().amax(dim=1)
    assert torch.equal(scales, top * torch.tensor(1.0 / 127.0, dtype=torch.float32, device="cuda"))
    for at in (0, (1 << 22) - 4, (1 << 22) + 1, (1 << 23) - 4, N - 9):
        assert np.array_equal(codes[at:at + 9].cpu().numpy(), _codes(x[at:at + 9])[0])
    assert torch.equal(codes.abs().amax(dim=1) == 127, top > 0) and torch.all(codes[top == 0] == 0)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,K", [(9, 1), (4096, 1), (4095, 255), (4097, 256), (4103, 511), (5000, 1000), (4099, 1023), (4111, 1024), (4100, 1025)])
def test_narrow_rows(N, K, bf16):
    """Few and many of them: a workgroup and a wavefront per row."""
    x = _rows(N, K, 1, bf16)
    room = (K + 127) // 128 * 128
    buf = torch.full((N, room + 16), 77, dtype=torch.int8, device="cuda")
    codes, scales = rfsf.rfsf_int8_quantize(x, codes=buf[:, :K])
    want, want_scales = _codes(x)
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), want_scales)
    assert torch.all(buf[:, K:room] == 0) and torch.all(buf[:, room:] == 77)


SIZES = [(1, 1, 1), (1, 1000, 1025), (2, 33, 64), (3, 40, 65), (5, 1000, 300), (8, 777, 129), (9, 500, 1001), (16, 65, 40), (17, 300, 2049), (40, 63, 5),
         (64, 64, 128), (65, 129, 127), (300, 257, 70), (130, 3000, 513), (1, 7, 10241), (4, 4, 131072),
         (8, 100, 1024), (8, 100, 1025), (16, 300, 511), (3, 17000, 129), (12, 16385, 200), (16, 20001, 70), (260, 17000, 33), (2500, 5124, 40)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("Nx,Ny,K", SIZES)
def test_against_64_bits(Nx, Ny, K, bf16):
    """The sums are exact: what is left is the sum's rounding to 32 bits and three products' or scales'."""
    x, y = _rows(Nx, K, 1, bf16), _rows(Ny, K, 2)
    codes, scales = rfsf.rfsf_int8_quantize(y)
    out = torch.full((Nx, Ny + 3), 5.0, device="cuda")
    got = rfsf.rfsf_int8_gram(x, codes, scales, K=out[:, 1:Ny + 1])
    qx, sx = _codes(x)
    sums = qx.astype(np.float64) @ codes.cpu().numpy().astype(np.float64).T
    want = sums * sx.astype(np.float64)[:, None] * scales.cpu().numpy().astype(np.float64)[None, :]
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= 4 * U * np.abs(want) + 1e-40)
    assert torch.all(out[:, 0] == 5) and torch.all(out[:, Ny + 1:] == 5)


def test_largest_codes_do_not_overflow():
    x = torch.full((3, 131072), -1.0, device="cuda")
    codes = torch.full((70, 131072), -128, dtype=torch.int8, device="cuda")
    got = rfsf.rfsf_int8_gram(x, codes, torch.ones(70, device="cuda"))
    assert torch.allclose(got.double(), torch.full((), 128.0 * 131072, dtype=torch.float64, device="cuda"), rtol=4 * U)


@pytest.mark.parametrize("Nx", [1, 3, 12, 40])
def test_what_lies_behind_the_columns_of_stored_rows_does_not_count(Nx):
    x, y = _rows(Nx, 70, 3), _rows(200, 70, 4)
    buf = torch.full((200, 144), 99, dtype=torch.int8, device="cuda")
    codes, scales = rfsf.rfsf_int8_quantize(y)
    buf[:, :70] = codes
    assert torch.equal(rfsf.rfsf_int8_gram(x, buf[:, :70], scales), rfsf.rfsf_int8_gram(x, codes, scales))


@pytest.mark.parametrize("Nx", [1, 5, 70])
def test_zero_rows_and_rows_that_are_not_finite(Nx):
    x, y = _rows(Nx, 300, 5), _rows(90, 300, 6)
    codes, scales = rfsf.rfsf_int8_quantize(y)
    for value, what in ((0.0, lambda t: t == 0), (float("nan"), torch.isnan), (float("inf"), torch.isnan)):
        z = x.clone()
        if value == 0.0:
            z[-1] = 0
        else:
            z[-1, 17] = value
        got = rfsf.rfsf_int8_gram(z, codes, scales)
        assert torch.all(what(got[-1])) and torch.equal(got[:-1], rfsf.rfsf_int8_gram(x, codes, scales)[:-1])


def test_small_workspaces_give_the_same():
    x, y = _rows(333, 200, 7), _rows(150, 200, 8)
    codes, scales = rfsf.rfsf_int8_quantize(y)
    whole = rfsf.rfsf_int8_gram(x, codes, scales)
    recommended, least = rfsf.rfsf_int8_gram_workspace_bytes(333, 150, 200)
    for size in (least, (least + recommended) // 2):
        workspace = torch.full((size + 3,), 255, dtype=torch.uint8, device="cuda")[3:]
        assert torch.equal(rfsf.rfsf_int8_gram(x, codes, scales, workspace=workspace), whole)


@pytest.mark.parametrize("Nx", [1, 300])
def test_on_another_stream_and_in_a_graph(Nx):
    x, y = _rows(Nx, 500, 9), _rows(400, 500, 10)
    codes, scales = rfsf.rfsf_int8_quantize(y)
    workspace = torch.empty(rfsf.rfsf_int8_gram_workspace_bytes(Nx, 400, 500)[0], dtype=torch.uint8, device="cuda")
    out = torch.empty(Nx, 400, device="cuda")
    first = rfsf.rfsf_int8_gram(x, codes, scales)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = rfsf.rfsf_int8_gram(x, codes, scales, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again)
    rfsf.rfsf_int8_gram(x, codes, scales, K=out, workspace=workspace)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rfsf.rfsf_int8_gram(x, codes, scales, K=out, workspace=workspace)
    for _ in range(3):
        x.mul_(-1.5)
        out.zero_()
        workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, rfsf.rfsf_int8_gram(x, codes, scales))


def test_refusals():
    x, y = _rows(3, 70, 11), _rows(5, 70, 12)
    codes, scales = rfsf.rfsf_int8_quantize(y)
    tight = codes.contiguous()                                  # rows of 70 bytes: no room behind the columns
    for c, s in ((tight, scales), (codes[:, :69], scales), (codes, scales[:4]), (codes.float(), scales), (codes.cpu(), scales)):
        with pytest.raises((ValueError, rfsf.RfsfTsError)):
            rfsf.rfsf_int8_gram(x, c, s)
    with pytest.raises(ValueError):
        rfsf.rfsf_int8_gram(x.half(), codes, scales)
    with pytest.raises(ValueError):
        rfsf.rfsf_int8_gram(x, codes, scales, K=torch.empty(3, 4, device="cuda"))
    with pytest.raises(rfsf.RfsfTsError):
        rfsf.rfsf_int8_gram(x, codes, scales, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
