"""The Gram against 8-bit rows on the GPU where the product of two scales is beyond what 32 bits hold, and the result is not."""
import pytest
import torch

import paper_2501_07145_amd as rfsf

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


# (rows, stored rows, columns): rows quantised by the workgroups, by a launch of their own, packed
@pytest.mark.parametrize("Nx,Ny,K", [(2, 100, 300), (5, 17000, 300), (12, 300, 1000), (40, 300, 300), (300, 700, 300)])
@pytest.mark.parametrize("bf16", [False, True])
def test_scales_far_from_one(Nx, Ny, K, bf16):
    """Each result is the exact sum, rounded, times two scales: three roundings, wherever it is a normal number of 32 bits. Beyond, infinity; an exact sum of zero is zero."""
    gen = torch.Generator().manual_seed(1)
    x, y = torch.randn(Nx, K, generator=gen), torch.randn(Ny, K, generator=gen)
    x[:, K // 2:] = x[:, :K // 2]
    y[0, K // 2:] = -y[0, :K // 2]                                         # (its sum with every row is zero)
    x *= torch.pow(2.0, torch.tensor([100.0, -75.0, -110.0, 60.0, 0.0]))[torch.arange(Nx) % 5][:, None]
    y *= torch.pow(2.0, torch.tensor([100.0, -75.0, 110.0, -40.0, 0.0, 20.0, -105.0]))[torch.arange(Ny) % 7][:, None]
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    codes, scales = rfsf.rfsf_int8_quantize(y.cuda())
    q, s = rfsf.rfsf_int8_quantize(x)
    sums = q.cpu().double() @ codes.cpu().double().T
    want = (sums * s.cpu().double()[:, None]) * scales.cpu().double()[None, :]
    got = rfsf.rfsf_int8_gram(x, codes, scales).cpu()
    assert torch.all(sums[:, 0] == 0) and torch.all(got[sums == 0] == 0)
    over = want.abs() > 2.0 ** 128 * (1 - 4 * U)
    assert torch.all(torch.isinf(got[want.abs() > 2.0 ** 128])) and torch.isfinite(got[~over]).all()
    off = (got.double() - want).abs()[~over]
    assert torch.all(off <= 4 * U * want.abs()[~over] + 2.0 ** -149)
    assert int(over.sum()) > 0


@pytest.mark.parametrize("Nx,Ny,K", [(2, 100, 300), (5, 17000, 300), (12, 300, 1000), (40, 300, 300), (300, 700, 300)])
def test_products_of_scales_below_the_normal_numbers(Nx, Ny, K):
    """Scales near 2^-80 and 2^-55, whose product has 14 bits: results near 2^-119 have all of theirs."""
    gen = torch.Generator().manual_seed(2)
    x, y = torch.randn(Nx, K, generator=gen) * 2.0 ** -75, torch.randn(Ny, K, generator=gen) * 2.0 ** -50
    codes, scales = rfsf.rfsf_int8_quantize(y.cuda())
    q, s = rfsf.rfsf_int8_quantize(x.cuda())
    product = s.cpu().double()[:, None] * scales.cpu().double()[None, :]
    want = (q.cpu().double() @ codes.cpu().double().T) * product
    assert torch.all(product < 2.0 ** -130)
    got = rfsf.rfsf_int8_gram(x.cuda(), codes, scales).cpu().double()
    assert torch.all((got - want).abs() <= 4 * U * want.abs() + 2.0 ** -149)
