"""How many bits of G = softmax - onehot reach the gradients: results that are differences of two almost equal numbers of G show them, whatever the
gradients' own type is."""
import pytest
import torch

import paper_2501_07145_amd as rfsf

pytestmark = pytest.mark.gpu


def _pairs(N, C, bf16, seed):
    """Phi, W, labels. Scores come from columns 0 .. 5 alone. Class 2j + 1 has the weights of class 2j but for column 0, where the two differ by 2^-8, so that
    their shares of a row differ by about 2^-9 of themselves; column 6 + j of W is 1 for one and -1 for the other, of Phi 0, so that
    dPhi there is G[:, 2j] - G[:, 2j + 1]. Sequences 2i and 2i + 1 and columns 6 + C / 2 + i of Phi in the same way."""
    gen = torch.Generator().manual_seed(seed)
    few, half_c, half_n = 6, C // 2, N // 2
    K = few + half_c + half_n
    w, phi = torch.zeros(C, K), torch.zeros(N, K)
    w[0:2 * half_c:2, 1:few] = torch.randn(half_c, few - 1, generator=gen).bfloat16().float()
    w[1:2 * half_c:2, 1:few] = w[0:2 * half_c:2, 1:few]
    w[0:2 * half_c:2, 0], w[1:2 * half_c:2, 0] = 2.0 ** -9, -2.0 ** -9
    phi[0:2 * half_n:2, 1:few] = (torch.randn(half_n, few - 1, generator=gen) / 2).bfloat16().float()
    phi[1:2 * half_n:2, 1:few] = phi[0:2 * half_n:2, 1:few]
    phi[0:2 * half_n:2, 0], phi[1:2 * half_n:2, 0] = 0.5, 0.25
    j, i = torch.arange(half_c), torch.arange(half_n)
    w[2 * j, few + j], w[2 * j + 1, few + j] = 1.0, -1.0
    phi[2 * i, few + half_c + i], phi[2 * i + 1, few + half_c + i] = 1.0, -1.0
    labels = torch.randint(0, C, (half_n,), generator=gen).repeat_interleave(2)
    labels = torch.cat([labels, labels[:N - 2 * half_n] * 0])
    dtype = torch.bfloat16 if bf16 else torch.float32
    return phi.to(dtype).cuda(), w.to(dtype).cuda(), labels.cuda(), few, half_c, half_n


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,C", [(60, 40), (12, 300), (300, 7), (620, 600), (1500, 900), (301, 2050)])
def test_differences_of_almost_equal_numbers(N, C, bf16):
    """dPhi and dW against 64 bits. An element is g1 - g2, of which each is off by: the scores' error (six products and sums of numbers below about 8,
    2^-22 of each operand: 2^-18 in all), the exponential's argument and the sum (2^-20), its way into the product (2^-16 of itself where it
    enters as two terms of bfloat16, less everywhere else); together below 2^-15. The result is rounded to its type. (With 11 bits, 2^-12.) Numbers below 2^-17 of the
    largest product that they take part in may be off by 2^-38 of that, and are left out."""
    phi, w, y, few, half_c, half_n = _pairs(N, C, bf16, 7)
    ones = torch.ones(N, device="cuda")
    _, dPhi, dW = rfsf.rfsf_softmax_xent(phi, w, y, weight=ones, need_dPhi=True, need_dW=True)
    x, v = phi.double(), w.double()
    g = torch.softmax(x[:, :few] @ v[:, :few].T.contiguous(), 1)
    g[torch.arange(N, device="cuda"), y] -= 1
    out = 2.0 ** -8 if bf16 else 2.0 ** -23
    largest = (g.abs() * v.abs().amax(1)).amax(1, keepdim=True)
    a, b = g[:, 0:2 * half_c:2], g[:, 1:2 * half_c:2]
    off = (dPhi[:, few:few + half_c].double() - (a - b)).abs()
    wrong = (off > 2.0 ** -15 * (a.abs() + b.abs()) + out * (a - b).abs() + 1e-30) & (torch.minimum(a.abs(), b.abs()) > 2.0 ** -17 * largest)
    assert int(wrong.sum()) == 0
    largest = x.abs().max()
    a, b = g[0:2 * half_n:2], g[1:2 * half_n:2]
    off = (dW[:, few + half_c:].double().T - (a - b)).abs()
    wrong = (off > 2.0 ** -15 * (a.abs() + b.abs()) + out * (a - b).abs() + 1e-30) & (torch.minimum(a.abs(), b.abs()) > 2.0 ** -17 * largest)
    assert int(wrong.sum()) == 0
