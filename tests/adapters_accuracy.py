"""How far scores with adapters may be from 64 bits, by the size that their rounding errors have on average, which says much less than the worst case of long sums does, and sizes
for every way that scores are worked on."""
import numpy as np
import torch

# rows, columns, classes, rank, adapters, bfloat16, what the way's last launches are: the shared product's tiles (256x: with a joined block of up to 32 classes) with the
# adapters' part in their epilogue or cut into parts, straight products of few rows, everything in one launch
CASES = [
    (1, 1025, 1000, 8, 20, False, "one"), (1, 1500, 4000, 16, 3, False, "one"), (16, 5121, 1003, 16, 50, False, "straight"), (60, 2049, 700, 20, 9, False, "straight"),
    (500, 449, 700, 24, 60, False, "64"), (78, 697, 300, 8, 60, False, "64 cut"), (1000, 100, 4000, 16, 50, False, "128"), (200, 4100, 1029, 16, 50, False, "128 cut"),
    (1306, 350, 5848, 8, 20, False, "256"), (928, 6555, 650, 24, 30, False, "256 cut"), (1165, 350, 6164, 8, 30, False, "256x"), (200, 4100, 8200, 16, 50, False, "256x cut"),
    (90, 12500, 333, 16, 9, False, "64 cut"), (700, 12500, 600, 16, 9, False, "128 cut"),
    (1, 1025, 1000, 8, 20, True, "one"), (16, 5121, 1003, 16, 50, True, "straight"), (60, 2049, 700, 20, 9, True, "straight"),
    (500, 602, 300, 24, 40, True, "64"), (78, 1014, 300, 16, 40, True, "64 cut"), (601, 405, 5389, 8, 30, True, "128"), (73, 2603, 6148, 16, 60, True, "128 cut"),
    (978, 334, 8163, 16, 5, True, "256"), (201, 5784, 7728, 8, 60, True, "256 cut"), (2030, 288, 4369, 16, 60, True, "256x"), (200, 4100, 8200, 16, 50, True, "256x cut"),
]

# The error of a score, relative to the root of the sum of its products' squares (shared ones and the adapter's), in the mean square. An operand of 22 bits is off by 2^-23 /
# sqrt(3) of each number, four of them, and products of pairs of terms that are left out are below 2^-24: together below 2^-21.5. B's part leaves out less than 2^-21 of each
# product. Sums in 32 bits, rounded once for 16 products: n / 16 roundings of 2^-25 of a partial sum, whose size grows with the square root of its length: 2^-25 sqrt(n / 32), for
# 12500 products 2^-20.7; three terms of each product: below 2^-20. Together below 2^-19; twice that is allowed. (One operand of 11 bits: 2^-12 / sqrt(3) = 2^-12.8, of one of
# two equal parts 2^-13.3. 16 bits instead of 24, cut off: between 0 and 2^-15 of a number, 2^-16 in the mean, 2^-16.5 of one of two equal parts.)
MEAN = 2.0 ** -18
# A single score, relative to the same: sixteen times that.
SINGLE = 2.0 ** -14


def problem(N, K, C, rank, count, bf16, device="cpu"):
    """X, W, A, B, scales (float32, numbers that bfloat16 has if asked for), adapters; the adapters' part is about as large as the shared one."""
    gen = torch.Generator().manual_seed(N + 3 * K + 5 * C)
    keep = (lambda t: t.bfloat16().float()) if bf16 else (lambda t: t)
    X, W, A, B = (keep(torch.randn(*s, generator=gen)).to(device) for s in ((N, K), (C, K), (count, rank, K), (count, C, rank)))
    B = keep(B / rank ** 0.5)
    return X, W, A, B, (1.0 + torch.arange(count) % 3 * 0.5).to(device), torch.randint(-1 if N > 1 else 0, count, (N,), generator=gen).to(device)


def scores(X, W, A, B, scale, adapters, x=lambda v: v, w=lambda v: v, a=lambda v: v, s=lambda v: v, b=lambda v: v):
    """The scores in 64 bits, and the size that their errors are measured by; x, w, a, s, b: what operands and inner products are rounded by."""
    X, W, A, B, scale = (t.double() for t in (X, W, A, B, scale))
    out = x(X) @ w(W).T
    size = X.square() @ W.square().T
    for e in range(len(A)):
        at = (adapters == e).nonzero()[:, 0]
        if len(at) > 0:
            inner = x(X[at]) @ a(A[e]).T * scale[e]
            out[at] += s(inner) @ b(B[e]).T
            size[at] += inner.square() @ B[e].square().T
    return out, size.sqrt()


def errors(have, want, size):
    """In the mean square over all scores, and the largest one."""
    e = ((have.double() - want) / size).cpu().numpy()
    return float(np.sqrt((e * e).mean())), float(np.abs(e).max())
