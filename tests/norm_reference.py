"""Layer norm and dropout from their formulas, in 64 bits on the CPU, and how far results of the stated arithmetic may be from them."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
BF16 = 2.0 ** -8            # half a step of bfloat16


def philox(counter, key):
    """Philox 4x32 of 10 rounds: counter [..., 4], key (two words), whole numbers below 2^32."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [int(v) for v in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def numbers(N, K, seed, offset=0, first_row=0):
    """The 16 bits that belong to each place of N rows of K columns."""
    groups = (K + 7) // 8
    c = np.zeros((N, groups, 4), dtype=np.uint64)
    c[..., 0] = np.arange(groups, dtype=np.uint64)[None]
    c[..., 1] = (first_row + np.arange(N, dtype=np.uint64))[:, None]
    c[..., 2], c[..., 3] = offset & 0xFFFFFFFF, offset >> 32 & 0xFFFFFFFF
    w = philox(c, (seed & 0xFFFFFFFF, seed >> 32))
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(N, 8 * groups)[:, :K].astype(np.int64)


def mask(N, K, p, seed, offset=0, first_row=0):
    """What dropout multiplies each place by."""
    t = int(np.rint(65536 * p))
    keep = numbers(N, K, seed, offset, first_row) >= t
    return np.where(keep, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)


def norm(X, gain, offset, eps, factor):
    """mean, rstd, Y."""
    X = np.asarray(X, dtype=np.float64)
    mean = X.mean(1)
    d = X - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(1) + eps)
    return mean, rstd, (d * rstd[:, None] * gain + offset) * factor


def norm_bounds(X, gain, offset, eps, factor, bf16):
    """Bounds of the errors of mean, rstd, Y. A sum over K columns is made of at most n = 64 + K / 512 additions one after another.

    The first mean is off by at most (n + 2) U mean|x| = t, which then is part of every x less it; what is left, rest, is the mean of these differences d, off by (n + 3) U
    mean|d| = c. var = mean(d^2) - rest^2 is off by (n + 3) U mean(d^2) + 2 |rest| c + 2 U rest^2. Then a sum, a root and a quotient, each rounded."""
    X = np.asarray(X, dtype=np.float64)
    n = 64 + X.shape[1] // 512
    mean, rstd, Y = norm(X, gain, offset, eps, factor)
    d = np.abs(X - mean[:, None])
    t = (n + 2) * U * np.abs(X).mean(1)
    c = (n + 3) * U * (d.mean(1) + t)
    var = (d * d).mean(1)
    d_var = (n + 3) * U * (var + 2 * t * d.mean(1) + t * t) + 2 * t * c + 2 * U * t * t
    d_rstd = rstd * (0.6 * d_var / (var + eps) + 4 * U)
    d_z = rstd[:, None] * (2 * U * (d + t[:, None]) + c[:, None]) + d * (d_rstd + U * rstd)[:, None]
    y = np.abs(Y)
    d_y = (np.abs(gain) * d_z + U * (np.abs(gain) * d * rstd[:, None] + np.abs(offset))) * np.abs(factor) + 2 * U * y
    if bf16:
        d_y = d_y * (1 + BF16) + BF16 * y
    return c + U * np.abs(mean) + 2.0 ** -149, d_rstd, d_y + (2.0 ** -133 if bf16 else 2.0 ** -148)


def back(X, mean, rstd, gain, dY, factor):
    """dX, dgain, doffset for given statistics."""
    X, mean, rstd, dY = (np.asarray(v, dtype=np.float64) for v in (X, mean, rstd, dY))
    z = (X - mean[:, None]) * rstd[:, None]
    h = dY * factor
    g = h * gain
    dX = rstd[:, None] * (g - g.mean(1)[:, None] - z * (g * z).mean(1)[:, None])
    return dX, (h * z).sum(0), h.sum(0)


def back_bounds(X, mean, rstd, gain, dY, factor, bf16):
    """Bounds of their errors. z has two roundings, h two (the factor's own and the product's), g one more. A sum over K columns is made of at most n = 64 + K /
    512 additions one after another, one over N rows of 128 + N / 128."""
    X, mean, rstd, dY = (np.asarray(v, dtype=np.float64) for v in (X, mean, rstd, dY))
    N, K = X.shape
    n, rows = 64 + K // 512, 128 + N // 128
    z = np.abs((X - mean[:, None]) * rstd[:, None])
    h = np.abs(dY * factor)
    g = np.abs(h * gain)
    sum_g, sum_gz = g.mean(1)[:, None], (g * z).mean(1)[:, None]
    dX, dgain, doffset = back(X, mean, rstd, gain, dY, factor)
    d_x = rstd[:, None] * ((3 + 3) * U * g + (n + 8) * U * sum_g + z * (n + 14) * U * sum_gz) + 2 * U * np.abs(dX)
    if bf16:
        d_x = d_x * (1 + BF16) + BF16 * np.abs(dX)
    least = 2.0 ** -133 if bf16 else 2.0 ** -148
    return d_x + least, (rows + 6) * U * (h * z).sum(0) + 2.0 ** -148 * N, (rows + 3) * U * h.sum(0) + 2.0 ** -148 * N
