"""Scores with low-rank adapters from their formula, in 64 bits on the CPU, and how far results of the stated arithmetic may be from them."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24


def scores(X, W, A, B, scale, adapters):
    """A [count, rank, K], B [count, C, rank], scale [count]; rows with adapters that do not exist are NaN."""
    X, W = np.asarray(X, dtype=np.float64), np.asarray(W, dtype=np.float64)
    out = X @ W.T
    for a in np.unique(adapters):
        if 0 <= a < len(A):
            at = adapters == a
            out[at] += scale[a] * ((X[at] @ np.asarray(A[a], dtype=np.float64).T) @ np.asarray(B[a], dtype=np.float64).T)
    out[adapters >= len(A)] = np.nan
    return out


def _product_bound(X, Y, bf16):
    """Bound of the error of X Y^T: a float32 operand enters with a relative error of 2^-22 or an absolute one of 2^-38 of the largest of its row, a product
    leaves out 2^-22; a bfloat16 operand enters whole down to 2^-38 of the largest. A sum of K products in 32 bits is off by at most K 2^-24 of the sum of
    magnitudes, for each term of the products (three of them)."""
    X, Y = np.abs(np.asarray(X, dtype=np.float64)), np.abs(np.asarray(Y, dtype=np.float64))
    K = X.shape[1]
    operand, terms, tiny = (0.0, 1, 2.0 ** -37) if bf16 else (3 * 2.0 ** -22, 3, 2.0 ** -37)
    big_x, big_y = X.max(1), Y.max(1)
    return (operand + terms * (K + 4) * U) * (X @ Y.T) + tiny * (big_x[:, None] * Y.sum(1)[None] + X.sum(1)[:, None] * big_y[None])


def bounds(X, W, A, B, scale, adapters, bf16):
    """The inner products are two roundings further (their scale), enter their sum with B whole, of which every product and addition is rounded; up
    to six terms of a product (B as it is: the products of its parts) are added up one after another. The result is the sum of both, rounded."""
    shared = _product_bound(X, W, bf16)
    out = shared + 2 * U * np.abs(np.asarray(X, dtype=np.float64) @ np.asarray(W, dtype=np.float64).T)
    for a in np.unique(adapters):
        if 0 <= a < len(A):
            at = adapters == a
            x, b = np.asarray(X[at], dtype=np.float64), np.abs(np.asarray(B[a], dtype=np.float64))
            s = np.abs(scale[a] * (x @ np.asarray(A[a], dtype=np.float64).T))
            ds = abs(scale[a]) * _product_bound(x, A[a], bf16) + 2 * U * s
            rank = b.shape[1]
            out[at] += ds @ b.T * (1 + 2.0 ** -10) + 6 * (rank + 8) * U * (s @ b.T)
    return out + 2.0 ** -120
