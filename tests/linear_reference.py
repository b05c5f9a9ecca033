"""The operators of linear models from their formulas, in 64 bits on the CPU, and how far results of the stated arithmetic may be
from them."""
from __future__ import annotations

import numpy as np


def xent(Phi, W, labels, scale):
    """Loss, gradients and what their bounds need; rows with negative labels are zeroed."""
    Phi, W, labels = np.array(Phi, dtype=np.float64), np.asarray(W, dtype=np.float64), np.asarray(labels)
    there = labels >= 0
    Phi[~there] = 0.0
    s = np.where(there, np.asarray(scale, dtype=np.float64), 0.0)
    l = Phi @ W.T
    top = l.max(1)
    e = np.exp(l - top[:, None])
    total = e.sum(1)
    at = np.where(there, labels, 0)
    rows = np.arange(len(labels))
    loss = np.where(there, np.log(total) + top - l[rows, at], 0.0)
    p = e / total[:, None]
    g = p.copy()
    g[rows, at] -= 1.0
    g[~there] = 0.0
    return {"loss": loss, "dPhi": (g * s[:, None]) @ W, "dW": (g * s[:, None]).T @ Phi, "l": l, "p": p, "g": g, "s": s, "Phi": Phi, "W": W}


def xent_bounds(r, bf16):
    """Elementwise bounds of the errors of loss, dPhi, dW.

    A float32 operand enters with a relative error of 2^-22 or an absolute one of 2^-38 of the largest of its row, a product leaves
    out 2^-22; a bfloat16 operand enters whole down to 2^-38 of the largest. A sum of n products in 32 bits is off by at most n 2^-24 of the sum of
    magnitudes, for each term of the products (three of them). exp, log and divisions: a few units of 2^-24, exp's argument rounded at 2^-24 of itself.
    G for the gradients' products: 22 bits (11 for bfloat16), or 2^-38 of the largest |s_n G_nc| times the largest number of the row it
    multiplies; results are rounded to their type."""
    Phi, W, s = np.abs(r["Phi"]), np.abs(r["W"]), np.abs(r["s"])
    N, K = Phi.shape
    C = W.shape[0]
    u = 2.0 ** -24
    big_phi, big_w = Phi.max(1, initial=0.0), W.max(1, initial=0.0)
    operand = 0.0 if bf16 else 3 * 2.0 ** -22
    terms = 1 if bf16 else 3
    tiny = 2.0 ** -37
    dl = (operand + terms * (K + 4) * u) * (Phi @ W.T) + tiny * (big_phi[:, None] * W.sum(1)[None, :] + Phi.sum(1)[:, None] * big_w[None, :])
    worst = dl.max(1)
    size = np.abs(r["l"]).max(1)
    d_loss = 2 * worst + 8 * u * (1 + size) + 8 * u * np.abs(r["loss"]) + (C // 64 + 64) * u
    # p = exp(l - top) / sum
    dp = r["p"] * (2 * worst[:, None] + 4 * u * np.abs(r["l"] - r["l"].max(1)[:, None]) + (C // 64 + 80) * u) + 2.0 ** -126
    g_bits = 2.0 ** -11 if bf16 else 3 * 2.0 ** -22
    dg = dp + g_bits * np.abs(r["g"])
    g = np.abs(r["g"])
    out = 2.0 ** -8 if bf16 else 2 * u
    reach = (g * big_w[None, :]).max(1) + big_w[np.argmax(g, 1)]
    d_phi = s[:, None] * (dg @ W + (operand + terms * (C + 4) * u) * (g @ W) + tiny * (reach[:, None] * C + g @ np.repeat(big_w[:, None], K, 1)))
    sg, sdg = g * s[:, None], dg * s[:, None]
    reach = (s * big_phi).max(initial=0.0)
    d_w = sdg.T @ Phi + (operand + terms * (N + 4) * u) * (sg.T @ Phi) + tiny * (N * reach + sg.T @ np.repeat(big_phi[:, None], K, 1))
    least = 2.0 ** -133 if bf16 else 2.0 ** -140
    return d_loss, d_phi + out * np.abs(r["dPhi"]) + least, d_w + out * np.abs(r["dW"]) + least
