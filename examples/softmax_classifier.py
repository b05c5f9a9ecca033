"""A softmax classifier on signature features, trained and served on the GPU.

Sequences of several classes (Brownian paths with a drift of the class's own) become RFSF-TS features, normalised by levels. A
linear softmax classifier is trained on them: rfsf_softmax_xent gives the loss and the gradient of the weights, RfsfAdamW takes the
steps, with states of 8 bits by default. With --norm the features go through a layer norm with gains and offsets that are trained too, with --dropout through
dropout behind it. The trained weights are then held as 8-bit integers, and rfsf_int8_gram scores new
sequences against them, as a batch and one at a time; so are the training features, for kernel values of new sequences against
stored ones. With --users each of some users has labels of their own (the classes' names permuted), for which a low-rank adapter beside the shared weights is trained; all
users' requests are then answered in one call.

  python examples/softmax_classifier.py [--classes 10] [--steps 200] [--state-bits 8|32] [--norm] [--dropout 0.1] [--users 5]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2501_07145_amd as rfsf  # noqa: E402


def sequences(n, L, d, classes, drifts, gen):
    """n paths of L points in d dimensions on [0, 1], and their classes."""
    y = torch.randint(0, classes, (n,), generator=gen, device="cuda")
    steps = torch.randn(n, L - 1, d, generator=gen, device="cuda") / (L - 1) ** 0.5
    steps += drifts[y][:, None, :] / (L - 1)
    return torch.cat([torch.zeros(n, 1, d, device="cuda"), steps.cumsum(1)], 1).contiguous(), y


def features(X, tables, D, M, lengthscale):
    Phi = rfsf.rfsf_ts_features(X, tables["W"], tables["hash"], tables["sign"], lengthscale, D)
    return rfsf.rfsf_ts_normalize_features(Phi, M, D)


def adapter_of(Phi, W, y, rank, steps=60, lr=0.05):
    """(A, B) of an adapter B A of this rank that fits W + B A to labels y: steps on the sum's gradient dW, of which B gets dW A^T and A gets B^T dW."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    A, B = torch.randn(rank, W.shape[1], generator=gen, device="cuda") / W.shape[1] ** 0.5, torch.zeros(W.shape[0], rank, device="cuda")
    optimizer = rfsf.RfsfAdamW([A, B])
    for t in range(1, steps + 1):
        merged = W + rfsf.rfsf_ts_gram(B, A.T.contiguous())
        _, _, dW = rfsf.rfsf_softmax_xent(Phi, merged, y, need_dW=True)
        dA, dB = rfsf.rfsf_ts_gram(B.T.contiguous(), dW.T.contiguous()), rfsf.rfsf_ts_gram(dW, A)
        optimizer.step([dA, dB], t, lr, weight_decay=0.0)
    return A, B


def run(classes=10, n_train=2000, n_test=500, L=50, d=4, M=3, F=64, D=128, steps=200, lr=2e-2, state_bits=8, seed=0, say=print, norm=False, dropout=0.0, users=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    drifts = 4.0 * torch.randn(classes, d, generator=gen, device="cuda")
    X, y = sequences(n_train, L, d, classes, drifts, gen)
    X_new, y_new = sequences(n_test, L, d, classes, drifts, gen)
    tables = {"W": torch.randn(M, d, F, generator=gen, device="cuda"),
              "hash": torch.randint(0, D, (M, 2 * F), generator=gen, device="cuda", dtype=torch.int32),
              "sign": torch.randint(0, 2, (M, 2 * F), generator=gen, device="cuda").float() * 2 - 1}
    lengthscale = 2.0 * d ** 0.5
    Phi = features(X, tables, D, M, lengthscale)
    Phi_new = features(X_new, tables, D, M, lengthscale)
    K = Phi.shape[1]

    W, dW, loss = (torch.zeros(*shape, device="cuda") for shape in ((classes, K), (classes, K), (n_train,)))
    recommended, _ = rfsf.rfsf_softmax_xent_workspace_bytes(n_train, K, classes, need_dW=True)
    workspace = torch.empty(recommended, dtype=torch.uint8, device="cuda")
    gain, offset = torch.ones(K, device="cuda"), torch.zeros(K, device="cuda")
    optimizer = rfsf.RfsfAdamW([W, gain, offset] if norm else [W], state_bits=state_bits)
    first = last = None
    for t in range(1, steps + 1):
        rate = lr * (1 - (t - 1) / steps)
        mask = rfsf.RfsfDropout(dropout, seed, offset=t) if dropout > 0 else None
        if norm:
            Y, mean, rstd = rfsf.rfsf_layer_norm(Phi, gain, offset, dropout=mask)
            _, dY, _ = rfsf.rfsf_softmax_xent(Y, W, y, need_dPhi=True, need_dW=True, loss=loss, dW=dW)
            _, dgain, doffset = rfsf.rfsf_layer_norm_backward(Phi, mean, rstd, dY, gain=gain, dropout=mask, need_dX=False)
            optimizer.step([dW, dgain, doffset], t, rate, weight_decay=1e-4)
        else:
            rows = rfsf.rfsf_dropout(Phi, mask) if mask is not None else Phi
            rfsf.rfsf_softmax_xent(rows, W, y, need_dW=True, loss=loss, dW=dW, workspace=workspace)
            optimizer.step([dW], t, rate, weight_decay=1e-4)
        if t in (1, steps):
            last = float(loss.mean())
            first = last if first is None else first
    if norm:
        Phi, Phi_new = (rfsf.rfsf_layer_norm(rows, gain, offset)[0] for rows in (Phi, Phi_new))
    test_loss, _, _ = rfsf.rfsf_softmax_xent(Phi_new, W, y_new)

    def share(scores):
        return float((scores.argmax(1) == y_new).float().mean())

    codes, scales = rfsf.rfsf_int8_quantize(W)
    batch = rfsf.rfsf_int8_gram(Phi_new, codes, scales)
    one = torch.cat([rfsf.rfsf_int8_gram(Phi_new[i:i + 1], codes, scales) for i in range(8)])
    stored, stored_scales = rfsf.rfsf_int8_quantize(Phi)
    kernel = rfsf.rfsf_int8_gram(Phi_new, stored, stored_scales)
    result = {"first_loss": first, "last_loss": last, "test_loss": float(test_loss.mean()), "accuracy": share(rfsf.rfsf_ts_gram(Phi_new, W)),
              "accuracy_int8": share(batch), "one_at_a_time": bool(torch.equal(one, batch[:8])),
              "kernel_error": float((kernel - rfsf.rfsf_ts_gram(Phi_new, Phi)).abs().max())}
    if users > 0:
        names = [torch.randperm(classes, generator=gen, device="cuda") for _ in range(users)]
        served = rfsf.RfsfAdapters(W, users, rank=min(8, classes))
        for u in range(users):
            served.set(u, *adapter_of(Phi, W, names[u][y], served.rank))
        who = torch.randint(0, users, (n_test,), generator=gen, device="cuda")
        wanted = torch.stack(names)[who, y_new]
        scores = served.scores(Phi_new, who)
        result["accuracy_users"] = float((scores.argmax(1) == wanted).float().mean())
        result["users_one_at_a_time"] = float((torch.cat([served.scores(Phi_new[i:i + 1], who[i:i + 1]) for i in range(8)]) - scores[:8]).abs().max())
        say(f"{users} users with names of their own for the classes, adapters of rank {served.rank}: accuracy {result['accuracy_users']:.3f}")
    say(f"{n_train} sequences, {K} columns, {classes} classes, {state_bits}-bit states: loss {first:.3f} -> {last:.3f}, on new sequences "
        f"{result['test_loss']:.3f}")
    say(f"accuracy on new sequences {result['accuracy']:.3f}, with 8-bit weights {result['accuracy_int8']:.3f}; kernel values against stored 8-bit "
        f"features within {result['kernel_error']:.4f}")
    return result


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--classes", type=int, default=10)
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    p.add_argument("--norm", action="store_true")
    p.add_argument("--dropout", type=float, default=0.0)
    p.add_argument("--users", type=int, default=0)
    a = p.parse_args()
    run(classes=a.classes, steps=a.steps, state_bits=a.state_bits, norm=a.norm, dropout=a.dropout, users=a.users)
