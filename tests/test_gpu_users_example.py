"""The classifier example with a layer norm, dropout and users' adapters: that it runs, and that an adapter's gradients are those of the loss."""
import importlib.util
import os

import pytest
import torch

import paper_2501_07145_amd as rfsf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location("softmax_classifier", os.path.join(ROOT, "examples", "softmax_classifier.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


@pytest.mark.parametrize("norm,dropout", [(True, 0.2), (True, 0.0), (False, 0.2)])
def test_runs(norm, dropout):
    r = _example().run(classes=6, n_train=300, n_test=100, steps=40, norm=norm, dropout=dropout, users=3, say=lambda text: None)
    assert abs(r["first_loss"] - 1.791759) < 1e-4                # log 6: all weights zero
    for name in ("accuracy", "accuracy_int8", "accuracy_users"):
        assert 0.0 <= r[name] <= 1.0
    assert r["users_one_at_a_time"] < 1e-3


def test_gradients_of_an_adapter_against_differences():
    gen = torch.Generator(device="cuda").manual_seed(4)
    Phi, W, A, B = (torch.randn(*s, generator=gen, device="cuda") for s in ((50, 33), (7, 33), (3, 33), (7, 3)))
    y = torch.randint(0, 7, (50,), generator=gen, device="cuda")
    _, _, dW = rfsf.rfsf_softmax_xent(Phi, W + B @ A, y, need_dW=True)
    dA, dB = rfsf.rfsf_ts_gram(B.T.contiguous(), dW.T.contiguous()), rfsf.rfsf_ts_gram(dW, A)

    def loss(a, b):
        return torch.nn.functional.cross_entropy(Phi.double() @ (W.double() + b @ a).T, y)

    a, b, h = A.double(), B.double(), 1e-5
    for grad, place in ((dA, 0), (dB, 1)):
        d = torch.randn(grad.shape, generator=gen, device="cuda", dtype=torch.float64)
        slope = (loss(a + h * d, b) - loss(a - h * d, b) if place == 0 else loss(a, b + h * d) - loss(a, b - h * d)) / (2 * h)
        # gradients of 32 bits, sums of up to 50 terms of either sign
        assert abs(float(slope - (grad.double() * d).sum())) < 200 * 2.0 ** -24 * float((grad.double() * d).abs().sum()) + 1e-8
