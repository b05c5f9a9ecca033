"""What the GPU tests of packed softmax cross entropies are there for: that their sizes are worked on in the tiles they name, and that their limits tell operands of 22 bits from
operands of 11. No GPU."""
import re

import numpy as np
import pytest

from tests import launches
from tests.linear_reference import xent
from tests.xent_accuracy import CASES, MEAN, MEAN_BF16, mean_error


def _tiles(names, epilogue):
    """Edges of the launched products' tiles, 256x with a joined block, and the products' modes."""
    found = [re.search(r"plane_product<\((?:plane::)?PlaneMode\)(\d), (\d+), \d+, \d+, \d+, \d+, (true|false), (\w+)>", n) for n in names]
    return {(m.group(2) + ("x" if m.group(3) == "true" else ""), int(m.group(1))) for m in found if m and m.group(4) == epilogue}


def test_every_kind_of_tile_is_tested(tmp_path):
    runs = launches.of_softmax_xent(tmp_path, [c[:4] + (3,) for c in CASES] + [c[:4] + (0,) for c in CASES])
    for case, both, alone in zip(CASES, runs, runs[len(CASES):]):
        bf16, scores, gradients, cut = case[3:]
        assert _tiles(both, "Scores") == {(scores, 0 if bf16 else 1)} and _tiles(both, "Gradient") == {(gradients, 3 if bf16 else 1)}, case
        assert any("add_kernel" in n for n in both) == cut, case
        assert len(_tiles(alone, "Scores")) == 1 and not _tiles(alone, "Gradient")
    for bf16 in (False, True):
        assert {c[4] for c in CASES if c[3] == bf16} == {"64", "128", "256", "256x"}
        assert {c[5] for c in CASES if c[3] == bf16} == {"64", "128", "256", "256x"}
        assert {c[5] for c in CASES if c[3] == bf16 and c[6]} >= {"64", "128", "256", "256x"}


def _rounded(x, bits):
    """Numbers of so many significand bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 2.0 ** bits), e - bits)


def _bf16(x):
    return _rounded(x, 8)


@pytest.mark.parametrize("lost", ["nothing", "Phi in the scores", "W in the scores", "G", "W in dPhi", "Phi in dW"])
@pytest.mark.parametrize("bf16", [False, True])
def test_the_limits_tell_one_term_from_two(lost, bf16):
    """The formula with operands rounded as two terms hold them (22 bits), and with one of them rounded to one term (11 bits)."""
    rng = np.random.default_rng(0)
    N, K, C = 500, 300, 700
    x, w, y, s = rng.standard_normal((N, K)) / K ** 0.5, rng.standard_normal((C, K)) * 2, rng.integers(0, C, N), 0.5 + rng.random(N)
    keep = _bf16 if bf16 else (lambda v: v.astype(np.float32).astype(np.float64))
    x, w = keep(x), keep(w)
    want = xent(x, w, y, s)
    bits = lambda name: 11 if lost == name else 22                                  # noqa: E731
    l = _rounded(x, bits("Phi in the scores")) @ _rounded(w, bits("W in the scores")).T
    top = l.max(1, keepdims=True)
    e = np.exp(l - top)
    loss = np.log(e.sum(1)) + top[:, 0] - l[np.arange(N), y]
    g = e / e.sum(1, keepdims=True)
    g[np.arange(N), y] -= 1
    g = _rounded(g * s[:, None], bits("G"))
    dPhi, dW = g @ _rounded(w, bits("W in dPhi")), g.T @ _rounded(x, bits("Phi in dW"))
    fails = [mean_error(loss, want["loss"]) > MEAN]
    for have, exact in ((dPhi, want["dPhi"]), (dW, want["dW"])):
        fails.append(mean_error(_bf16(have), _bf16(exact)) > MEAN_BF16 if bf16 else mean_error(have, exact) > MEAN)
    # bfloat16 operands are whole in one term, and there only G can be lost
    expected = {"nothing": [], "Phi in the scores": [0], "W in the scores": [0], "G": [1, 2], "W in dPhi": [1], "Phi in dW": [2]}[lost]
    if bf16 and lost != "G":
        expected = []
    assert all(fails[k] for k in expected) and (expected or not any(fails))
