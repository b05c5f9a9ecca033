"""What the GPU tests of scores with adapters are there for: that their sizes are worked on in the ways they name, that there is one for every kernel, and that their limits
tell operands of 22 bits from operands of 11. No GPU."""
import pytest
import torch

from tests.adapters_accuracy import CASES, MEAN, errors, problem, scores
from tests.linear_launches import launches
from tests.test_gpu_adapters import CASES as OTHER_CASES

OURS = ("one_kernel<", "place_kernel<", "order_kernel", "finish_kernel", "join_kernel<")


def _way(names):
    tiles = [n for n in names if n.startswith("plane_product<")]
    if any(n.startswith("one_kernel<") for n in names):
        return "one"
    if not tiles:
        return "straight"
    mode, edge = tiles[0].split("<")[1].split(", ")[:2]
    return edge + ("x" if ", true, " in tiles[0] else "") + (" cut" if "Parts" in tiles[0] else "")


def test_every_way_is_tested(tmp_path):
    out, known = launches(tmp_path, [("scores", *c[:6], 1.0) for c in CASES])
    for case, names in zip(CASES, out):
        assert _way(names) == case[6], (case, names)
    for bf16 in (False, True):
        assert {c[6] for c in CASES if c[5] == bf16} == {"one", "straight"} | {e + cut for e in ("64", "128", "256", "256x") for cut in ("", " cut")}
    others, _ = launches(tmp_path, [("scores", *c, bf16, 1.0) for c in OTHER_CASES for bf16 in (0, 1)])
    wanted = {k for k in known if k.startswith(OURS) or "Adapted" in k or "Parts" in k or k.startswith(("few_kernel<true", "few_kernel<false"))}
    assert len(wanted) > 30 and wanted - {n for names in out + others for n in names} == set()


def _rounded(bits, cut=False):
    """Numbers of so many significand bits, to the nearest, or cut off."""
    def of(v):
        m, e = torch.frexp(v)
        m = m * 2.0 ** bits
        return torch.ldexp(m.trunc() if cut else m.round(), e - bits)
    return of


SMALL = [(300, 700, 400, 16, 9), (20, 5121, 300, 8, 9), (70, 12500, 60, 16, 4)]


@pytest.mark.parametrize("size", SMALL)
@pytest.mark.parametrize("lost", ["nothing", "x", "w", "a", "s", "b"])
def test_the_limit_tells_one_term_from_two(size, lost):
    """Operands rounded as two terms hold them (22 bits), inner products and B as three that are cut off (24), and one of them with a term less."""
    data = problem(*size, False)
    want, by = scores(*data)
    rounds = {n: _rounded(22) for n in "xwa"} | {n: _rounded(24, True) for n in "sb"}
    if lost != "nothing":
        rounds[lost] = _rounded(11) if lost in "xwa" else _rounded(16, True)
    assert (errors(scores(*data, **rounds)[0], want, by)[0] > MEAN) == (lost != "nothing")


@pytest.mark.parametrize("case", [c for c in CASES if not c[5]] + [c + (False, "") for c in OTHER_CASES])
def test_one_term_is_not_enough_in_any_float32_case(case):
    """Both shared operands as one term, scaled by their row's largest number, without an adapter. What single numbers lose is a matter of luck: of fewer
    than eight all may be lost by less."""
    N, K, C = case[:3]
    rows, classes = min(N, 64), min(C, 512)
    X, W, A, B, scale, adapters = problem(N, K, C, *case[3:5], False)
    X, W, none = X[:rows], W[:classes], torch.full((rows,), -1)
    want, by = scores(X, W, A, B, scale, none)
    half = lambda v: torch.ldexp(torch.ldexp(v, 15 - torch.frexp(v.abs().amax(1, keepdim=True))[1]).half().double(), torch.frexp(v.abs().amax(1, keepdim=True))[1] - 15)   # noqa: E731
    assert errors(scores(X, W, A, B, scale, none, x=half, w=half)[0], want, by)[0] > MEAN or min(rows * K, classes * K) < 8
