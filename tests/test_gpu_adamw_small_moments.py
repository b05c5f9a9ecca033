"""AdamW with 8-bit states on the GPU where v is very small, or much smaller than the largest of its block: a v above zero stays above zero."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf

pytestmark = pytest.mark.gpu

F = np.float32
BETAS = (0.9, 0.995)


def _codes_of_v(v):
    """Codes and scales from the definition in 32-bit operations: the nearest code to (v / scale)^(1/4), at least the first one that does not stand for
    zero in 32 bits. Quotients of numbers below 2^-119 are of 2^64 times them."""
    v = v.reshape(-1, 256)
    top = v.max(1, keepdims=True)
    lift = np.where(top < F(2.0 ** -119), F(2.0 ** 64), F(1))
    inverse = np.where(top > 0, F(1) / np.where(top > 0, top * lift, F(1)), F(0)).astype(F)
    code = np.minimum(np.rint(np.sqrt(np.sqrt((v * lift) * inverse)) * F(255)), F(255))
    least = np.ones_like(top)
    small = (top > 0) & (top < F(2.0 ** -116))
    least[small] = np.ceil(np.sqrt(np.sqrt(F(2.0 ** -85) / (top[small] * F(2.0 ** 64)))) * F(255))
    return np.where(v > 0, np.maximum(code, np.minimum(least, F(255))), code).reshape(-1).astype(np.uint8), top[:, 0]


def _gradients(kind, blocks, seed):
    """256 numbers a block, their magnitudes spread over the block's range of powers of two."""
    rng = np.random.default_rng(seed)
    low, high = {"tiny": (-70, -56), "least": (-70, -69), "wide": (-40, 20), "widest": (-68, 30), "threshold": (-60, -54)}[kind]
    top = rng.uniform(low, high, (blocks, 1)) if not kind.startswith("wide") else np.full((blocks, 1), high)
    g = np.exp2(rng.uniform(low, top, (blocks, 256))) * rng.choice([-1.0, 1.0], (blocks, 256))
    g[:, ::17] = 0
    return g.reshape(-1).astype(F)


@pytest.mark.parametrize("kind", ["tiny", "least", "wide", "widest", "threshold"])
def test_v_above_zero_stays_above_zero(kind):
    """The codes are the definition's; what they stand for is above zero exactly where v is; and with eps = 0 a step without gradients, which divides m by the
    root of what the codes stand for, leaves all parameters finite."""
    g = _gradients(kind, 50, 3)
    p = torch.randn(len(g), generator=torch.Generator().manual_seed(1)).cuda()
    opt = rfsf.RfsfAdamW([p], state_bits=8)
    opt.step([torch.from_numpy(g).cuda()], 1, 1e-3, betas=BETAS, eps=1e-8)
    v = (g * F(1 - BETAS[1])) * g
    assert np.all((v > 0) == (g != 0))                                   # (in 32 bits, as the step has it)
    code, scale = _codes_of_v(v)
    assert np.array_equal(opt.state["v_scale"][0].cpu().numpy(), scale) and np.array_equal(opt.state["v"][0].cpu().numpy(), code)
    have = opt.moments()[1][0].cpu().numpy()
    assert np.all((have > 0) == (v > 0))
    if not kind.startswith("wide"):
        q = torch.where(torch.from_numpy(g).cuda() == 0, torch.full_like(p, 1e-4), torch.zeros_like(p))       # (numbers without a past need a gradient for eps = 0)
        opt.step([q], 2, 1e-3, betas=BETAS, eps=0.0)
    else:
        opt.step([torch.where(torch.from_numpy(g).cuda() == 0, torch.ones_like(p), torch.zeros_like(p))], 2, 1e-3, betas=BETAS, eps=0.0)
    assert torch.isfinite(p).all()


def test_blocks_of_zeros_and_blocks_that_are_not_finite():
    g = torch.zeros(768, device="cuda")
    g[300] = float("inf")
    g[600] = 1e-20
    p = torch.zeros(768, device="cuda")
    opt = rfsf.RfsfAdamW([p], state_bits=8)
    opt.step([g], 1, 1e-3)
    scale, code = opt.state["v_scale"][0].cpu(), opt.state["v"][0].cpu()
    assert scale[0] == 0 and torch.isnan(scale[1]) and scale[2] > 0
    assert torch.all(code[:512] == 0) and code[600] == 255 and int((code != 0).sum()) == 1
