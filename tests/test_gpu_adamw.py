"""AdamW steps on the GPU against the formula in 64 bits, and 8-bit states against their definition."""
import numpy as np
import pytest
import torch

import paper_2501_07145_amd as rfsf

pytestmark = pytest.mark.gpu

SETTINGS = dict(lr=2e-3, betas=(0.9, 0.995), eps=1e-8, weight_decay=0.02, grad_scale=0.25)
SIZES = [1, 2, 3, 5, 63, 64, 255, 256, 257, 1000, 4095, 4096, 4097, 8195, 70001]
U = 2.0 ** -24


def _np(t):
    return t.detach().double().cpu().numpy()


def _tensors(sizes, seed, grad_dtype=torch.float32, offset=0):
    """Parameters and gradients; offset: numbers that the tensors start behind an aligned address."""
    gen = torch.Generator().manual_seed(seed)

    def some(n, scale, dtype=torch.float32):
        return (torch.randn(n + offset, generator=gen) * scale).to(dtype).cuda()[offset:]

    return [some(n, 0.1) for n in sizes], [some(n, 1e-2, grad_dtype) for n in sizes]


def _formula(p, g, m, v, step):
    """The new p, m, v in 64 bits, and how far 32 bits may be off: a rounding of 2^-24 for each operation and each constant."""
    b1, b2 = SETTINGS["betas"]
    lr, wd, eps = SETTINGS["lr"], SETTINGS["weight_decay"], SETTINGS["eps"]
    g = g * SETTINGS["grad_scale"]
    m2, v2 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    size = b1 * np.abs(m) + (1 - b1) * np.abs(g)
    c1, c2 = 1 - b1 ** step, 1 - b2 ** step
    root = np.sqrt(v2 / c2) + eps
    p2 = p * (1 - lr * wd) - lr / c1 * m2 / root
    dm, dv = 5 * U * size, 6 * U * v2
    dp = 4 * U * np.abs(p) + lr / c1 * (dm + 16 * U * np.abs(m2)) / root + U * np.abs(p2)
    return (p2, m2, v2), (dp + 1e-40, dm + 1e-40, dv + 1e-40)


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 2])
@pytest.mark.parametrize("copy", [False, True])
def test_32_bit_states(grad_dtype, offset, copy):
    params, _ = _tensors(SIZES, 0, offset=offset)
    copies = [torch.empty(n + offset, dtype=torch.bfloat16, device="cuda")[offset:] for n in SIZES] if copy else None
    opt = rfsf.RfsfAdamW(params, copies=copies)
    for step in (1, 2, 3):
        _, grads = _tensors(SIZES, step, grad_dtype, offset)
        before = [(_np(p), _np(g), _np(m), _np(v)) for p, g, m, v in zip(params, grads, opt.state["m"], opt.state["v"])]
        opt.step(grads, step, **SETTINGS)
        for k, b in enumerate(before):
            want, bound = _formula(*b, step)
            for have, w, d in zip((params[k], opt.state["m"][k], opt.state["v"][k]), want, bound):
                assert np.all(np.abs(_np(have) - w) <= d), (SIZES[k], step)
            if copy:
                assert torch.equal(copies[k], params[k].to(torch.bfloat16))


def _codes_of(m, v):
    """Codes and scales of one tensor's m and v, from the definition in 32-bit operations."""
    f = np.float32
    n = len(m)
    pad = (-n) % 256
    m, v = np.pad(m, (0, pad)).reshape(-1, 256), np.pad(v, (0, pad)).reshape(-1, 256)
    ms, vs = np.abs(m).max(1), v.max(1)
    with np.errstate(divide="ignore"):
        mi = np.where(ms < f(2.0 ** -119), f(0), f(1) / ms).astype(f)[:, None]
        vi = np.where(vs < f(2.0 ** -119), f(0), f(1) / vs).astype(f)[:, None]
    mc = np.minimum(np.rint(np.sqrt(np.abs(m) * mi) * f(127)), f(127))
    share = v * vi
    vc = np.minimum(np.rint(np.sqrt(np.sqrt(share)) * f(255)), f(255))
    vc = np.where(share > 0, np.maximum(vc, f(1)), vc)
    return np.where(m < 0, -mc, mc).reshape(-1)[:n].astype(np.int8), ms, vc.reshape(-1)[:n].astype(np.uint8), vs


def _moments_of(g, m, v):
    """The new m and v in 32-bit operations, each rounded by itself."""
    f = np.float32
    b1, b2 = SETTINGS["betas"]
    g = g * f(SETTINGS["grad_scale"])
    return m * f(b1) + g * f(1 - b1), v * f(b2) + (g * f(1 - b2)) * g


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_8_bit_states(grad_dtype, offset):
    """The step is the formula on the numbers that the codes stand for; the new codes and scales are the definition's to the bit."""
    params, _ = _tensors(SIZES, 0, offset=offset)
    state = {"m": [torch.zeros(n + offset, dtype=torch.int8, device="cuda")[offset:] for n in SIZES],
             "v": [torch.zeros(n + offset, dtype=torch.uint8, device="cuda")[offset:] for n in SIZES]}
    state.update({k: [torch.zeros((n + 255) // 256, device="cuda") for n in SIZES] for k in ("m_scale", "v_scale")})
    opt = rfsf.RfsfAdamW(params, state_bits=8, state=state)
    for step in (1, 2, 3):
        _, grads = _tensors(SIZES, step, grad_dtype, offset)
        grads[3].zero_()                                       # a block without gradients from the start
        m, v = opt.moments()
        for k in range(len(SIZES)):                            # what the codes stand for, to the bit
            u = state["m"][k].cpu().numpy().astype(np.float32) * np.float32(1 / 127)
            w = state["v"][k].cpu().numpy().astype(np.float32) * np.float32(1 / 255)
            w, at = w * w, np.arange(SIZES[k]) // 256
            assert np.array_equal(m[k].cpu().numpy(), (u * np.abs(u)) * state["m_scale"][k].cpu().numpy()[at])
            assert np.array_equal(v[k].cpu().numpy(), (w * w) * state["v_scale"][k].cpu().numpy()[at])
        before = [(_np(p), _np(g), _np(a), _np(b)) for p, g, a, b in zip(params, grads, m, v)]
        opt.step(grads, step, **SETTINGS)
        for k, b in enumerate(before):
            want, bound = _formula(*b, step)
            assert np.all(np.abs(_np(params[k]) - want[0]) <= bound[0]), (SIZES[k], step)
            m2, v2 = _moments_of(*(x.astype(np.float32) for x in b[1:]))
            assert m2.dtype == np.float32 and np.all(np.abs(m2 - want[1]) <= bound[1]) and np.all(np.abs(v2 - want[2]) <= bound[2])
            for name, code in zip(("m", "m_scale", "v", "v_scale"), _codes_of(m2, v2)):
                assert np.array_equal(state[name][k].cpu().numpy(), code), (name, SIZES[k], step)
        assert torch.all(state["m"][3] == 0) and torch.all(state["v"][3] == 0)


def test_more_tensors_than_a_launch_describes():
    sizes = [1 + (k * 37) % 600 for k in range(131)]
    sizes[50] = 0
    params, grads = _tensors(sizes, 4)
    alone = [p.clone() for p in params]
    rfsf.RfsfAdamW(params).step(grads, 1, **SETTINGS)
    for p, g in zip(alone, grads):
        rfsf.RfsfAdamW([p]).step([g], 1, **SETTINGS)
    assert all(torch.equal(a, b) for a, b in zip(alone, params))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_infinities_and_nan_show_where_they_are(bits, value):
    params, grads = _tensors([1000], 5)
    grads[0][300] = value
    opt = rfsf.RfsfAdamW(params, state_bits=bits)
    opt.step(grads, 1, **SETTINGS)
    m, v = opt.moments()
    block = torch.zeros(1000, dtype=torch.bool, device="cuda")
    if bits == 8:
        block[256:512] = True
        assert torch.all(torch.isnan(m[0][block])) and torch.all(torch.isnan(v[0][block]))
    else:
        block[300] = True
    assert not torch.isfinite(m[0][300]) and torch.isfinite(m[0][~block]).all() and torch.isfinite(v[0][~block]).all()
    assert torch.isnan(params[0][300]) and torch.isfinite(params[0]).sum() == 999


def test_steps_lead_to_the_minimum_with_either_state():
    """Least squares: both kinds of state come within the learning rate's neighbourhood of the solution."""
    gen = torch.Generator().manual_seed(6)
    goal = torch.randn(2000, generator=gen).cuda()
    for bits in (8, 32):
        p = torch.zeros(2000, device="cuda")
        opt = rfsf.RfsfAdamW([p], state_bits=bits)
        for t in range(1, 1001):
            opt.step([p - goal], t, lr=2e-2 * (1 - t / 1001), weight_decay=0.0)
        assert (p - goal).abs().max() < 2e-2


def test_on_another_stream_and_in_a_graph():
    params, grads = _tensors(SIZES, 7)
    twin = [p.clone() for p in params]
    a, b = rfsf.RfsfAdamW(params, state_bits=8), rfsf.RfsfAdamW(twin, state_bits=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.step(grads, 1, **SETTINGS, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    b.step(grads, 1, **SETTINGS)
    assert all(torch.equal(x, y) for x, y in zip(params, twin))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(grads, 2, **SETTINGS)
    for _ in range(3):
        for g in grads:
            g.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        b.step(grads, 2, **SETTINGS)
        assert all(torch.equal(x, y) for x, y in zip(params, twin))
        assert all(torch.equal(x, y) for k in a.state for x, y in zip(a.state[k], b.state[k]))


def test_refusals():
    p = [torch.zeros(10, device="cuda")]
    g = [torch.zeros(10, device="cuda")]
    opt = rfsf.RfsfAdamW(p)
    for bad in ([], [g[0][:9]], [g[0].half()], [torch.zeros(20, device="cuda")[::2]], [torch.zeros(10)]):
        with pytest.raises(ValueError):
            opt.step(bad, 1, 1e-3)
    with pytest.raises(rfsf.RfsfTsError):
        opt.step(g, 0, 1e-3)
    with pytest.raises(ValueError):
        rfsf.RfsfAdamW(p, state={"m": g})
    with pytest.raises(ValueError):
        rfsf.RfsfAdamW(p, state_bits=8, state={"m": g, "v": g, "m_scale": g, "v_scale": g})
    with pytest.raises(ValueError):
        rfsf.RfsfAdamW(p, copies=g)
