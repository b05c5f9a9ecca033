"""Timing cases of the operators around a linear model on signature features.

Between the feature rows (N sequences, K = 1 + M*D columns) and the linear classifier that is trained on them stand a layer norm
with gains and offsets of its own and dropout, whose mask comes from a counter-based generator and is never stored. A trained
classifier serves many users at once, each with a low-rank adapter of their own beside the shared weights. Every case is one call
of one of these; the program keeps its output buffers, workspaces and laid out weights from call to call.

`run` has each operator twice: as the library's call, and in elementary operations of 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
WORD = 0xFFFFFFFF


def listed():
    return [
        # a sequence that has just come in, answered by a model with a layer norm: latency
        dict(name="norm_one", op="norm", N=1, K=1025, bf16=False, p=0.0),
        # a training set of the "large" configuration's width in mixed precision, with dropout behind the norm: bound by memory
        dict(name="norm_large", op="norm", N=30000, K=10241, bf16=True, p=0.1),
        # the smallest batch of the configuration table, all gradients: latency and launches
        dict(name="back_tiny", op="back", N=16, K=193, bf16=False, p=0.0, dX=True),
        # the paper's pen digits (5 levels of 200), features that are fixed: gradients of gains and offsets alone
        dict(name="back_digits", op="back", N=7494, K=1001, bf16=False, p=0.25, dX=False),
        # very many short rows in mixed precision: the reduction over rows counts
        dict(name="back_narrow", op="back", N=200003, K=65, bf16=True, p=0.0, dX=True),
        # all gradients at the "large" configuration's width, with dropout
        dict(name="back_large", op="back", N=10000, K=10241, bf16=False, p=0.1, dX=True),
        # a small batch
        dict(name="dropout_small", op="dropout", N=100, K=1025, bf16=False, p=0.5),
        # mixed precision, all rows of a training set at a time
        dict(name="dropout_large", op="dropout", N=30000, K=5121, bf16=True, p=0.1),
        # one request to a classifier of 1000 classes, with its user's adapter: latency
        dict(name="adapted_one", op="adapted", N=1, K=1025, C=1000, R=8, E=20, bf16=False),
        # a handful of requests, most of them of different users: bound by reading weights and adapters
        dict(name="adapted_few", op="adapted", N=16, K=5121, C=5003, R=16, E=50, bf16=False),
        # an ordinary batch of many users' requests in mixed precision
        dict(name="adapted_batch", op="adapted", N=333, K=5121, C=10000, R=16, E=100, bf16=True),
        # a large batch over a large vocabulary
        dict(name="adapted_large", op="adapted", N=8192, K=2049, C=32768, R=32, E=64, bf16=True),
    ]


def _spread(rng, low, high):
    """A whole number, even over the logarithm of the range, odd ones as likely as even ones."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["norm", "back", "dropout", "adapted", "adapted"])
    bf16 = rng.random() < 0.5
    if op == "adapted":
        while True:
            c = dict(op=op, N=_spread(rng, 1, 8192), K=_spread(rng, 65, 10241), C=_spread(rng, 10, 50000), R=_spread(rng, 4, 64),
                     E=_spread(rng, 1, 128), bf16=bf16)
            if c["N"] * c["K"] * c["C"] <= 1 << 38 and c["C"] * c["K"] <= 1 << 28 and c["N"] * c["C"] <= 1 << 28 and \
                    c["E"] * c["R"] * (c["K"] + c["C"]) <= 1 << 27:
                return c
    while True:
        c = dict(op=op, N=_spread(rng, 1, 300000), K=_spread(rng, 65, 16385), bf16=bf16, p=rng.choice([0.0, rng.uniform(0.02, 0.6)]))
        if op == "dropout":
            c["p"] = rng.uniform(0.02, 0.6)
        if op == "back":
            c["dX"] = rng.random() < 0.6
        if c["N"] * c["K"] <= 100000000:
            return c


def _rows(N, K, dtype):
    """Memory for rows that are a multiple of eight numbers apart."""
    return torch.zeros(N, (K + 7) // 8 * 8, dtype=dtype, device=DEV)[:, :K]


def _normal(N, K, scale, gen, dtype):
    """Normal numbers in such memory, made a part of the rows at a time."""
    out = _rows(N, K, dtype)
    step = max(1, (1 << 26) // K)
    for a in range(0, N, step):
        n = min(step, N - a)
        out[a:a + n] = torch.randn(n, K, device=DEV, generator=gen) * scale
    return out


def _features(N, K, gen, dtype):
    """Rows like level-wise normalised features: a constant column, then numbers that share a mean, norm about 1."""
    x = _normal(N, K, 1.0 / math.sqrt(2.0 * K), gen, dtype)
    x += (torch.randn(1, K, device=DEV, generator=gen) / math.sqrt(2.0 * K)).to(dtype)
    x[:, 0] = 0.4
    return x


def _inputs(case, seed):
    """The data of a case."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000003 * (seed + 1) + 29)
    N, K = case["N"], case["K"]
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    s = {"X": _features(N, K, gen, dtype), "seed": 0x9E3779B97F4A7C15 * (seed + 1) % (1 << 64), "step": 1000 + seed}
    if case["op"] in ("norm", "back"):
        s["gain"] = 1.0 + 0.1 * torch.randn(K, device=DEV, generator=gen)
        s["offset"] = 0.1 * torch.randn(K, device=DEV, generator=gen)
    if case["op"] == "back":
        s["dY"] = _normal(N, K, 1.0 / N, gen, dtype)
        # what the forward pass has left
        step = max(1, (1 << 26) // K)
        parts = [torch.var_mean(s["X"][a:a + step].double(), dim=1, correction=0) for a in range(0, N, step)]
        s["mean"] = torch.cat([m for _, m in parts]).float()
        s["rstd"] = torch.rsqrt(torch.cat([v for v, _ in parts]) + EPS).float()
    if case["op"] == "adapted":
        C, R, E = case["C"], case["R"], case["E"]
        s["W"] = _normal(C, K, 2.0, gen, dtype)
        s["A"] = [_normal(R, K, 1.0, gen, dtype) for _ in range(E)]
        s["B"] = [(torch.randn(C, R, device=DEV, generator=gen) * (0.5 / math.sqrt(R))).to(dtype) for _ in range(E)]
        s["scale"] = [2.0 / (1 + e % 3) for e in range(E)]
        # frequent and rare users; one request in ten has no adapter
        u = torch.rand(N, device=DEV, generator=gen)
        s["adapters"] = (E * u * torch.sqrt(u)).long().clamp_(0, E - 1)
        s["adapters"][torch.rand(N, device=DEV, generator=gen) < 0.1] = -1
        if N == 1:
            s["adapters"].zero_()
    return s


def prepare(case, seed):
    """The data, and what a program keeps from call to call: output buffers, workspaces, the weights laid out."""
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if not own:
        return s
    import paper_2501_07145_amd as rfsf
    N, K, op, dtype = case["N"], case["K"], case["op"], s["X"].dtype
    if op != "adapted":
        s["dropout"] = rfsf.RfsfDropout(case["p"], s["seed"], offset=s["step"]) if case["p"] > 0 else None
    if op == "norm":
        s["out"], s["mean"], s["rstd"] = _rows(N, K, dtype), torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    elif op == "back":
        s["dX"] = _rows(N, K, dtype) if case["dX"] else None
        s["dgain"], s["doffset"] = torch.empty(K, device=DEV), torch.empty(K, device=DEV)
        rec, _ = rfsf.rfsf_layer_norm_backward_workspace_bytes(N, K, dtype, need_dX=case["dX"])
        s["workspace"] = torch.empty(rec, dtype=torch.uint8, device=DEV)
    elif op == "dropout":
        s["out"] = _rows(N, K, dtype)
    else:
        s["classifier"] = rfsf.RfsfAdapters(s["W"], case["E"], case["R"])
        for e in range(case["E"]):
            s["classifier"].set(e, s["A"][e], s["B"][e], s["scale"][e])
        rec, _ = s["classifier"].workspace_bytes(N)
        s["workspace"] = torch.empty(rec, dtype=torch.uint8, device=DEV)
        s["out"] = torch.empty(N, case["C"], device=DEV)
    return s


def run(s):
    return {"norm": _norm, "back": _back, "dropout": _dropout, "adapted": _adapted}[s["case"]["op"]](s)


def _sixteen_bits(N, K, seed, step):
    """A number of 16 bits for every place of N rows of K columns: Philox 4x32 of 10 rounds, key `seed`, counter (column / 8, row, step), whose four
    words are the numbers of eight columns."""
    words = [torch.arange((K + 7) // 8, device=DEV)[None, :], torch.arange(N, device=DEV)[:, None],
             torch.full((1, 1), step & WORD, device=DEV), torch.full((1, 1), step >> 32, device=DEV)]
    key = [seed & WORD, seed >> 32]
    for _ in range(10):
        first, second = words[0] * 0xD2511F53, words[2] * 0xCD9E8D57
        words = [(second >> 32 & WORD) ^ words[1] ^ key[0], second & WORD, (first >> 32 & WORD) ^ words[3] ^ key[1], first & WORD]
        key = [(key[0] + 0x9E3779B9) & WORD, (key[1] + 0xBB67AE85) & WORD]
    eight = [part.to(torch.int32) for w in words for part in (w & 0xFFFF, w >> 16)]
    return torch.stack(eight, 2).view(N, -1)[:, :K]


def _keep(s):
    """Where dropout keeps numbers, and what it multiplies these by."""
    N, K = s["X"].shape
    drop = round(65536 * s["case"]["p"])
    return _sixteen_bits(N, K, s["seed"], s["step"]) >= drop, 65536 / (65536 - drop)


def _norm(s):
    if own:
        import paper_2501_07145_amd as rfsf
        return rfsf.rfsf_layer_norm(s["X"], s["gain"], s["offset"], eps=EPS, dropout=s["dropout"], out=s["out"], mean=s["mean"], rstd=s["rstd"])
    x = s["X"].float()
    mean = x.mean(1)
    z = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((z * z).mean(1) + EPS)
    y = z * rstd[:, None] * s["gain"] + s["offset"]
    if s["case"]["p"] > 0:
        keep, factor = _keep(s)
        y = torch.where(keep, y * factor, torch.zeros((), device=DEV))
    return y.to(s["X"].dtype), mean, rstd


def _back(s):
    case = s["case"]
    if own:
        import paper_2501_07145_amd as rfsf
        out = rfsf.rfsf_layer_norm_backward(s["X"], s["mean"], s["rstd"], s["dY"], gain=s["gain"], dropout=s["dropout"], need_dX=case["dX"],
                                            dX=s["dX"], dgain=s["dgain"], doffset=s["doffset"], workspace=s["workspace"])
        return [t for t in out if t is not None]
    z = (s["X"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    h = s["dY"].float()
    if case["p"] > 0:
        keep, factor = _keep(s)
        h = torch.where(keep, h * factor, torch.zeros((), device=DEV))
    gains = [(h * z).sum(0), h.sum(0)]
    if not case["dX"]:
        return gains
    g = h * s["gain"]
    dx = (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True)) * s["rstd"][:, None]
    return [dx.to(s["X"].dtype)] + gains


def _dropout(s):
    if own:
        import paper_2501_07145_amd as rfsf
        return rfsf.rfsf_dropout(s["X"], s["dropout"], out=s["out"])
    keep, factor = _keep(s)
    return torch.where(keep, s["X"].float() * factor, torch.zeros((), device=DEV)).to(s["X"].dtype)


def _adapted(s):
    if own:
        return s["classifier"].scores(s["X"], s["adapters"], out=s["out"], workspace=s["workspace"])
    x = s["X"].float()
    out = x @ s["W"].float().T
    for e in range(s["case"]["E"]):
        rows = (s["adapters"] == e).nonzero()[:, 0]
        if len(rows) > 0:
            out[rows] += ((x[rows] @ s["A"][e].float().T) * s["scale"][e]) @ s["B"][e].float().T
    return out


def work(case):
    N, K, size = case["N"], case["K"], 2 if case["bf16"] else 4
    if case["op"] == "norm":
        return {"bytes": 2 * N * K * size + 8 * N + 8 * K, "flops": 8 * N * K}
    if case["op"] == "back":
        return {"bytes": (2 + case["dX"]) * N * K * size + 8 * N + 12 * K, "flops": (14 if case["dX"] else 6) * N * K}
    if case["op"] == "dropout":
        return {"bytes": 2 * N * K * size, "flops": N * K}
    C, R = case["C"], case["R"]
    users = min(case["E"], N)
    return {"bytes": size * (N * K + C * K + users * R * (K + C)) + 8 * N + 4 * N * C, "flops": 2 * N * (K * C + R * (K + C))}


def _numbers64(N, K, seed, step):
    """The generator's numbers again, products of 32-bit words put together from halves."""
    low = 0xFFFF

    def product(a, m):
        """(high, low) words of a times m."""
        a0, a1, m0, m1 = a & low, a >> 16, m & low, m >> 16
        b = a0 * m0
        mid = a1 * m0 + (b >> 16)
        rest = a0 * m1 + (mid & low)
        return a1 * m1 + (mid >> 16) + (rest >> 16), (rest & low) * 65536 + (b & low)

    out = torch.empty(N, (K + 7) // 8, 8, dtype=torch.int32, device=DEV)
    rows = max(1, (1 << 25) // K)
    for a in range(0, N, rows):
        n = min(rows, N - a)
        shape = (n, out.shape[1])
        c = [torch.arange(shape[1], device=DEV).expand(shape), torch.arange(a, a + n, device=DEV)[:, None].expand(shape)]
        c += [torch.full(shape, v, device=DEV) for v in (step % (1 << 32), step // (1 << 32))]
        for i in range(10):
            k0, k1 = (seed + i * 0x9E3779B9) & WORD, ((seed >> 32) + i * 0xBB67AE85) & WORD
            h0, l0 = product(c[0], 0xD2511F53)
            h2, l2 = product(c[2], 0xCD9E8D57)
            c = [h2.bitwise_xor(c[1]).bitwise_xor(k0), l2, h0.bitwise_xor(c[3]).bitwise_xor(k1), l0]
        for i in range(8):
            out[a:a + n, :, i] = (c[i // 2] // (65536 if i % 2 else 1) % 65536).int()
    return out.flatten(1)[:, :K]


def exact(case, seed):
    """What `run` returns, from the definitions, in 64 bits."""
    s = _inputs(case, seed)
    f64, N, K = torch.float64, case["N"], case["K"]
    X = s["X"]
    if case["op"] == "adapted":
        W, out = s["W"].to(f64), torch.empty(N, case["C"], dtype=f64, device=DEV)
        for a in range(0, N, 2048):
            torch.matmul(X[a:a + 2048].to(f64), W.t(), out=out[a:a + 2048])
        del W
        for e, count in zip(*(t.tolist() for t in torch.unique(s["adapters"], return_counts=True))):
            if e >= 0:
                at = torch.where(s["adapters"] == e)[0]
                inner = torch.matmul(X.index_select(0, at).to(f64), s["A"][e].to(f64).t())
                out.index_add_(0, at, torch.matmul(inner, s["B"][e].to(f64).t()), alpha=s["scale"][e])
        return out
    p = case["p"]
    dropped = round(65536 * p) if p > 0 else 0
    weight = 65536 / (65536 - dropped)
    numbers = _numbers64(N, K, s["seed"], s["step"]) if dropped else None
    step = max(1, (1 << 26) // K)
    parts, sums = [], [torch.zeros(K, dtype=f64, device=DEV) for _ in range(2)]
    for a in range(0, N, step):
        at = slice(a, a + step)
        x = X[at].to(f64)
        mask = (numbers[at] >= dropped).to(f64) * weight if dropped else torch.ones((), dtype=f64, device=DEV)
        if case["op"] == "dropout":
            parts.append((x * mask,))
        elif case["op"] == "norm":
            variance, mean = torch.var_mean(x, dim=1, correction=0)
            rstd = (variance + EPS).pow(-0.5)
            y = torch.addcmul(s["offset"].to(f64), (x - mean[:, None]) * rstd[:, None], s["gain"].to(f64)) * mask
            parts.append((y, mean, rstd))
        else:
            rstd = s["rstd"][at].to(f64)[:, None]
            z = (x - s["mean"][at].to(f64)[:, None]) * rstd
            h = s["dY"][at].to(f64) * mask
            sums[0] += torch.einsum("nk,nk->k", h, z)
            sums[1] += h.sum(dim=0)
            if case["dX"]:
                g = h * s["gain"].to(f64)
                both = torch.stack([g.sum(dim=1), torch.einsum("nk,nk->n", g, z)]) / K
                parts.append((rstd * (g - both[0][:, None] - z * both[1][:, None]),))
    whole = [torch.cat(t) for t in zip(*parts)]
    if case["op"] == "dropout":
        return whole[0]
    return tuple(whole) if case["op"] == "norm" else whole + sums
