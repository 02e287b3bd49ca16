"""Cases for measuring the operators at the two ends of a token model: layer norm, the embedding lookup, and the
softmax cross entropy of a linear layer over a vocabulary, each forward and backward. Each case can run in a plain
form (elementary torch operations in fp32) and, with `own` true, through the library's public entry points."""
import math

import torch

own = False

_D = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one sentence of 64 tokens of a BERT-large sized model: latency counts
        {"name": "ln one sentence", "op": "ln", "M": 64, "D": 1024, "dtype": "bf16", "slack": 0, "add": False, "backward": False},
        # a training batch of 32 x 512 tokens at that width
        {"name": "ln batch", "op": "ln", "M": 16384, "D": 1024, "dtype": "bf16", "slack": 0, "add": False, "backward": False},
        # its gradient, with the gradient that goes past the norm along the residual added on the way
        {"name": "ln backward batch", "op": "ln", "M": 16384, "D": 1024, "dtype": "bf16", "slack": 0, "add": True, "backward": True},
        # odd features in fp32, a slice of a wider tensor
        {"name": "ln backward ragged", "op": "ln", "M": 2999, "D": 771, "dtype": "f32", "slack": 6, "add": False, "backward": True},
        # one sentence's tokens looked up: latency counts
        {"name": "embedding one sentence", "op": "emb", "N": 64, "V": 30522, "D": 1024, "dtype": "bf16", "scale": 1.0, "pad": 0.0, "tied": False, "backward": False},
        # a batch of 64 x 512 tokens, scaled by the square root of the width
        {"name": "embedding batch", "op": "emb", "N": 32768, "V": 30522, "D": 1024, "dtype": "bf16", "scale": 32.0, "pad": 0.05, "tied": False, "backward": False},
        # the dense gradient of a table from a batch of 32 x 512 tokens: every row of the flat gradient vector is written
        {"name": "embedding backward", "op": "emb", "N": 16384, "V": 30522, "D": 1024, "dtype": "bf16", "scale": 1.0, "pad": 0.0, "tied": False, "backward": True},
        # a large padded batch into a head's gradient that is there already (tied weights), fp32, an odd vocabulary and width
        {"name": "embedding backward tied", "op": "emb", "N": 65536, "V": 50257, "D": 771, "dtype": "f32", "scale": 27.75, "pad": 0.3, "tied": True, "backward": True},
        # the ten-way classifier of a small model: latency counts
        {"name": "ce small", "op": "ce", "N": 128, "V": 10, "D": 64, "bias": True, "ignored": 0.0, "backward": False},
        # the loss of 16 x 512 tokens over a BERT-large sized vocabulary
        {"name": "ce vocabulary", "op": "ce", "N": 8192, "V": 30522, "D": 1024, "bias": True, "ignored": 0.1, "backward": False},
        # its gradient
        {"name": "ce backward vocabulary", "op": "ce", "N": 8192, "V": 30522, "D": 1024, "bias": True, "ignored": 0.1, "backward": True},
        # a ragged batch into a 1000-way classifier from an odd number of features
        {"name": "ce backward odd", "op": "ce", "N": 777, "V": 1000, "D": 513, "bias": False, "ignored": 0.0, "backward": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    d = _log(rng, lo, hi)
    return -(-d // 8) * 8 if rng.random() < 0.6 else d


def draw(rng):
    op, back = rng.choice(["ln", "emb", "ce"]), rng.random() < 0.5
    if op == "ln":
        while True:
            M, D = _log(rng, 16, 60000), _width(rng, 24, 16000)
            if 10_000 <= M * D <= 16_000_000:
                break
        return {"op": op, "M": M, "D": D, "dtype": rng.choice(["f32", "bf16"]), "slack": rng.choice([0, 0, 8, 3]), "add": back and rng.random() < 0.5, "backward": back}
    if op == "emb":
        while True:
            N, V, D = _log(rng, 32, 100000), _log(rng, 100, 200000), _width(rng, 24, 4000)
            if 10_000 <= N * D <= 40_000_000 and V * D <= 60_000_000:
                break
        return {"op": op, "N": N, "V": V, "D": D, "dtype": rng.choice(["f32", "bf16"]), "scale": rng.choice([1.0, math.sqrt(D)]),
                "pad": rng.choice([0.0, 0.1, 0.5]), "tied": back and rng.random() < 0.4, "backward": back}
    while True:
        N, V, D = _log(rng, 1, 16000), _log(rng, 2, 130000), _width(rng, 16, 4000)
        if 100_000 <= N * V * D <= 1.2e11 and N * V <= 200_000_000:
            break
    return {"op": op, "N": N, "V": V, "D": D, "bias": rng.random() < 0.5, "ignored": rng.choice([0.0, 0.15, 0.85]), "backward": back}


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _words(g, n, V):
    """n token numbers by a Zipf-like law (the k-th word about as likely as 1 / k), the words in any order."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    k = torch.exp(u * math.log(V + 1.0)).long().sub_(1).clamp_(0, V - 1)
    return torch.randperm(V, generator=g, device="cuda")[k]


def _prepare_ln(case, seed):
    g = _gen(seed)
    M, D, dt, wide = case["M"], case["D"], _D[case["dtype"]], case["D"] + case["slack"]
    x = _randn(g, M, wide, scale=1.3)
    x += _randn(g, wide, scale=0.5) + _randn(g, M, 1, scale=0.5)
    st = dict(case=case, x=x.to(dt)[:, :D], w=1.0 + _randn(g, D, scale=0.2), b=_randn(g, D, scale=0.2), eps=1e-5)
    if case["backward"]:
        f = st["x"].float()
        st["mean"] = f.mean(1)
        st["rstd"] = torch.rsqrt((f - st["mean"][:, None]).square().mean(1) + st["eps"])
        st["dy"] = _randn(g, M, wide, scale=0.01, dtype=dt)[:, :D]
        st["add"] = _randn(g, M, wide, scale=0.01, dtype=dt)[:, :D] if case["add"] else None
    return st


def _prepare_emb(case, seed):
    g = _gen(seed)
    N, V, D, dt = case["N"], case["V"], case["D"], _D[case["dtype"]]
    ids = _words(g, N, V)
    if case["pad"]:
        ids = torch.where(torch.rand(N, generator=g, device="cuda") < case["pad"], torch.full_like(ids, -1), ids)
    st = dict(case=case, ids=ids)
    if not case["backward"]:
        st["table"] = _randn(g, V, D, scale=0.02, dtype=dt)
        return st
    st["dy"] = _randn(g, N, D, scale=0.01, dtype=dt)
    if case["tied"]:
        st["grad"] = _randn(g, V, D, scale=0.01, dtype=dt)       # the head's share, that the lookup's is added to
        st["out"] = st["grad"].clone()
    return st


def _prepare_ce(case, seed):
    g = _gen(seed)
    N, V, D, bf = case["N"], case["V"], case["D"], torch.bfloat16
    # rows that know something of their target: their logit stands out by a few units
    target = _words(g, N, V)
    w = _randn(g, V, D, scale=1.5 * D ** -0.5, dtype=bf)
    x = _randn(g, N, D)
    x = (x + w[target].float() * (2.0 * torch.rand(N, 1, generator=g, device="cuda"))).to(bf)
    live = torch.rand(N, generator=g, device="cuda") >= case["ignored"]
    target = torch.where(live, target, torch.full_like(target, -100))
    st = dict(case=case, x=x, w=w, b=_randn(g, V, scale=0.3, dtype=bf) if case["bias"] else None, target=target)
    if case["backward"]:
        st["dloss"] = live.float() / live.sum().clamp_min(1)     # of the mean over the rows that count
        lse = []
        for i in range(0, N, 1024):
            z = st["x"][i:i + 1024].float() @ w.float().T
            lse.append(torch.logsumexp(z + st["b"].float() if case["bias"] else z, 1))
        st["lse"] = torch.cat(lse)
    return st


def prepare(case, seed):
    return {"ln": _prepare_ln, "emb": _prepare_emb, "ce": _prepare_ce}[case["op"]](case, seed)


# ---------------------------------------------------------------------------------------------- the plain forms

def _plain_ln(st):
    case, x = st["case"], st["x"].float()
    dt = st["x"].dtype
    if not case["backward"]:
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = torch.rsqrt(d.square().mean(1) + st["eps"])
        return (d * rstd[:, None] * st["w"] + st["b"]).to(dt), mean, rstd
    xh = (x - st["mean"][:, None]) * st["rstd"][:, None]
    dy = st["dy"].float()
    t = dy * st["w"]
    dx = (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True)) * st["rstd"][:, None]
    if st["add"] is not None:
        dx = dx + st["add"].float()
    return dx.to(dt), (dy * xh).sum(0), dy.sum(0)


def _plain_emb(st):
    case, ids = st["case"], st["ids"]
    live = (ids >= 0) & (ids < case["V"])
    at = torch.where(live, ids, torch.zeros_like(ids))
    if not case["backward"]:
        t = st["table"]
        return (t[at].float() * case["scale"] * live[:, None]).to(t.dtype)
    dy = st["dy"]
    sums = torch.zeros(case["V"], case["D"], device="cuda").index_add_(0, at, dy.float() * live[:, None]) * case["scale"]
    if not case["tied"]:
        return sums.to(dy.dtype)
    st["out"].copy_(st["grad"])
    st["out"].copy_(st["out"].float() + sums)
    return st["out"]


def _plain_ce(st):
    case, x, w, target = st["case"], st["x"].float(), st["w"].float(), st["target"]
    z = x @ w.T
    if st["b"] is not None:
        z += st["b"].float()
    live = (target >= 0) & (target < case["V"])
    at = torch.where(live, target, torch.zeros_like(target))
    rows = torch.arange(case["N"], device="cuda")
    if not case["backward"]:
        top = z.amax(1)
        lse = torch.log(torch.exp(z - top[:, None]).sum(1)) + top
        return torch.where(live, lse - z[rows, at], torch.zeros_like(lse)), lse
    z.sub_(st["lse"][:, None]).exp_()
    z[rows, at] -= 1.0
    z *= torch.where(live, st["dloss"], torch.zeros_like(st["dloss"]))[:, None]
    bf = torch.bfloat16
    return (z @ w).to(bf), (z.T @ x).to(bf), z.sum(0).to(bf) if st["b"] is not None else None


# ---------------------------------------------------------------------------------------------- the library's calls

def _own(st):
    import paper_2510_08522_b200 as D
    case = st["case"]
    if case["op"] == "ln":
        if not case["backward"]:
            return D.layer_norm(st["x"], st["w"], st["b"], eps=st["eps"])
        return D.layer_norm_backward(st["dy"], st["x"], st["mean"], st["rstd"], st["w"], add=st["add"])
    if case["op"] == "emb":
        if not case["backward"]:
            return D.embedding(st["ids"], st["table"], scale=case["scale"])
        if not case["tied"]:
            return D.embedding_backward(st["dy"], st["ids"], case["V"], scale=case["scale"])
        st["out"].copy_(st["grad"])
        return D.embedding_backward(st["dy"], st["ids"], case["V"], scale=case["scale"], out=st["out"], accumulate=True)
    if not case["backward"]:
        return D.linear_cross_entropy(st["x"], st["w"], st["target"], st["b"])
    need = (True, True, st["b"] is not None)
    return D.linear_cross_entropy_backward(st["dloss"], st["x"], st["w"], st["target"], st["lse"], st["b"], need=need)


def run(st):
    if own:
        return _own(st)
    return {"ln": _plain_ln, "emb": _plain_emb, "ce": _plain_ce}[st["case"]["op"]](st)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "ln":
        n = case["M"] * case["D"]
        if not case["backward"]:
            return {"bytes": 2 * e * n + 8 * case["D"] + 8 * case["M"], "flops": 8 * n}
        return {"bytes": (3 + case["add"]) * e * n + 12 * case["D"] + 8 * case["M"], "flops": 14 * n}
    if case["op"] == "emb":
        N, V, D = case["N"], case["V"], case["D"]
        live = int(N * (1.0 - case["pad"]))
        rows = min(live, V)                                      # at most so many rows of the table
        if not case["backward"]:
            return {"bytes": 8 * N + e * D * (rows + N), "flops": N * D}
        if not case["tied"]:
            return {"bytes": 8 * N + e * D * (live + V), "flops": N * D}
        # the tied case sets the head's share anew in every pass: a copy of the table, then rows that are read and written
        return {"bytes": 8 * N + e * D * (live + 2 * V + 2 * rows), "flops": N * D}
    N, V, D = case["N"], case["V"], case["D"]
    b = 2 * V if case["bias"] else 0
    if not case["backward"]:
        return {"bytes": 2 * D * (N + V) + b + 16 * N, "flops": 2 * N * V * D}
    return {"bytes": 4 * D * (N + V) + 2 * b + 16 * N, "flops": 6 * N * V * D}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits

def _exact_ln(st, case):
    x, w = st["x"].double(), st["w"].double()
    D = case["D"]
    if not case["backward"]:
        mean = x.sum(1) / D
        var = ((x - mean[:, None]) ** 2).sum(1) / D
        r = 1.0 / torch.sqrt(var + st["eps"])
        return (x - mean[:, None]) * r[:, None] * w + st["b"].double(), mean, r
    r, dy = st["rstd"].double()[:, None], st["dy"].double()
    h = (x - st["mean"].double()[:, None]) * r
    a = (dy * w).sum(1, keepdim=True) / D
    c = (dy * w * h).sum(1, keepdim=True) / D
    dx = r * (w * dy - (a + h * c))
    return dx if st["add"] is None else dx + st["add"].double(), (dy * h).sum(0), dy.sum(0)


def _exact_emb(st, case):
    ids, V, D, s = st["ids"], case["V"], case["D"], case["scale"]
    keep = torch.nonzero((ids >= 0) & (ids < V))[:, 0]
    if not case["backward"]:
        y = torch.zeros(case["N"], D, dtype=torch.float64, device="cuda")
        y[keep] = s * st["table"].double()[ids[keep]]
        return y
    total = st["grad"].double() if case["tied"] else torch.zeros(V, D, dtype=torch.float64, device="cuda")
    order = keep[torch.argsort(ids[keep], stable=True)]
    for part in order.split(8192):
        total.index_put_((ids[part],), s * st["dy"][part].double(), accumulate=True)
    return total


def _exact_ce(st, case):
    N, V, t = case["N"], case["V"], st["target"]
    w = st["w"].double()
    b = st["b"].double() if case["bias"] else torch.zeros(V, dtype=torch.float64, device="cuda")
    ok = (t >= 0) & (t < V)
    if not case["backward"]:
        loss, lse = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.empty(N, dtype=torch.float64, device="cuda")
        for i in range(0, N, 1024):
            z = st["x"][i:i + 1024].double() @ w.T + b
            lse[i:i + 1024] = torch.logsumexp(z, 1)
            hit = torch.nonzero(ok[i:i + 1024])[:, 0]
            loss[i + hit] = lse[i + hit] - z[hit, t[i + hit]]
        return loss, lse
    dx = torch.empty(N, case["D"], dtype=torch.float64, device="cuda")
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    for i in range(0, N, 1024):
        x = st["x"][i:i + 1024].double()
        p = torch.exp(x @ w.T + b - st["lse"][i:i + 1024].double()[:, None])
        hit = torch.nonzero(ok[i:i + 1024])[:, 0]
        p[hit, t[i + hit]] -= 1.0
        p *= (st["dloss"][i:i + 1024].double() * ok[i:i + 1024])[:, None]
        dx[i:i + 1024] = p @ w
        dw += p.T @ x
        db += p.sum(0)
    return dx, dw, db if case["bias"] else None


def exact(case, seed):
    st = prepare(case, seed)
    return {"ln": _exact_ln, "emb": _exact_emb, "ce": _exact_ce}[case["op"]](st, case)
