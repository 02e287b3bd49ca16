"""Cases for measuring the training operators: AdamW over many tensors, group norm with an activation
(channels last, forward and backward), and the matrix product with bias, activation and residual in its
epilogue (forward and backward). Each case can run in a plain form (elementary torch operations in fp32) and,
with `own` true, through the library's public entry points."""
import math
import random

import torch

own = False

BLOCK = 256          # elements of one block of optimizer state: one scale of each moment per block
TILE = 1 << 24       # parameters per slice of the fp64 form
_D = {"f32": torch.float32, "bf16": torch.bfloat16}
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, t=37)


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a small model's step, sized like the smallest gradient workload (1 Mi parameters): latency counts
        {"name": "adamw small f32", "op": "adamw", "P": 1048576, "tensors": 16, "align": 256, "grad": "f32", "bits": 32, "clip": True, "copies": False},
        # tensors packed tightly into one flat vector (a ResNet-50 sized parameter count, 161 segments): starts
        # at any element; bf16 gradients, moments held in 8 bits, dithered
        {"name": "adamw packed 8-bit", "op": "adamw", "P": 25557032, "tensors": 161, "align": 1, "grad": "bf16", "bits": 8, "clip": False, "copies": False},
        # a VGG-16 sized fp32 step with the gradients' global norm clipped (fp32 moments)
        {"name": "adamw large f32", "op": "adamw", "P": 138357544, "tensors": 32, "align": 256, "grad": "f32", "bits": 32, "clip": True, "copies": False},
        # a BERT-large sized mixed-precision step: bf16 gradients, fp32 masters with bf16 copies, 8-bit moments
        {"name": "adamw large 8-bit", "op": "adamw", "P": 340000000, "tensors": 398, "align": 256, "grad": "bf16", "bits": 8, "clip": False, "copies": True},
        # one sample of a late stage, as evaluated alone: latency
        {"name": "gn one sample", "op": "gn", "N": 1, "L": 64, "C": 256, "G": 32, "dtype": "f32", "act": "silu", "slack": 0, "backward": False},
        # an early stage on CIFAR-sized images at the largest batch size the controller hands out
        {"name": "gn batch 1024", "op": "gn", "N": 1024, "L": 1024, "C": 64, "G": 16, "dtype": "bf16", "act": "relu", "slack": 0, "backward": False},
        # the gradient of a first ImageNet-sized stage: a sample (1.6 MB) is larger than one SM's shared memory
        {"name": "gn backward large", "op": "gn", "N": 64, "L": 3136, "C": 256, "G": 32, "dtype": "bf16", "act": "silu", "slack": 0, "backward": True},
        # odd image, six channels to a group, a channel slice of a wider tensor
        {"name": "gn backward ragged", "op": "gn", "N": 37, "L": 729, "C": 90, "G": 15, "dtype": "f32", "act": "gelu", "slack": 7, "backward": True},
        # a single row: the weights are read once
        {"name": "linear one row", "op": "linear", "M": 1, "N": 4096, "K": 4096, "act": "none", "residual": True, "save": False, "backward": False},
        # the widening half of a BERT-large sized feed-forward block in training (keeps what backward needs)
        {"name": "linear wide gelu", "op": "linear", "M": 8192, "N": 4096, "K": 1024, "act": "gelu", "residual": False, "save": True, "backward": False},
        # the gradient of its narrowing half, without activation
        {"name": "linear backward gelu", "op": "linear", "M": 8192, "N": 4096, "K": 1024, "act": "gelu", "residual": False, "save": True, "backward": True},
        # a ragged batch into a 1000-way classifier from an odd number of features
        {"name": "linear backward odd", "op": "linear", "M": 777, "N": 1000, "K": 513, "act": "relu", "residual": False, "save": True, "backward": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adamw", "gn", "linear"])
    if op == "adamw":
        bits = rng.choice([8, 32])
        P = _log(rng, 50_000, 120_000_000)
        return {"op": op, "P": P, "tensors": min(_log(rng, 1, 400), max(1, P // 64)), "align": rng.choice([1, 256]), "grad": rng.choice(["f32", "bf16"]),
                "bits": bits, "clip": bits == 32 and rng.random() < 0.5, "copies": rng.random() < 0.5}
    if op == "gn":
        while True:
            cpg, G, L, N = _log(rng, 1, 64), _log(rng, 1, 64), _log(rng, 1, 5000), _log(rng, 1, 1024)
            if 20_000 <= cpg * G * L * N <= 48_000_000 and cpg * G <= 2048 and L != 3072:
                break
        return {"op": op, "N": N, "L": L, "C": cpg * G, "G": G, "dtype": rng.choice(["f32", "bf16"]), "act": rng.choice(["none", "relu", "silu", "gelu"]),
                "slack": rng.choice([0, 0, 8, 3]), "backward": rng.random() < 0.5}
    while True:
        M, N, K = _log(rng, 1, 8192), _log(rng, 16, 5000), _log(rng, 16, 5000)
        if rng.random() < 0.5:
            N, K = -(-N // 8) * 8, -(-K // 8) * 8
        if 50_000 <= M * N * K <= 3.4e10 and 3072 not in (M, N, K):
            break
    back = rng.random() < 0.5
    return {"op": op, "M": M, "N": N, "K": K, "act": rng.choice(["none", "relu", "silu", "gelu"]), "residual": not back and rng.random() < 0.5,
            "save": back or rng.random() < 0.5, "backward": back}


# ---------------------------------------------------------------------------------------------- inputs

def _sizes(case):
    """Tensor sizes by a log-normal law (a few large tensors, many small), summing to P."""
    P, n = case["P"], case["tensors"]
    r = random.Random(P * 1009 + n)
    w = [math.exp(r.gauss(0.0, 1.5)) for _ in range(n)]
    s = [1 + int((P - n) * x / sum(w)) for x in w]
    s[max(range(n), key=s.__getitem__)] += P - sum(s)
    return s


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _encode8(x, steps):
    """Blocks of values (nb, BLOCK), their square-root code and their scale."""
    s = x.abs().amax(1)
    c = torch.round((x.abs() / s.clamp_min(1e-30)[:, None]).sqrt() * steps)
    return (c * x.sign()), s


def _prepare_adamw(case, seed):
    g = _gen(seed)
    sizes, a = _sizes(case), case["align"]
    starts, blocks, at, nb = [], [], 0, 0
    for n in sizes:
        starts.append(at)
        blocks.append(nb)
        at += -(-n // a) * a
        nb += -(-n // BLOCK)
    lens = torch.tensor(sizes, device="cuda")
    # element j of the flat vector <-> its place among the state blocks (None where the two layouts coincide)
    flat = place = None
    if a % BLOCK:
        t = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), lens)
        within = torch.arange(int(sum(sizes)), device="cuda") - (torch.cumsum(lens, 0) - lens)[t]
        flat, place = torch.tensor(starts, device="cuda")[t] + within, torch.tensor(blocks, device="cuda")[t] * BLOCK + within
        del t, within
    live = torch.zeros(nb * BLOCK, dtype=torch.bool, device="cuda")
    for n, b in zip(sizes, blocks):
        live[b * BLOCK: b * BLOCK + n] = True
    decay = [n > 4096 for n in sizes]                       # vectors (norms, biases) are not decayed
    nblk = torch.tensor([-(-n // BLOCK) for n in sizes], device="cuda")
    decay_block = torch.repeat_interleave(torch.tensor(decay, device="cuda"), nblk)
    p = _randn(g, at, scale=0.05)
    grad = _randn(g, at, scale=0.02, dtype=_D[case["grad"]])
    copy = p.to(torch.bfloat16) if case["copies"] else None
    view = lambda x: [x[s:s + n] for s, n in zip(starts, sizes)]  # noqa: E731
    m = _randn(g, nb * BLOCK, scale=0.01).mul_(live)
    r = _randn(g, nb * BLOCK).abs_().mul_(0.02).mul_(live)        # square root of the second moment
    st = dict(case=case, nb=nb, sizes=sizes, starts=starts, flat=flat, place=place, live=live, decay=decay, decay_block=decay_block, p=p, grad=grad, copy=copy, seed=seed)
    if case["bits"] == 8:
        cm, sm = _encode8(m.view(nb, BLOCK), 127)
        cr, sr = _encode8(r.view(nb, BLOCK), 255)
        st.update(m=cm.to(torch.int8).view(-1), v=cr.to(torch.uint8).view(-1), m_scale=sm, v_scale=sr,
                  m_out=torch.empty(nb * BLOCK, dtype=torch.bfloat16, device="cuda"), v_out=torch.empty(nb * BLOCK, dtype=torch.bfloat16, device="cuda"))
        st["scale"] = torch.full((1,), 0.875, device="cuda")     # the caller's own factor (a loss scale, a clip)
    else:
        st.update(m=m, v=r.square_(), m_scale=None, v_scale=None)
    if own:
        import paper_2510_08522_b200 as D
        st["opt"] = D.AdamW(view(p), view(grad), state_bits=case["bits"], copies=view(copy) if copy is not None else None, decay=decay)
        st["norm"] = torch.empty(2, device="cuda")
    return st


def _prepare_gn(case, seed):
    g = _gen(seed)
    N, L, C, G, dt = case["N"], case["L"], case["C"], case["G"], _D[case["dtype"]]
    wide = C + case["slack"]
    x = _randn(g, N, L, wide, scale=1.5)
    x += _randn(g, wide, scale=0.7)
    x = x.to(dt)[:, :, :C]
    st = dict(case=case, x=x, w=1.0 + _randn(g, C, scale=0.2), b=_randn(g, C, scale=0.2), eps=1e-5)
    if case["backward"]:
        st["dy"] = _randn(g, N, L, wide, dtype=dt)[:, :, :C]
        f = x.float().reshape(N, L, G, C // G)
        st["mean"] = f.mean((1, 3))
        st["rstd"] = torch.rsqrt((f - st["mean"][:, None, :, None]).square().mean((1, 3)) + st["eps"])
    return st


def _prepare_linear(case, seed):
    g = _gen(seed)
    M, N, K, bf = case["M"], case["N"], case["K"], torch.bfloat16
    st = dict(case=case, x=_randn(g, M, K, dtype=bf), w=_randn(g, N, K, scale=K ** -0.5, dtype=bf), b=_randn(g, N, scale=0.1, dtype=bf))
    if case["residual"]:
        st["r"] = _randn(g, M, N, dtype=bf)
    if case["backward"]:
        st["dy"] = _randn(g, M, N, dtype=bf)
        st["z"] = _randn(g, M, N, dtype=bf) if case["act"] != "none" else None
    return st


def prepare(case, seed):
    return {"adamw": _prepare_adamw, "gn": _prepare_gn, "linear": _prepare_linear}[case["op"]](case, seed)


# ---------------------------------------------------------------------------------------------- the plain forms

def _act(u, act):
    if act == "relu":
        return u.clamp_min(0.0)
    if act == "silu":
        return u * torch.sigmoid(u)
    if act == "gelu":
        return 0.5 * u * (1.0 + torch.erf(u * math.sqrt(0.5)))
    return u


def _act_grad(u, act):
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "silu":
        s = torch.sigmoid(u)
        return s * (1.0 + u * (1.0 - s))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(u)


def _dither(n, seed):
    """Two 16-bit uniform numbers for each state element, a fixed mixing of its index and the seed (multiply,
    xor-shift; 32-bit words held in 64-bit integers)."""
    M = 0xFFFFFFFF
    h = torch.arange(n, device="cuda") * 0x9E3779B1 + ((seed * 0x85EBCA6B + 0x1B873593) & M)
    h &= M
    h ^= h >> 16
    h *= 0x85EBCA6B
    h &= M
    h ^= h >> 13
    h *= 0xC2B2AE35
    h &= M
    h ^= h >> 16
    return (h & 0xFFFF).float() * 2.0 ** -16, (h >> 16).float() * 2.0 ** -16


def _plain_adamw(s):
    case, nb, h = s["case"], s["nb"], HYPER
    n = nb * BLOCK
    if s["flat"] is None:
        p, g = s["p"].view(nb, BLOCK), s["grad"].view(nb, BLOCK).float()
    else:
        p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        p[s["place"]] = s["p"][s["flat"]]
        g[s["place"]] = s["grad"][s["flat"]].float()
        p, g = p.view(nb, BLOCK), g.view(nb, BLOCK)
    live = s["live"].view(nb, BLOCK)
    out = {}
    if case["clip"]:
        norm = torch.where(live, g, 0.0).square().sum().sqrt()
        coef = torch.clamp(1.0 / (norm + 1e-6), max=1.0)
        out["norm"], out["coef"] = norm, coef
    else:
        coef = s["scale"] if case["bits"] == 8 else None
    g = torch.where(live, g if coef is None else g * coef, 0.0)
    if case["bits"] == 8:
        a = s["m"].view(nb, BLOCK).float() * (1.0 / 127.0)
        m = a * a.abs() * s["m_scale"][:, None]
        a = s["v"].view(nb, BLOCK).float() * (1.0 / 255.0)
        v = (a * a * s["v_scale"][:, None]).square()
    else:
        m, v = s["m"].view(nb, BLOCK), s["v"].view(nb, BLOCK)
    m = m * h["beta1"] + g * (1.0 - h["beta1"])
    v = v * h["beta2"] + g * g * (1.0 - h["beta2"])
    root = v.sqrt()
    step = m / (root * (1.0 / math.sqrt(1.0 - h["beta2"] ** h["t"])) + h["eps"])
    keep = torch.where(s["decay_block"], 1.0 - h["lr"] * h["weight_decay"], 1.0)[:, None]
    p = p * keep - step * (h["lr"] / (1.0 - h["beta1"] ** h["t"]))
    if s["flat"] is None:
        s["p"].copy_(torch.where(live, p, s["p"].view(nb, BLOCK)).view(-1))
    else:
        s["p"][s["flat"]] = p.view(-1)[s["place"]]
    out["p"] = s["p"]
    if s["copy"] is not None:
        if s["flat"] is None:
            s["copy"].copy_(torch.where(live, p.bfloat16(), s["copy"].view(nb, BLOCK)).view(-1))
        else:
            s["copy"][s["flat"]] = p.bfloat16().view(-1)[s["place"]]
        out["copy"] = s["copy"]
    if case["bits"] == 8:
        um, uv = _dither(n, s["seed"])
        sm, sr = m.abs().amax(1), root.amax(1)
        cm = torch.floor((m.abs() / sm.clamp_min(1e-30)[:, None]).sqrt() * 127.0 + um.view(nb, BLOCK)).clamp_max(127.0) * m.sign()
        cr = torch.floor((root / sr.clamp_min(1e-30)[:, None]).sqrt() * 255.0 + uv.view(nb, BLOCK)).clamp_max(255.0)
        cr = torch.where(root > 0, cr.clamp_min(1.0), 0.0)
        s["m"].copy_(cm.to(torch.int8).view(-1))
        s["v"].copy_(cr.to(torch.uint8).view(-1))
        s["m_scale"].copy_(sm)
        s["v_scale"].copy_(sr)
        a = cm * (1.0 / 127.0)
        s["m_out"].copy_((a * a.abs() * sm[:, None]).view(-1))
        a = cr * (1.0 / 255.0)
        s["v_out"].copy_((a * a * sr[:, None]).square().view(-1))
        out["m"], out["v"] = s["m_out"], s["v_out"]
    else:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        out["m"], out["v"] = s["m"], s["v"]
    return out


def _plain_gn(s):
    c, x = s["case"], s["x"]
    N, L, C, G = c["N"], c["L"], c["C"], c["G"]
    f = x.float().reshape(N, L, G, C // G)
    w, b = s["w"].view(G, C // G), s["b"].view(G, C // G)
    if not c["backward"]:
        mean = f.mean((1, 3))
        d = f - mean[:, None, :, None]
        rstd = torch.rsqrt(d.square().mean((1, 3)) + s["eps"])
        y = _act(d * rstd[:, None, :, None] * w + b, c["act"])
        return {"y": y.to(x.dtype).view(N, L, C), "mean": mean, "rstd": rstd}
    r = s["rstd"][:, None, :, None]
    xh = (f - s["mean"][:, None, :, None]) * r
    du = s["dy"].float().reshape(N, L, G, C // G)
    if c["act"] != "none":
        du = du * _act_grad(xh * w + b, c["act"])
    dxh = du * w
    n = L * (C // G)
    dx = r * (dxh - (dxh.sum((1, 3), keepdim=True) + xh * (dxh * xh).sum((1, 3), keepdim=True)) / n)
    return {"dx": dx.to(x.dtype).view(N, L, C), "dw": (du * xh).sum((0, 1)).view(C), "db": du.sum((0, 1)).view(C)}


def _plain_linear(s):
    c, x, w = s["case"], s["x"].float(), s["w"].float()
    if not c["backward"]:
        z = x @ w.t() + s["b"].float()
        y = _act(z, c["act"])
        if c["residual"]:
            y = y + s["r"].float()
        out = {"y": y.bfloat16()}
        if c["save"] and c["act"] != "none":
            out["z"] = z.bfloat16()
        return out
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_grad(s["z"].float(), c["act"])
    return {"dx": (dz @ w).bfloat16(), "dw": (dz.t() @ x).bfloat16(), "db": dz.sum(0).bfloat16()}


# ---------------------------------------------------------------------------------------------- the library's calls

def _own_adamw(s):
    opt, case, out = s["opt"], s["case"], {}
    scale = s.get("scale")
    if case["clip"]:
        opt.grad_norm(1.0, out=s["norm"])
        scale = s["norm"][1:]
        out["norm"], out["coef"] = s["norm"][0], s["norm"][1]
    if case["bits"] == 8:
        opt.step(s["m"], s["v"], s["m_scale"], s["v_scale"], grad_scale=scale, seed=s["seed"], **HYPER)
        opt.moments(s["m"], s["v"], s["m_scale"], s["v_scale"], s["m_out"], s["v_out"])
        out["m"], out["v"] = s["m_out"], s["v_out"]
    else:
        opt.step(s["m"], s["v"], grad_scale=scale, **HYPER)
        out["m"], out["v"] = s["m"], s["v"]
    out["p"] = s["p"]
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    return out


def _own_gn(s):
    import paper_2510_08522_b200 as D
    c = s["case"]
    if not c["backward"]:
        y, mean, rstd = D.group_norm(s["x"], c["G"], s["w"], s["b"], s["eps"], c["act"])
        return {"y": y, "mean": mean, "rstd": rstd}
    dx, dw, db = D.group_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], c["G"], s["w"], s["b"], c["act"])
    return {"dx": dx, "dw": dw, "db": db}


def _own_linear(s):
    import paper_2510_08522_b200 as D
    c = s["case"]
    if not c["backward"]:
        y, z = D.linear(s["x"], s["w"], s["b"], act=c["act"], residual=s.get("r"), save=c["save"])
        return {"y": y, "z": z} if z is not None else {"y": y}
    dx, dw, db = D.linear_backward(s["dy"], s["x"], s["w"], s["z"], act=c["act"])
    return {"dx": dx, "dw": dw, "db": db}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"adamw": _own_adamw, "gn": _own_gn, "linear": _own_linear}[op](state)
    return {"adamw": _plain_adamw, "gn": _plain_gn, "linear": _plain_linear}[op](state)


# ---------------------------------------------------------------------------------------------- work and 64 bits

def work(case):
    if case["op"] == "adamw":
        P, e = case["P"], 2 if case["grad"] == "bf16" else 4
        moments = 2 * 2 * 1 + 2 * 2 if case["bits"] == 8 else 2 * 2 * 4      # both moments in and out; as bf16 values too
        return {"bytes": P * (8 + e + moments + (2 if case["copies"] else 0)), "flops": 16 * P}
    if case["op"] == "gn":
        n, e = case["N"] * case["L"] * case["C"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * e * (3 if case["backward"] else 2) + 8 * case["N"] * case["G"] + 8 * case["C"] * (2 if case["backward"] else 1), "flops": n * (16 if case["backward"] else 9)}
    M, N, K = case["M"], case["N"], case["K"]
    if case["backward"]:
        z = case["act"] != "none"
        return {"bytes": 2 * (2 * M * K + 2 * N * K + M * N * (2 if z else 1) + N), "flops": 4 * M * N * K}
    return {"bytes": 2 * (M * K + N * K + N + M * N * (1 + case["residual"] + (case["save"] and case["act"] != "none"))), "flops": 2 * M * N * K}


def _exact_adamw(case, seed):
    """Tensor by tensor, from the definition: t = 37 steps of bias correction, decoupled decay, block codes."""
    global own
    was, own = own, False
    s = _prepare_adamw(case, seed)
    own = was
    h, nb = HYPER, s["nb"]
    P64 = s["p"].double()
    C64 = s["copy"].double() if s["copy"] is not None else None
    M64 = torch.zeros(nb * BLOCK, dtype=torch.float64, device="cuda")
    V64 = torch.zeros(nb * BLOCK, dtype=torch.float64, device="cuda")
    coef, out = 1.0, {}
    if case["clip"]:
        total = sum(float((s["grad"][a:a + n].double() ** 2).sum()) for a, n in zip(s["starts"], s["sizes"]))
        norm = math.sqrt(total)
        coef = min(1.0, 1.0 / (norm + 1e-6))
        out["norm"], out["coef"] = norm, coef
    elif case["bits"] == 8:
        coef = float(s["scale"])
    key = (seed * 0x85EBCA6B + 0x1B873593) % 2 ** 32
    block = 0
    for a, n, dec in zip(s["starts"], s["sizes"], s["decay"]):
        for lo in range(0, n, TILE):
            k = min(TILE, n - lo)
            q = -(-k // BLOCK)
            i0 = block * BLOCK + lo
            span = slice(i0, i0 + q * BLOCK)
            pad = lambda x: torch.nn.functional.pad(x.double(), (0, q * BLOCK - k)).view(q, BLOCK)  # noqa: E731
            g = pad(s["grad"][a + lo:a + lo + k]) * coef
            if case["bits"] == 8:
                bs = slice(i0 // BLOCK, i0 // BLOCK + q)
                cm, cv = s["m"][span].double().view(q, BLOCK), s["v"][span].double().view(q, BLOCK)
                m = torch.sign(cm) * (cm / 127) ** 2 * s["m_scale"][bs, None].double()
                v = ((cv / 255) ** 2 * s["v_scale"][bs, None].double()) ** 2
            else:
                m, v = s["m"][span].double().view(q, BLOCK), s["v"][span].double().view(q, BLOCK)
            m = h["beta1"] * m + (1 - h["beta1"]) * g
            v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
            mhat, vhat = m / (1 - h["beta1"] ** h["t"]), v / (1 - h["beta2"] ** h["t"])
            p = pad(s["p"][a + lo:a + lo + k])
            p = p - h["lr"] * mhat / (vhat ** 0.5 + h["eps"]) - (h["lr"] * h["weight_decay"] * p if dec else 0)
            P64[a + lo:a + lo + k] = p.reshape(-1)[:k]
            if C64 is not None:
                C64[a + lo:a + lo + k] = p.reshape(-1)[:k]
            if case["bits"] == 8:
                w = (torch.arange(i0, i0 + q * BLOCK, device="cuda") * 0x9E3779B1 + key) % 2 ** 32
                w = (w ^ (w >> 16)) * 0x85EBCA6B % 2 ** 32
                w = (w ^ (w >> 13)) * 0xC2B2AE35 % 2 ** 32
                w = (w ^ (w >> 16)).view(q, BLOCK)
                am, av = m.abs().max(1, keepdim=True).values, v.max(1, keepdim=True).values.sqrt()
                r = v.sqrt()
                cm = torch.minimum(((m.abs() / am).nan_to_num(0.0) ** 0.5 * 127 + (w % 65536) / 65536).floor(), torch.tensor(127.0, device="cuda"))
                cv = torch.minimum(((r / av).nan_to_num(0.0) ** 0.5 * 255 + (w // 65536) / 65536).floor(), torch.tensor(255.0, device="cuda"))
                cv = torch.where(r > 0, torch.maximum(cv, torch.ones_like(cv)), torch.zeros_like(cv))
                m, v = torch.sign(m) * (cm / 127) ** 2 * am, ((cv / 255) ** 2 * av) ** 2
            M64[span], V64[span] = m.reshape(-1), v.reshape(-1)
        block += -(-n // BLOCK)
    out.update(p=P64, m=M64, v=V64)
    if C64 is not None:
        out["copy"] = C64
    return out


def _exact_gn(case, seed):
    s = _prepare_gn(case, seed)
    N, C, G = case["N"], case["C"], case["G"]
    k = C // G
    parts = {"y": [], "mean": [], "rstd": [], "dx": []}
    dw = db = 0.0
    w, b = s["w"].double(), s["b"].double()

    def act(u):
        if case["act"] == "relu":
            return torch.where(u > 0, u, 0.0), torch.where(u > 0, 1.0, 0.0)
        if case["act"] == "silu":
            e = 1 / (1 + torch.exp(-u))
            return u * e, e + u * e * (1 - e)
        if case["act"] == "gelu":
            c = 0.5 * torch.erfc(-u / 2 ** 0.5)
            return u * c, c + u * torch.exp(-u * u / 2) / (2 * math.pi) ** 0.5
        return u, torch.ones_like(u)

    per = max(1, TILE // (case["L"] * C))
    for i in range(0, N, per):
        x = s["x"][i:i + per].double()
        n = x.shape[0]
        by = x.view(n, -1, G, k).transpose(1, 2).reshape(n, G, -1) if x.is_contiguous() else x.unflatten(2, (G, k)).transpose(1, 2).reshape(n, G, -1)
        if case["backward"]:
            mean, rstd = s["mean"][i:i + per].double(), s["rstd"][i:i + per].double()
        else:
            mean = by.mean(2)
            rstd = (by.var(2, unbiased=False) + s["eps"]) ** -0.5
        full = lambda t: t.repeat_interleave(k, 1)[:, None, :]  # noqa: E731
        xh = (x - full(mean)) * full(rstd)
        y, slope = act(xh * w + b)
        if not case["backward"]:
            parts["y"].append(y)
            parts["mean"].append(mean)
            parts["rstd"].append(rstd)
            continue
        du = s["dy"][i:i + per].double() * slope
        dw, db = dw + (du * xh).sum((0, 1)), db + du.sum((0, 1))
        e = du * w
        group = lambda t: full(t.sum(1).view(n, G, k).sum(2) / (k * case["L"]))  # noqa: E731
        parts["dx"].append((e - group(e) - xh * group(e * xh)) * full(rstd))
    out = {name: torch.cat(v) for name, v in parts.items() if v}
    if case["backward"]:
        out["dw"], out["db"] = dw, db
    return out


def _exact_linear(case, seed):
    s = _prepare_linear(case, seed)
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()

    def value(z):
        return {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0), "silu": lambda: z / (1 + torch.exp(-z)),
                "gelu": lambda: z * 0.5 * torch.erfc(-z / 2 ** 0.5)}[case["act"]]()

    if not case["backward"]:
        z = torch.addmm(b, x, w.T)
        y = value(z) + (s["r"].double() if case["residual"] else 0)
        return {"y": y, "z": z} if case["save"] and case["act"] != "none" else {"y": y}
    dz = s["dy"].double()
    if case["act"] != "none":
        z = s["z"].double().requires_grad_(True)
        (slope,) = torch.autograd.grad(value(z).sum(), z)
        dz = dz * slope
    return {"dx": dz.mm(w), "dw": dz.T.mm(x), "db": dz.sum(0)}


def exact(case, seed):
    return {"adamw": _exact_adamw, "gn": _exact_gn, "linear": _exact_linear}[case["op"]](case, seed)
