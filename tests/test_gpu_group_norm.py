"""Group norm with an activation, channels last, against the definition in fp64: both types, every activation, shapes from one value to
several thousand positions, odd channels and groups, slices, large means, constant groups, and the gradient
against the formula and against differences.

Tolerances are forward error bounds with e = 2^-24. A value passes at most G = 150 additions on its way into a sum (64 in a
thread, 8 in a column, 64 and 5 in a group, 8 over a cluster or the chunks of a large image), so a sum is within
G e of the sum of magnitudes; a variance of deviations within (G + 8) e of itself plus the square of the mean's error. Errors
then follow the formulas term by term. bf16 results get half a spacing (2^-8 of the value) more."""
import math

import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
GAMMA = 150 * E


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def act64(torch, u, act):
    """value, slope"""
    if act == "relu":
        return torch.where(u > 0, u, 0.0), (u > 0).double()
    if act == "silu":
        s = torch.sigmoid(u)
        return u * s, s * (1 + u * (1 - s))
    if act == "gelu":
        c = 0.5 * torch.erfc(-u / math.sqrt(2))
        return u * c, c + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    return u, torch.ones_like(u)


def make(N, L, C, dtype, slack=0, mean=0.0, seed=0):
    torch, _ = _d()
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(N, L, C + slack, generator=g, device="cuda") * 1.5 + mean
    return x.to(dtype)[:, :, :C], torch.randn(N, L, C + slack, generator=g, device="cuda").to(dtype)[:, :, :C], \
        1 + 0.3 * torch.randn(C, generator=g, device="cuda"), 0.3 * torch.randn(C, generator=g, device="cuda")


def check_forward(x, G, w, b, eps, act, got):
    torch, _ = _d()
    y, mean, rstd = got
    N, L, C = x.shape
    k = C // G
    X = x.double().reshape(N, L, G, k)
    mu = X.mean((1, 3), keepdim=True)
    dmu = GAMMA * X.abs().mean((1, 3), keepdim=True) + 2 * E * mu.abs()
    d = X - mu
    var = d.square().mean((1, 3), keepdim=True)
    dvar = (GAMMA + 8 * E) * var + 2 * dmu.square()
    rs = (var + eps) ** -0.5
    lo = torch.clamp(var - dvar, min=0) + eps * (1 - E)
    drs = torch.maximum(rs - (var + dvar + eps * (1 + E)) ** -0.5, torch.where(lo > 0, lo, torch.inf) ** -0.5 - rs) + 3 * E * rs
    assert torch.all((mean.double() - mu[:, 0, :, 0]).abs() <= dmu[:, 0, :, 0])
    assert torch.all((rstd.double() - rs[:, 0, :, 0]).abs() <= drs[:, 0, :, 0])
    W = torch.ones(C, device="cuda").double() if w is None else w.double()
    Bv = torch.zeros(C, device="cuda").double() if b is None else b.double()
    W, Bv = W.view(G, k), Bv.view(G, k)
    u = d * rs * W + Bv
    du = W.abs() * (rs * (dmu + E * d.abs()) + drs * (d.abs() + dmu)) + 2 * E * (d * rs * W).abs() + E * u.abs() + W.abs() * rs * dmu
    ref, _ = act64(torch, u, act)
    tol = 1.13 * du + (0 if act in ("none", "relu") else 8 * E * (1 + u.abs()) * u.abs()) + 1e-37
    if y.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
    err = (y.double().reshape(N, L, G, k) - ref).abs()
    assert torch.all(err <= tol), float((err / tol).max())


def check_backward(dy, x, mean, rstd, G, w, b, act, got):
    torch, _ = _d()
    dx, dw, db = got
    N, L, C = x.shape
    k, n = C // G, L * (C // G)
    sh = lambda t: t.double().reshape(N, L, G, k)  # noqa: E731
    X, DY = sh(x), sh(dy)
    mu, rs = mean.double()[:, None, :, None], rstd.double()[:, None, :, None]
    W = (torch.ones(C, device="cuda") if w is None else w).double().view(G, k)
    Bv = (torch.zeros(C, device="cuda") if b is None else b).double().view(G, k)
    xh = (X - mu) * rs
    u = xh * W + Bv
    eu = 3 * E * (xh * W).abs() + E * u.abs()
    _, slope = act64(torch, u, act)
    du = DY * slope
    if act == "none":
        edu = torch.zeros_like(du)
    elif act == "relu":
        edu = torch.where(u.abs() <= eu, DY.abs(), 0.0)
    else:
        edu = DY.abs() * (1.2 * eu + 8 * E * (1 + u.abs())) + E * du.abs()
    A, Bs = (du * xh).sum(1), du.sum(1)                                 # (N, G, k)
    eA = (edu * xh.abs() + 4 * E * (du * xh).abs()).sum(1) + GAMMA * (du * xh).abs().sum(1)
    eB = edu.sum(1) + GAMMA * du.abs().sum(1)
    s2, s1 = (A * W).sum(2)[:, None, :, None] / n, (Bs * W).sum(2)[:, None, :, None] / n
    e2 = ((eA + GAMMA * A.abs()) * W.abs()).sum(2)[:, None, :, None] / n
    e1 = ((eB + GAMMA * Bs.abs()) * W.abs()).sum(2)[:, None, :, None] / n
    ref = rs * (du * W - s1 - xh * s2)
    tol = rs * (W.abs() * (edu + 2 * E * du.abs()) + e1 + xh.abs() * e2 + 6 * E * ((W * du).abs() + s1.abs() + (xh * s2).abs())) + 1e-37
    if dx.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
    err = (sh(dx) - ref).abs()
    assert torch.all(err <= tol), float((err / tol).max())
    # over the images: N/8 additions in a row, 8 rows
    g2 = (N / 8 + 10) * E
    for out, S, eS in ((dw, A, eA), (db, Bs, eB)):
        e = (out.double() - S.sum(0).reshape(-1)).abs()
        t = (eS.sum(0) + g2 * S.abs().sum(0)).reshape(-1) + 1e-37
        assert torch.all(e <= t), float((e / t).max())


# N, L, C, G, slack
SHAPES = [
    (1, 1, 1, 1, 0), (1, 1, 8, 8, 0), (2, 1, 8, 1, 0), (3, 2, 6, 3, 0), (1, 7, 16, 4, 0), (5, 9, 24, 3, 0), (2, 33, 30, 10, 0), (2, 64, 256, 32, 0),
    (1, 64, 256, 32, 8), (3, 49, 90, 15, 7), (2, 49, 96, 12, 3), (70, 16, 512, 32, 0), (300, 4, 40, 8, 0), (2, 1024, 64, 16, 0), (1, 3136, 64, 8, 0),
    (2, 729, 90, 15, 7), (1, 5000, 8, 2, 0), (1, 300, 2048, 2, 0), (1, 20, 1023, 1, 0), (1, 20, 1023, 1, 1), (2, 5, 3000, 3, 0), (1, 40000, 32, 4, 0),
    (2, 9001, 33, 3, 2), (1, 12, 16384, 16, 0), (4, 100, 200, 5, 0),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_shapes(shape, dtype):
    torch, D = _d()
    N, L, C, G, slack = shape
    act = ["none", "relu", "silu", "gelu"][(N + L + C) % 4]
    x, dy, w, b = make(N, L, C, getattr(torch, dtype), slack)
    got = D.group_norm(x, G, w, b, 1e-5, act)
    check_forward(x, G, w, b, 1e-5, act, got)
    y2, m2, r2 = D.group_norm(x, G, w, b, 1e-5, act)
    assert torch.equal(got[0], y2) and torch.equal(got[1], m2) and torch.equal(got[2], r2)
    back = D.group_norm_backward(dy, x, got[1], got[2], G, w, b, act)
    check_backward(dy, x, got[1], got[2], G, w, b, act, back)
    again = D.group_norm_backward(dy, x, got[1], got[2], G, w, b, act)
    assert all(torch.equal(p, q) for p, q in zip(back, again))


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_activations_without_weights_and_in_place(act, dtype):
    torch, D = _d()
    x, dy, w, b = make(4, 50, 64, getattr(torch, dtype), seed=3)
    for ww, bb in ((None, None), (w, None), (None, b), (w, b)):
        got = D.group_norm(x, 8, ww, bb, 1e-3, act)
        check_forward(x, 8, ww, bb, 1e-3, act, got)
        back = D.group_norm_backward(dy, x, got[1], got[2], 8, ww, bb, act)
        check_backward(dy, x, got[1], got[2], 8, ww, bb, act, back)
        z = x.clone()
        D.group_norm(z, 8, ww, bb, 1e-3, act, out=z)
        assert torch.equal(z, got[0])
        for target in (dy.clone(), x.clone()):
            src = (target, x) if target.data_ptr() != x.data_ptr() and torch.equal(target, dy) else (dy, target)
            out = D.group_norm_backward(src[0], src[1], got[1], got[2], 8, ww, bb, act, out=target)
            assert torch.equal(out[0], back[0])


@pytest.mark.parametrize("L", [5, 1024, 30000])
def test_large_mean_and_constant_groups(L):
    # the variance is taken from deviations: a mean a thousand deviations away costs nothing
    torch, D = _d()
    x, _, w, b = make(2, L, 32, torch.float32, mean=1500.0)
    x[1] = 7.25
    got = D.group_norm(x, 4, w, b, 1e-5, "none")
    check_forward(x, 4, w, b, 1e-5, "none", got)
    assert torch.all((got[2][1] - 1e-5 ** -0.5).abs() < 1e-3 * 1e-5 ** -0.5)


def test_outlier_first_position():
    torch, D = _d()
    x, _, w, b = make(1, 2000, 16, torch.float32)
    x[0, 0] = 3e4
    check_forward(x, 2, w, b, 1e-5, "none", D.group_norm(x, 2, w, b, 1e-5, "none"))


def test_a_nan_stays_in_its_group():
    torch, D = _d()
    x, _, w, b = make(2, 300, 32, torch.float32)
    clean = D.group_norm(x, 4, w, b, 1e-5, "relu")[0].clone()
    x[1, 17, 9] = float("nan")
    x[0, 3, 31] = float("inf")
    y, mean, rstd = D.group_norm(x, 4, w, b, 1e-5, "relu")
    assert torch.isnan(y[1, :, 8:16]).all() and torch.isnan(mean[1, 1]) and torch.isnan(y[0, :, 24:]).all()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1, :, 8:16] = False
    keep[0, :, 24:] = False
    assert torch.equal(y[keep], clean[keep])


def test_image_tensors_and_transposed_batches():
    torch, D = _d()
    x, dy, w, b = make(6, 35, 48, torch.bfloat16)
    got = D.group_norm(x, 6, w, b, act="silu")
    img = x.reshape(6, 5, 7, 48)
    assert torch.equal(D.group_norm(img, 6, w, b, act="silu")[0].reshape(6, 35, 48), got[0])
    base = torch.empty(35, 6, 48, dtype=torch.bfloat16, device="cuda")          # images interleaved by position
    base.copy_(x.transpose(0, 1))
    t = base.transpose(0, 1)
    assert torch.equal(D.group_norm(t, 6, w, b, act="silu")[0], got[0])
    back = D.group_norm_backward(dy, x, got[1], got[2], 6, w, b, "silu")
    assert all(torch.equal(p, q) for p, q in zip(back, D.group_norm_backward(dy, t, got[1], got[2], 6, w, b, "silu")))


def test_broadcast_inputs():
    torch, D = _d()
    x, dy, w, b = make(4, 60, 32, torch.bfloat16)
    _, mean, rstd = D.group_norm(x, 4, w, b, act="silu")
    for one in (dy[:, :1], dy[:1]):
        wide = one.expand(4, 60, 32)
        a = D.group_norm_backward(wide, x, mean, rstd, 4, w, b, "silu")
        c = D.group_norm_backward(wide.contiguous(), x, mean, rstd, 4, w, b, "silu")
        assert all(torch.equal(p, q) for p, q in zip(a, c))
    r = x[:1].expand(4, 60, 32)
    assert all(torch.equal(p, q) for p, q in zip(D.group_norm(r, 4, w, b), D.group_norm(r.contiguous(), 4, w, b)))


def test_against_differences():
    torch, D = _d()
    x, dy, w, b = make(2, 11, 12, torch.float32, seed=8)
    for act in ("none", "silu", "gelu"):
        def loss(x_, w_, b_):
            X = x_.double().reshape(2, 11, 3, 4)
            mu = X.mean((1, 3), keepdim=True)
            xh = (X - mu) * (X.var((1, 3), unbiased=False, keepdim=True) + 1e-5) ** -0.5
            u = (xh * w_.double().view(3, 4) + b_.double().view(3, 4)).reshape(2, 11, 12)
            return float((act64(torch, u, act)[0] * dy.double()).sum())

        _, mean, rstd = D.group_norm(x, 3, w, b, 1e-5, act)
        dx, dw, db = D.group_norm_backward(dy, x, mean, rstd, 3, w, b, act)
        h = 1e-5
        # central differences in fp64: truncation h^2/6 * third derivative (< 100 here), rounding 1e-16 * |loss| / h
        for t, gr, idx in ((x, dx, (1, 4, 7)), (x, dx, (0, 0, 0)), (w, dw, (5,)), (b, db, (11,))):
            hi, lo = t.double().clone(), t.double().clone()
            hi[idx] += h
            lo[idx] -= h
            args = lambda v: tuple(v if t is q else q for q in (x, w, b))  # noqa: E731
            num = (loss(*args(hi)) - loss(*args(lo))) / (2 * h)
            assert abs(num - float(gr[idx])) <= 2e-5 * (1 + abs(num)), (act, idx, num, float(gr[idx]))


def test_empty_problems():
    torch, D = _d()
    w, b = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    for shape in ((0, 5, 8), (3, 0, 8)):
        x = torch.empty(shape, device="cuda")
        y, mean, rstd = D.group_norm(x, 2, w, b)
        assert y.shape == shape
        dx, dw, db = D.group_norm_backward(x, x, mean, rstd, 2, w, b)
        assert dx.shape == shape and not dw.any() and not db.any()


def test_other_stream_and_graph():
    torch, D = _d()
    x, dy, w, b = make(3, 700, 90, torch.float32, 7)
    ref = D.group_norm(x, 15, w, b, act="gelu")
    rb = D.group_norm_backward(dy, x, ref[1], ref[2], 15, w, b, "gelu")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            y, m, r = D.group_norm(x, 15, w, b, act="gelu")
            back = D.group_norm_backward(dy, x, m, r, 15, w, b, "gelu")
        g.replay()
        g.replay()
    side.synchronize()
    assert torch.equal(y, ref[0]) and all(torch.equal(p, q) for p, q in zip(back, rb))


def test_refusals():
    torch, D = _d()
    x, dy, w, b = make(2, 10, 12, torch.float32)
    bad = [lambda: D.group_norm(x, 5, w, b), lambda: D.group_norm(x, 0, w, b), lambda: D.group_norm(x, 3, w[:11], b), lambda: D.group_norm(x, 3, w.double(), b),
           lambda: D.group_norm(x, 3, w, b, act="tanh"), lambda: D.group_norm(x, 3, w, b, eps=-1.0), lambda: D.group_norm(x.cpu(), 3), lambda: D.group_norm(x.half(), 3),
           lambda: D.group_norm(x.transpose(1, 2), 2), lambda: D.group_norm(x, 3, w, b, out=torch.empty(2, 10, 11, device="cuda")),
           lambda: D.group_norm(torch.zeros(1, 2, 1025, device="cuda"), 1), lambda: D.group_norm(x[:, :1].expand(2, 10, 12), 3, out=x[:, :1].expand(2, 10, 12))]
    for f in bad:
        with pytest.raises(D.DmxError):
            f()
    m = torch.zeros(2, 3, device="cuda")
    with pytest.raises(D.DmxError):
        D.group_norm_backward(dy, x, m[:1], m, 3, w, b)


def test_results_may_be_written_where_images_take_turns_by_rows():
    torch, D = _d()
    x, dy, w, b = make(3, 20, 16, torch.float32, seed=9)
    y, mean, rstd = D.group_norm(x, 4, w, b, act="silu")
    dx, dw, db = D.group_norm_backward(dy, x, mean, rstd, 4, w, b, act="silu")
    turns = torch.zeros(20, 3, 24, device="cuda")
    got = D.group_norm(x, 4, w, b, act="silu", out=turns.transpose(0, 1)[:, :, :16])
    assert torch.equal(got[0], y) and torch.equal(turns[..., :16].transpose(0, 1), y) and not turns[..., 16:].any()
    got = D.group_norm_backward(dy, x, mean, rstd, 4, w, b, act="silu", out=turns.transpose(0, 1)[:, :, :16])
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db) and not turns[..., 16:].any()
    with pytest.raises(D.DmxError):
        D.group_norm(x, 4, w, b, out=torch.empty(1, 20, 16, device="cuda").expand(3, 20, 16))
