"""The matrix product with bias, activation and residual, and its gradient, against the definition in fp64: every
tile width, the exchanged and the split forms, odd extents, any alignment, and refusals.

Tolerances are forward error bounds with e = 2^-24. Products of two bf16 are exact in fp32; a sum of k of them takes
at most k additions that may truncate, so it is within 2 k e of the sum of magnitudes. An activation (slope at
most 1.13) adds 8 e (1 + |u|) |u|, its slope 8 e (1 + |u|) |dy|. A value rounded to bf16 moves by at most 2^-8 of itself:
outputs, and dz where there is an activation."""
import math

import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = 2.0 ** -8


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def act64(torch, u, act):
    if act == "relu":
        return torch.where(u > 0, u, 0.0), (u > 0).double()
    if act == "silu":
        s = torch.sigmoid(u)
        return u * s, s * (1 + u * (1 - s))
    if act == "gelu":
        c = 0.5 * torch.erfc(-u / math.sqrt(2))
        return u * c, c + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    return u, torch.ones_like(u)


def mat(g, M, N, slack=0, offset=0, scale=1.0):
    """A bf16 matrix whose rows are N + slack elements apart, starting `offset` elements into its memory."""
    import torch
    flat = (torch.randn(M * (N + slack) + offset + 8, generator=g, device="cuda") * scale).bfloat16()
    return flat[offset:offset + M * (N + slack)].view(M, N + slack)[:, :N]


def check(got, ref, err, what):
    tol = err + U * (ref.abs() + err) + 1e-38
    bad = (got.double() - ref).abs() / tol
    assert bad.max() <= 1, (what, float(bad.max()))


def run(M, N, K, act="none", residual=False, bias=True, slack=(0, 0, 0), offset=(0, 0, 0), seed=0):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, w = mat(g, M, K, slack[0], offset[0]), mat(g, N, K, slack[1], offset[1], K ** -0.5)
    b = mat(g, 1, N, 0, offset[2], 0.5)[0] if bias else None
    r = mat(g, M, N, slack[2], offset[2]) if residual else None
    y, z = D.linear(x, w, b, act=act, residual=r, save=True)
    X, W = x.double(), w.double()
    u = X @ W.t() + (b.double() if bias else 0)
    eu = 2 * (K + 2) * E * (X.abs() @ W.abs().t() + (b.double().abs() if bias else 0))
    v, _ = act64(torch, u, act)
    ev = eu if act == "none" else 1.13 * eu + 8 * E * (1 + u.abs()) * u.abs()
    if residual:
        v = v + r.double()
        ev = ev + E * v.abs()
    check(y, v, ev, "y")
    if act == "none":
        assert z is None
    else:
        check(z, u, eu, "z")
    # backward, from z as saved
    dy = mat(g, M, N, slack[2], offset[2])
    z = z if act != "none" else None
    dx, dw, db = D.linear_backward(dy, x, w, z, act=act)
    DY = dy.double()
    if act == "none":
        dz, edz, rdz = DY, torch.zeros_like(DY), torch.zeros_like(DY)
    else:
        Z = z.double()
        _, s = act64(torch, Z, act)
        dz = DY * s
        edz = torch.zeros_like(DY) if act == "relu" else 8 * E * (1 + Z.abs()) * DY.abs() + 2 * E * dz.abs()
        rdz = U * (dz.abs() + edz) + edz
    check(dx, dz @ W, rdz @ W.abs() + 2 * (N + 1) * E * ((dz.abs() + rdz) @ W.abs()), "dx")
    check(dw, dz.t() @ X, rdz.t() @ X.abs() + 2 * (M + 1) * E * ((dz.abs() + rdz).t() @ X.abs()), "dw")
    check(db, dz.sum(0), edz.sum(0) + (M / 64 + 40) * E * dz.abs().sum(0), "db")
    again = D.linear(x, w, b, act=act, residual=r, save=True)[0]
    assert torch.equal(again, y)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), D.linear_backward(dy, x, w, z, act=act)))
    assert D.linear_status() == 0


@pytest.mark.parametrize("M,N,K", [(128, 128, 64), (128, 256, 64), (256, 64, 128), (1, 128, 64), (32, 128, 64), (33, 128, 64), (64, 256, 192),
                                   (65, 128, 64), (300, 520, 200), (1000, 768, 512), (2048, 1024, 512)])
def test_aligned(M, N, K):
    run(M, N, K)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M", [5, 200])
def test_epilogues(act, residual, M):
    run(M, 264, 136, act, residual)
    run(M, 264, 136, act, residual, bias=False)


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 7, 3), (2, 1, 9), (3, 5, 8), (17, 33, 65), (127, 129, 63), (129, 127, 513), (777, 1000, 513), (70, 31, 1), (1, 1000, 4097)])
def test_odd(M, N, K):
    run(M, N, K, "gelu", True)


@pytest.mark.parametrize("M,N,K", [(1, 512, 4096), (8, 128, 8192), (40, 384, 2048), (100, 40, 5000), (128, 128, 4096), (256, 256, 3000)])
def test_split_and_exchanged(M, N, K):
    run(M, N, K, "silu", True)


@pytest.mark.parametrize("slack,offset", [((8, 16, 24), (0, 0, 0)), ((3, 0, 0), (0, 0, 0)), ((0, 5, 1), (0, 0, 0)), ((0, 0, 0), (1, 3, 5)), ((8, 8, 8), (8, 8, 8)), ((1, 2, 3), (4, 5, 6))])
@pytest.mark.parametrize("M", [9, 150])
def test_strides_and_starts(slack, offset, M):
    run(M, 136, 72, "relu", True, slack=slack, offset=offset)
    run(M, 131, 77, "none", True, slack=slack, offset=offset)


def test_many_tiles_reuse_both_accumulators():
    run(4096, 3000, 320, "gelu")
    run(20000, 128, 64, "relu", True)


def test_outputs_given_and_in_place():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w, b, r = mat(g, 100, 64), mat(g, 72, 64), mat(g, 1, 72)[0], mat(g, 100, 72)
    y, _ = D.linear(x, w, b, residual=r)
    out = r.clone()
    assert D.linear(x, w, b, residual=out, out=out)[0] is out and torch.equal(out, y)
    dy = mat(g, 100, 72)
    dx, dw, db = D.linear_backward(dy, x, w)
    flat = torch.zeros(3 + 72 * 64 + 72, dtype=torch.bfloat16, device="cuda")        # a flat gradient vector, packed from an odd place
    D.linear_backward(dy, x, w, need=(False, True, True), out=(None, flat[3:3 + 72 * 64].view(72, 64), flat[3 + 72 * 64:]))
    assert torch.equal(flat[3:3 + 72 * 64].view(72, 64), dw) and torch.equal(flat[3 + 72 * 64:], db) and not flat[:3].any()
    only = D.linear_backward(dy, x, w, need=(True, False, False))
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None


def test_against_differences():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w, b, dy = mat(g, 12, 24), mat(g, 16, 24, scale=0.2), mat(g, 1, 16)[0], mat(g, 12, 16)
    _, z = D.linear(x, w, b, act="gelu", save=True)
    dx, dw, db = D.linear_backward(dy, x, w, z, act="gelu")

    def loss(X, W, Bv):
        return float((act64(torch, X @ W.t() + Bv, "gelu")[0] * dy.double()).sum())

    h = 1e-5
    # the analytic gradient is taken at z rounded to bf16 (slope moves by 1.2 * 2^-8 |z|) and rounded twice more
    for k, (t, gr, idx) in enumerate(((x, dx, (3, 7)), (w, dw, (5, 11)), (b, db, (9,)))):
        args = [x.double(), w.double(), b.double()]
        hi, lo = args[k].clone(), args[k].clone()
        hi[idx] += h
        lo[idx] -= h
        num = (loss(*[hi if i == k else a for i, a in enumerate(args)]) - loss(*[lo if i == k else a for i, a in enumerate(args)])) / (2 * h)
        scale = {0: dy[3].double().abs() @ w[:, 7].double().abs(), 1: dy[:, 5].double().abs() @ x[:, 11].double().abs(), 2: dy[:, 9].double().abs().sum()}[k]
        assert abs(num - float(gr[idx])) <= float((1.2 * U * z.abs().max().double() + 3 * U) * scale), (k, num, float(gr[idx]))


def test_empty_and_degenerate():
    torch, D = _d()
    e = lambda *s: torch.ones(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    assert D.linear(e(0, 8), e(16, 8))[0].shape == (0, 16)
    assert D.linear(e(4, 8), e(0, 8))[0].shape == (4, 0)
    y, z = D.linear(e(4, 0), e(16, 0), 2 * e(16), act="relu", residual=e(4, 16), save=True)
    assert torch.equal(y, 3 * e(4, 16)) and torch.equal(z, 2 * e(4, 16))
    dx, dw, db = D.linear_backward(e(0, 16), e(0, 8), e(16, 8))
    assert dx.shape == (0, 8) and not dw.any() and not db.any()
    dx, dw, db = D.linear_backward(e(4, 0), e(4, 8), e(0, 8))
    assert not dx.any() and dw.shape == (0, 8)


def test_nan_and_infinity_stay_in_their_rows():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(5)
    for M in (20, 200):
        x, w = mat(g, M, 100), mat(g, 50, 100)
        clean = D.linear(x, w)[0]
        x[7, 99] = float("nan")
        x[11, 0] = float("inf")
        y = D.linear(x, w)[0]
        rows = [i for i in range(M) if i not in (7, 11)]
        assert torch.isnan(y[7]).all() and not torch.isfinite(y[11]).any() and torch.equal(y[rows], clean[rows])


def test_broadcast_inputs():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(7)
    for M in (40, 200):
        x, w, r, dy = mat(g, 1, 64).expand(M, 64), mat(g, 72, 64), mat(g, 1, 72).expand(M, 72), mat(g, 1, 72).expand(M, 72)
        y, z = D.linear(x, w, act="gelu", residual=r, save=True)
        same = D.linear(x.contiguous(), w, act="gelu", residual=r.contiguous(), save=True)
        assert torch.equal(y, same[0]) and torch.equal(z, same[1])
        a, b = D.linear_backward(dy, x, w, z, act="gelu"), D.linear_backward(dy.contiguous(), x.contiguous(), w, z, act="gelu")
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        a, b = D.linear_backward(dy, x, w), D.linear_backward(dy.contiguous(), x.contiguous(), w)
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_other_stream_and_graph():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w, b, dy = mat(g, 300, 200, 3), mat(g, 136, 200), mat(g, 1, 136)[0], mat(g, 300, 136)
    ref = D.linear(x, w, b, act="silu", save=True)
    rb = D.linear_backward(dy, x, w, ref[1], act="silu")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y, z = D.linear(x, w, b, act="silu", save=True)
            back = D.linear_backward(dy, x, w, z, act="silu")
        graph.replay()
        graph.replay()
    side.synchronize()
    assert torch.equal(y, ref[0]) and all(torch.equal(p, q) for p, q in zip(back, rb))


def test_refusals():
    torch, D = _d()
    e = lambda *s: torch.ones(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for f in (lambda: D.linear(e(4, 8).float(), e(16, 8)), lambda: D.linear(e(4, 8), e(16, 9)), lambda: D.linear(e(4, 8), e(16, 8), e(15)),
              lambda: D.linear(e(4, 8), e(16, 8), act="tanh"), lambda: D.linear(e(4, 8), e(16, 8), residual=e(4, 15)), lambda: D.linear(e(8, 4).t(), e(16, 8)),
              lambda: D.linear(e(4, 8).cpu(), e(16, 8)), lambda: D.linear(e(4, 8), e(16, 8), out=e(1, 16).expand(4, 16)), lambda: D.linear_backward(e(4, 16), e(4, 8), e(16, 8), act="relu"),
              lambda: D.linear_backward(e(4, 15), e(4, 8), e(16, 8)), lambda: D.linear(e(8), e(16, 8))):
        with pytest.raises(D.DmxError):
            f()
