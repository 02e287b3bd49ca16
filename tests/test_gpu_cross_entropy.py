"""The softmax cross entropy of a linear layer and its gradient against the definition in fp64.

Tolerances are forward error bounds with E = 2^-24, U = 2^-8 (half a step of bf16). A logit: products of two bf16 are exact in fp32, a sum of
D of them takes at most D additions that may truncate. A sum of exponentials: at most 64 additions in a chunk and one rescaling (2 ulp) and
addition per pair that is joined (an eighth of all pairs, then eight); a term's exponential is good to 2 ulp and its argument to E of
the distance, and zero below 2^-126 (the instruction flushes: an absolute error of one such number). The logarithm and the product with ln 2 add a few E of the result. G is rounded to bf16 before the two products, whose sums
are within 2 k E of their magnitudes."""
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = 2.0 ** -8


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def mat(g, M, N, slack=0, offset=0, scale=1.0):
    """A bf16 matrix whose rows are N + slack elements apart, starting `offset` elements into its memory."""
    import torch
    flat = (torch.randn(M * (N + slack) + offset + 8, generator=g, device="cuda") * scale).bfloat16()
    return flat[offset:offset + M * (N + slack)].view(M, N + slack)[:, :N]


def check(got, ref, err, what, half=0.0):
    tol = err + half * (ref.abs() + err) + 1e-38
    bad = (got.double() - ref).abs() / tol
    assert bad.max() <= 1, (what, float(bad.max()))


def compare(torch, D, x, w, target, b=None, dloss=None, need=(True, True, True), out=(None, None, None)):
    N, V, n = x.shape[0], w.shape[0], x.shape[1]
    loss, lse = D.linear_cross_entropy(x, w, target, b)
    assert loss.dtype == lse.dtype == torch.float32 and loss.shape == lse.shape == (N,)
    dloss = torch.full((1,), 1.0 / N, device="cuda").expand(N) if dloss is None else dloss
    got = D.linear_cross_entropy_backward(dloss, x, w, target, lse, b, need=need, out=out)
    X, W, Bv = x.double(), w.double(), (torch.zeros(V, device="cuda") if b is None else b).double()
    dx, dw, db = torch.empty(N, n, dtype=torch.float64, device="cuda"), torch.zeros_like(W), torch.zeros(V, dtype=torch.float64, device="cuda")
    ex, ew, eb = torch.empty_like(dx), torch.zeros_like(dw), torch.zeros_like(db)
    pairs = -(-V // 64) * 4
    step = max(1, min(N, 60_000_000 // V))
    for i in range(0, N, step):
        s = slice(i, i + step)
        xa, t = X[s], target[s].long()
        z = xa @ W.t() + Bv
        ez = 2 * (n + 2) * E * (xa.abs() @ W.abs().t() + Bv.abs())
        ref = torch.logsumexp(z, 1)
        p = torch.exp(z - ref[:, None])
        el = (p * ez.nan_to_num(0.0, 0.0)).sum(1) + E * (100 + 5 * (pairs / 8 + 10) + 2 * (p * (z - ref[:, None]).abs()).nan_to_num(0.0).sum(1)) + 6 * E * ref.abs()
        check(lse[s], ref, el, "lse")
        live = (t >= 0) & (t < V)
        at, rows = t.clamp(0, V - 1), torch.arange(len(t), device="cuda")
        want = torch.where(live, ref - z[rows, at], 0.0)
        check(loss[s], want, torch.where(live, el + ez[rows, at] + 2 * E * (ref.abs() + z[rows, at].abs()), 0.0), "loss")
        far = z - lse[s].double()[:, None]
        p = torch.exp(far)
        one = torch.zeros_like(p)
        one[rows, at] = live.double()
        d = torch.where(live, dloss[s].double(), 0.0)[:, None]
        G = (p - one) * d
        # (an exponential below 2^-126 is zero; its product with dloss and its rounding to bf16 may lose as much again)
        eg = (d.abs() * 2.0 ** -125 + 2.0 ** -125 + d.abs() * (p * (ez + 4 * E * far.abs() + 4 * E * lse[s].double().abs()[:, None] + 8 * E) + 4 * E * (p + one))).nan_to_num(0.0)
        eh = eg + U * (G.abs() + eg)
        dx[s], ex[s] = G @ W, eh @ W.abs() + 2 * (V + 2) * E * (G.abs() @ W.abs())
        dw += G.t() @ xa
        ew += eh.t() @ xa.abs() + 2 * (N + 2) * E * (G.abs().t() @ xa.abs())
        db += G.sum(0)
        eb += eg.sum(0) + (N + 2) * E * G.abs().sum(0)
    for o, ref, err, wanted, what in zip(got, (dx, dw, db), (ex, ew, eb), need, ("dx", "dw", "db")):
        if not wanted:
            assert o is None
            continue
        assert o.dtype == torch.bfloat16
        check(o, ref, err, what, U)
    assert D.linear_status() == 0
    return (loss, lse, *got)


def problem(torch, N, V, n, seed=0, bias=True, ignored=0.2, slack=(0, 0), offset=(0, 0), it="int64"):
    g = torch.Generator(device="cuda").manual_seed(seed + N + V + n)
    x, w = mat(g, N, n, slack[0], offset[0]), mat(g, V, n, slack[1], offset[1], 2.0 * n ** -0.5)
    b = mat(g, 1, V, 0, offset[1], 0.5)[0] if bias else None
    target = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=getattr(torch, it))
    miss = torch.rand(N, generator=g, device="cuda") < ignored
    target[miss] = torch.tensor([-100, -1, V, 2 ** 31 - 1], device="cuda")[torch.randint(0, 4, (N,), generator=g, device="cuda")].to(target.dtype)[miss]
    return x, w, target, b


# every tile width, pairs of CTAs, one and several tiles per CTA, odd extents (operands that are laid out first), one row, one word
SHAPES = [(1, 1, 1), (1, 2, 8), (2, 1, 64), (1, 30522, 64), (3, 10, 64), (128, 10, 64), (64, 1000, 200), (65, 257, 72), (100, 128, 513), (129, 129, 129), (777, 1000, 513),
          (1024, 2048, 512), (300, 5000, 1024), (4100, 300, 128), (2000, 7001, 96), (5000, 5000, 40), (33, 65537, 16), (16000, 33, 24), (40, 1000, 4096)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("bias", [False, True])
def test_shapes(shape, bias):
    torch, D = _d()
    x, w, t, b = problem(torch, *shape, bias=bias, it="int32" if shape[0] % 2 else "int64")
    first = compare(torch, D, x, w, t, b, need=(True, True, bias))
    lse = first[1]
    again = (*D.linear_cross_entropy(x, w, t, b), *D.linear_cross_entropy_backward(torch.full((shape[0],), 1.0 / shape[0], device="cuda"), x, w, t, lse, b, need=(True, True, bias)))
    assert all(a is c or torch.equal(a, c) for a, c in zip(first, again))


@pytest.mark.parametrize("N,V,n", [(8192, 30522, 72), (70000, 5003, 40), (20000, 20001, 264)])
def test_several_pieces_of_the_vocabulary(N, V, n):
    torch, D = _d()
    x, w, t, b = problem(torch, N, V, n)
    a = compare(torch, D, x, w, t, b)
    one = D.linear_cross_entropy_backward(torch.full((1,), 1.0 / N, device="cuda").expand(N), x, w, t, a[1], b, need=(True, False, False))
    assert torch.equal(one[0], a[2]) and one[1] is None and one[2] is None
    only = D.linear_cross_entropy_backward(torch.full((1,), 1.0 / N, device="cuda").expand(N), x, w, t, a[1], b, need=(False, False, True))
    assert only[0] is None and only[1] is None and torch.equal(only[2], a[4])


@pytest.mark.parametrize("slack,offset", [((8, 8), (0, 0)), ((3, 0), (0, 0)), ((0, 5), (0, 0)), ((8, 8), (1, 0)), ((0, 0), (0, 3)), ((1, 1), (1, 1))])
def test_strides_and_starts(slack, offset):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(3)
    for N, V, n in ((50, 300, 64), (200, 77, 65)):
        x, w, t, b = problem(torch, N, V, n, slack=slack, offset=offset)
        outs = (mat(g, N, n, slack[0], offset[0]), mat(g, V, n, slack[1], offset[1]), torch.zeros(V + 3, device="cuda", dtype=torch.bfloat16)[offset[1]:offset[1] + V])
        got = compare(torch, D, x, w, t, b, dloss=torch.randn(N, 3, generator=g, device="cuda")[:, 1], out=outs)
        assert all(a is c for a, c in zip(got[2:], outs))
    one = mat(g, 1, 64)
    x, w, t, b = problem(torch, 60, 90, 64)
    compare(torch, D, one.expand(60, 64), w, t, b)
    compare(torch, D, x, one.expand(90, 64), t, b)
    compare(torch, D, x, w, torch.stack([t, t], 1)[:, 0], b)


def test_logits_of_all_sizes():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(4)
    for scale in (1e-3, 30.0, 1e3):
        x, w, t, b = problem(torch, 200, 700, 64)
        compare(torch, D, (x * scale).bfloat16(), w, t, b)
    x, w, t, _ = problem(torch, 200, 700, 64)
    compare(torch, D, x * 0, w, t, None)                                     # all the same
    compare(torch, D, x, w, t, (torch.randn(700, generator=g, device="cuda") + 5000).bfloat16())
    # words that do not occur: whole tiles, all but one, the first of all
    b = torch.zeros(700, device="cuda", dtype=torch.bfloat16)
    for gone in (slice(0, 300), slice(256, 700), slice(0, 699), slice(1, 700), slice(0, 1)):
        c = b.clone()
        c[gone] = -float("inf")
        keep = torch.ones(700, dtype=torch.bool, device="cuda")
        keep[gone] = False
        tk = torch.nonzero(keep)[:, 0][t.clamp(0, 699) % int(keep.sum())]
        loss, lse = D.linear_cross_entropy(x, w, tk, c)
        small = D.linear_cross_entropy(x, w[keep].contiguous(), torch.cumsum(keep, 0)[tk] - 1, None)
        assert torch.allclose(loss, small[0], rtol=2e-5, atol=2e-5) and torch.allclose(lse, small[1], rtol=2e-5, atol=2e-5)
        dx, dw, db = D.linear_cross_entropy_backward(torch.ones(200, device="cuda"), x, w, tk, lse, c)
        assert dx.isfinite().all() and not dw[gone].any() and not db[gone].any() and dw.isfinite().all()


def test_rows_that_are_not_finite_stay_alone():
    torch, D = _d()
    x, w, t, b = problem(torch, 300, 400, 64, ignored=0.0)
    loss, lse = D.linear_cross_entropy(x, w, t, b)
    one = torch.ones(300, device="cuda")
    dx = D.linear_cross_entropy_backward(one, x, w, t, lse, b)[0]
    y = x.clone()
    y[7, 3], y[299, 0], y[130, 5] = float("nan"), float("inf"), -float("inf")
    t2 = t.clone()
    t2[130] = -1                                                             # an ignored row that is not finite
    l2, e2 = D.linear_cross_entropy(y, w, t2, b)
    hit = torch.zeros(300, dtype=torch.bool, device="cuda")
    hit[[7, 299, 130]] = True
    assert torch.equal(l2[~hit], loss[~hit]) and torch.equal(e2[~hit], lse[~hit]) and l2[[7, 299]].isnan().all() and l2[130] == 0
    got = D.linear_cross_entropy_backward(one, y, w, t2, e2, b)
    assert torch.equal(got[0][~hit], dx[~hit]) and got[0][[7, 299]].isnan().all() and not got[0][130].any()


def test_weights_of_rows():
    """dloss of any size and sign, zeros, and values that are not finite, which stay in their rows of dx."""
    torch, D = _d()
    x, w, t, b = problem(torch, 300, 400, 64)
    g = torch.Generator(device="cuda").manual_seed(11)
    r = torch.randn(300, generator=g, device="cuda")
    for d in (r, r * 1e-30, r * 1e20, r * torch.exp(20 * torch.randn(300, generator=g, device="cuda")), torch.where(r > 0, r, 0.0), r * 0, -torch.ones(300, device="cuda")):
        compare(torch, D, x, w, t, b, dloss=d)
    lse = D.linear_cross_entropy(x, w, t, b)[1]
    want = D.linear_cross_entropy_backward(r, x, w, t, lse, b)[0]
    for odd in (float("nan"), float("inf")):
        d = r.clone()
        live = torch.nonzero((t >= 0) & (t < 400))[:, 0]
        d[live[5]] = odd
        keep = torch.ones(300, dtype=torch.bool, device="cuda")
        keep[live[5]] = False
        if float(r[live[5]].abs()) == float(r.abs().max()):
            continue
        dx, dw, db = D.linear_cross_entropy_backward(d, x, w, t, lse, b)
        assert torch.equal(dx[keep], want[keep]) and not dx[live[5]].isfinite().any() and not dw.isfinite().any() and not db.isfinite().any()
    d = torch.zeros(300, device="cuda")
    d[live[5]] = float("nan")
    assert D.linear_cross_entropy_backward(d, x, w, t, lse, b)[0][live[5]].isnan().all()


def test_nothing_to_do():
    torch, D = _d()
    w = torch.randn(30, 16, device="cuda").bfloat16()
    x, t = w[:0], torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = D.linear_cross_entropy(x, w, t)
    dx, dw, db = D.linear_cross_entropy_backward(loss, x, w, t, lse)
    assert loss.shape == (0,) and dx.shape == (0, 16) and not dw.any() and not db.any()
    x, t = torch.randn(50, 16, device="cuda").bfloat16(), torch.full((50,), -100, device="cuda")
    loss, lse = D.linear_cross_entropy(x, w, t)                              # every row ignored
    got = D.linear_cross_entropy_backward(torch.ones(50, device="cuda"), x, w, t, lse)
    assert not loss.any() and not any(o.any() for o in got)
    assert D.linear_cross_entropy_backward(torch.ones(50, device="cuda"), x, w, t, lse, need=(False, False, False)) == (None, None, None)


def test_gradient_against_differences():
    """The slope of the mean loss along random directions, by central differences of the definition in 64 bits at bf16 points."""
    torch, D = _d()
    x, w, t, b = problem(torch, 90, 150, 40)
    n = int(((t >= 0) & (t < 150)).sum())
    loss, lse = D.linear_cross_entropy(x, w, t, b)
    grads = D.linear_cross_entropy_backward(torch.full((90,), 1.0 / n, device="cuda"), x, w, t, lse, b)
    at = [v.double() for v in (x, w, b)]
    live = (t >= 0) & (t < 150)

    def value(p):
        z = p[0] @ p[1].t() + p[2]
        return float((torch.logsumexp(z, 1) - z[torch.arange(90, device="cuda"), t.clamp(0, 149)])[live].sum() / n)
    assert abs(value(at) - float(loss.double().sum() / n)) < 1e-5
    g = torch.Generator(device="cuda").manual_seed(5)
    for i in range(3):
        v = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-5
        slope = (value([p + e * v if j == i else p for j, p in enumerate(at)]) - value([p - e * v if j == i else p for j, p in enumerate(at)])) / (2 * e)
        mine = grads[i].double() * v
        assert abs(slope - float(mine.sum())) <= 3 * U * float(mine.abs().sum())     # an entry: two roundings to bf16 and the fp32 errors


def test_recorded_for_differentiation():
    torch, D = _d()
    x, w, t, b = problem(torch, 60, 90, 32)
    loss, lse = D.linear_cross_entropy(x, w, t, b)
    g = torch.rand(60, device="cuda")
    want = D.linear_cross_entropy_backward(g, x, w, t, lse, b)
    leaves = [v.clone().requires_grad_(True) for v in (x, w, b)]
    l2, e2 = D.linear_cross_entropy(leaves[0], leaves[1], t, leaves[2])
    assert torch.equal(l2, loss) and l2.requires_grad and not e2.requires_grad
    l2.backward(g)
    assert all(torch.equal(v.grad, o) for v, o in zip(leaves, want))
    p = torch.nn.Parameter(w.clone())
    D.linear_cross_entropy(x, p, t)[0].mean().backward()                     # an expanded gradient, only the weight, no bias
    lse = D.linear_cross_entropy(x, w, t)[1]
    assert torch.equal(p.grad, D.linear_cross_entropy_backward(torch.full((1,), 1 / 60, device="cuda").expand(60), x, w, t, lse, need=(False, True, False))[1])
    with torch.no_grad():
        assert not D.linear_cross_entropy(x, p, t)[0].requires_grad


def test_captured_and_replayed_on_another_stream():
    torch, D = _d()
    sets = [problem(torch, 100, 500, 64), problem(torch, 33, 70, 65)]
    g = torch.Generator(device="cuda").manual_seed(6)

    def all_of():
        out = []
        for x, w, t, b in sets:
            loss, lse = D.linear_cross_entropy(x, w, t, b)
            out += [loss, lse, *D.linear_cross_entropy_backward(torch.ones_like(loss), x, w, t, lse, b)]
        return out
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_of()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = all_of()
    for x, w, t, b in sets:
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        t.copy_(torch.randint(-5, w.shape[0], t.shape, generator=g, device="cuda"))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, all_of()))


def test_refusals():
    torch, D = _d()
    x, w, t, b = problem(torch, 20, 30, 16)
    lse = g = torch.zeros(20, device="cuda")
    f, r = D.linear_cross_entropy, D.linear_cross_entropy_backward
    bad = [lambda: f(x.float(), w.float(), t), lambda: f(x, w[:, :15], t), lambda: f(x, w.half(), t), lambda: f(x, w, t[:19]), lambda: f(x, w, t.float()), lambda: f(x, w, t.cpu()),
           lambda: f(x, w, t, b[:29]), lambda: f(x, w, t, b.float()), lambda: f(x.t(), w, t), lambda: f(x[None], w, t), lambda: f(x, w[:0], t), lambda: f(x[:, :0], w[:, :0], t),
           lambda: f(x, w.cpu(), t), lambda: f(x, w, t[:, None]), lambda: r(g[:19], x, w, t, lse), lambda: r(g.double(), x, w, t, lse), lambda: r(g, x, w, t, lse[:19]), lambda: r(g, x, w, t, lse.bfloat16()),
           lambda: r(g, x, w, t, lse, out=(x[:19], None, None)), lambda: r(g, x, w, t, lse, out=(None, w.float(), None)), lambda: r(g, x, w, t, lse, out=(None, None, b[:29])),
           lambda: r(g, x, w, t, lse, out=(x[:1].expand(20, 16), None, None)), lambda: r(g, x, w, t, None), lambda: r(g, x, w, t.to(torch.uint8), lse)]
    for call in bad:
        with pytest.raises(D.DmxError):
            call()
    torch.cuda.synchronize()


# few words or few rows: products of few tiles over a long k, whose ranges are added by a launch of their own
@pytest.mark.parametrize("N,V,n", [(1, 30522, 264), (5, 20011, 72), (64, 9000, 1024), (130, 30000, 136), (16000, 10, 64), (9999, 300, 40), (5000, 65, 300), (2048, 2000, 24), (2049, 2000, 24)])
def test_few_tiles_over_a_long_extent(N, V, n):
    torch, D = _d()
    x, w, t, b = problem(torch, N, V, n)
    g = torch.Generator(device="cuda").manual_seed(7)
    a = compare(torch, D, x, w, t, b, dloss=torch.rand(N, generator=g, device="cuda") / N)
    wide = (torch.zeros(N, n + 3, device="cuda", dtype=torch.bfloat16)[:, :n], torch.zeros(V, n + 3, device="cuda", dtype=torch.bfloat16)[:, 3:], None)
    g = torch.Generator(device="cuda").manual_seed(7)
    again = D.linear_cross_entropy_backward(torch.rand(N, generator=g, device="cuda") / N, x, w, t, a[1], b, need=(True, True, False), out=wide)
    assert torch.equal(again[0], a[2]) and torch.equal(again[1], a[3])
