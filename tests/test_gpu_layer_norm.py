"""Layer norm and its gradient against the definition in 64 bits.

Tolerances, with u = 2^-24 and h = half a step of the output's type: every value is rounded once to its type, and before that it
carries the fp32 errors of at most 64 operations in a row (32 values a thread, trees of at most 8 levels, a few products), each
relative to the magnitudes that enter it. Sums over rows add one more operation for each row a thread takes."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def close(torch, got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %.3g over its bound" % (what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol).nan_to_num(1e9).max()))


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def check(torch, D, x, w, b, dy, add=None, eps=1e-5):
    n = x.shape[-1]
    M = x.numel() // n
    X, W = x.double(), torch.ones(n, dtype=torch.float64, device="cuda") if w is None else w.double()
    Bv = torch.zeros(n, dtype=torch.float64, device="cuda") if b is None else b.double()
    mean = X.mean(-1)
    d = X - mean[..., None]
    rstd = 1 / torch.sqrt(d.square().mean(-1) + eps)
    xh = d * rstd[..., None]
    y, m, r = D.layer_norm(x, w, b, eps)
    assert y.dtype == x.dtype and y.shape == x.shape and m.shape == r.shape == x.shape[:-1]
    h = half_step(torch, x.dtype)
    want = xh * W + Bv
    close(torch, m, mean, 2 * U * mean.abs() + 64 * U * d.abs().mean(-1) + 1e-12 * X.abs().mean(-1) + 1e-40, "mean")
    close(torch, r, rstd, 64 * U * rstd, "rstd")
    close(torch, y, want, h * want.abs() + 64 * U * ((xh * W).abs() + W.abs() + Bv.abs()), "y")
    # backward, from the statistics as they are stored
    G, R = dy.double() * W, r.double()[..., None]
    hh = (X - m.double()[..., None]) * R
    c1, c2 = G.mean(-1, keepdim=True), (G * hh).mean(-1, keepdim=True)
    want = R * (G - c1 - hh * c2) + (0 if add is None else add.double())
    dx, dw, db = D.layer_norm_backward(dy, x, m, r, w, add=add)
    size = R * (G.abs() + G.abs().mean(-1, keepdim=True) + hh.abs() * (G * hh).abs().mean(-1, keepdim=True)) + (0 if add is None else add.double().abs())
    close(torch, dx, want, h * want.abs() + 64 * U * size, "dx")
    rows = 64 + M / 250
    T = (dy.double() * hh).reshape(M, n)
    close(torch, dw, T.sum(0), rows * U * T.abs().sum(0) + 1e-40, "dweight")
    close(torch, db, dy.double().reshape(M, n).sum(0), rows * U * dy.double().abs().reshape(M, n).sum(0) + 1e-40, "dbias")
    return y, m, r, dx, dw, db


def randn(torch, g, *shape, dtype="bfloat16"):
    return torch.randn(*shape, generator=g, device="cuda").to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("D_", [1, 2, 7, 8, 9, 63, 64, 65, 72, 77, 255, 256, 264, 257, 511, 512, 520, 771, 1000, 1023, 1024, 1025, 1032, 1500, 2048, 4095, 4096, 4104, 8191,
                                8192, 8193, 8200, 16384, 20001, 32768, 40000, 65535, 65536])
def test_widths(D_, dtype):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(D_)
    for M in (1, 2, 5, 37) if D_ > 1024 else (1, 3, 4, 33, 130):
        x = randn(torch, g, M, D_, dtype=dtype) + randn(torch, g, M, 1, dtype=dtype)
        check(torch, D, x, 1 + 0.3 * randn(torch, g, D_, dtype="float32"), randn(torch, g, D_, dtype="float32"), randn(torch, g, M, D_, dtype=dtype),
              add=randn(torch, g, M, D_, dtype=dtype) if M % 2 else None)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,D_", [(20000, 64), (20001, 40), (9001, 256), (7003, 510), (12007, 1024), (5003, 771), (3001, 4096), (1501, 2056), (333, 16384), (333, 9999)])
def test_teams_take_many_rows(M, D_, dtype):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(M)
    a = [randn(torch, g, M, D_, dtype=dtype) for _ in range(3)]
    w, b = randn(torch, g, D_, dtype="float32"), randn(torch, g, D_, dtype="float32")
    first = check(torch, D, a[0], w, b, a[1], a[2])
    again = (*D.layer_norm(a[0], w, b), *D.layer_norm_backward(a[1], a[0], first[1], first[2], w, add=a[2]))
    assert all(torch.equal(s, t) for s, t in zip(first, again))


@pytest.mark.parametrize("D_", [48, 1000, 1024, 4096, 16384])
@pytest.mark.parametrize("slack,start", [(8, 0), (3, 0), (8, 1), (0, 1)])
def test_strides_and_starts(D_, slack, start):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(D_ + slack)
    for dtype in ("float32", "bfloat16"):
        cut = lambda: torch.randn(9 * (D_ + slack) + 8, generator=g, device="cuda").to(getattr(torch, dtype))[start:].as_strided((9, D_), (D_ + slack, 1))  # noqa: E731
        x, dy, add = cut(), cut(), cut()
        wide = torch.randn(D_ + 1, generator=g, device="cuda")
        for w in (wide[:D_], wide[1:], None):
            y, m, r, dx, dw, db = check(torch, D, x, w, w, dy, add)
        # into a given tensor; over an input
        out = cut()
        assert D.layer_norm(x, w, w, out=out)[0] is out and torch.equal(out, y)
        for over in range(3):
            a = [dy.clone(), x.clone(), add.clone()]
            want = D.layer_norm_backward(a[0], a[1], m, r, w, add=a[2])[0]      # (of these dense copies: another layout may add in another order)
            assert torch.equal(D.layer_norm_backward(a[0], a[1], m, r, w, add=a[2], out=a[over])[0], want)
        t = x.clone()
        want = D.layer_norm(t, w, w)[0]
        D.layer_norm(t, w, w, out=t)
        assert torch.equal(t, want)
        a = [dy, x, add]
        D.layer_norm_backward(dy, x, m, r, w, add=add, out=add)                 # and in place with the strides there are
        assert torch.equal(add, dx)


def test_shapes_of_several_dimensions_and_repeated_rows():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = randn(torch, g, 3, 5, 7, 40), randn(torch, g, 3, 5, 7, 40)
    w = randn(torch, g, 40, dtype="float32")
    y, m, r, dx, dw, db = check(torch, D, x, w, w, dy)
    flat = D.layer_norm(x.view(-1, 40), w, w)
    assert torch.equal(flat[0].view_as(y), y) and m.shape == (3, 5, 7)
    check(torch, D, x[:, :, 2], w, None, dy[:, :, 3])              # every seventh row
    check(torch, D, x[0, 0, 0], w, None, dy[0, 0, 0])              # one row without a leading dimension
    one = randn(torch, g, 1, 40)
    check(torch, D, one.expand(50, 40), w, w, dy.view(-1, 40)[:50])
    check(torch, D, x.view(-1, 40)[:50], w, w, one.expand(50, 40), add=one.expand(50, 40))
    with pytest.raises(D.DmxError):
        D.layer_norm(x[:, :3], w, w)                               # rows at no one stride
    with pytest.raises(D.DmxError):
        D.layer_norm(x.transpose(2, 3), None, None)
    with pytest.raises(D.DmxError):
        D.layer_norm(one.expand(50, 40), w, w, out=one.expand(50, 40))


def test_nothing_to_do():
    torch, D = _d()
    for shape in ((0, 24), (4, 0, 24)):
        x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        y, m, r = D.layer_norm(x)
        dx, dw, db = D.layer_norm_backward(x, x, m, r)
        assert y.shape == dx.shape == x.shape and m.shape == x.shape[:-1] and not dw.any() and not db.any() and dw.shape == (24,)
    with pytest.raises(D.DmxError):
        D.layer_norm(torch.empty(4, 0, device="cuda"))


@pytest.mark.parametrize("D_", [48, 1024, 2900, 20000])
def test_means_far_from_zero(D_):
    """fp32 rows whose mean is up to a million deviations away: rstd and y keep their bounds."""
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(D_)
    for far in (1e2, 1e4, 1e6):
        x = torch.randn(17, D_, generator=g, device="cuda") + far
        check(torch, D, x, None, None, torch.randn(17, D_, generator=g, device="cuda"), eps=0.0)
    x = torch.full((3, D_), 0.1, device="cuda")                    # no spread at all
    y, m, r = D.layer_norm(x, None, None, eps=1e-5)
    close(torch, r, torch.full((3,), 1e-5 ** -0.5, device="cuda", dtype=torch.float64), 64 * U * 1e-5 ** -0.5, "rstd")
    assert float(y.abs().max()) <= 64 * U and torch.equal(m, x[:, 0])


@pytest.mark.parametrize("D_", [40, 1024, 2000, 9000])
def test_rows_that_are_not_finite_stay_alone(D_):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = torch.randn(20, D_, generator=g, device="cuda"), torch.randn(20, D_, generator=g, device="cuda")
    want = D.layer_norm(x)
    back = D.layer_norm_backward(dy, x, want[1], want[2])
    x2 = x.clone()
    x2[3, 5], x2[7, D_ - 1], x2[19, 0] = float("nan"), float("inf"), -float("inf")
    got = D.layer_norm(x2)
    hit = torch.tensor([3, 7, 19], device="cuda")
    keep = torch.tensor([i for i in range(20) if i not in (3, 7, 19)], device="cuda")
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])
    assert got[0][hit].isnan().all() and got[2][hit].isnan().all()
    dx = D.layer_norm_backward(dy, x2, got[1], got[2])[0]
    assert torch.equal(dx[keep], back[0][keep]) and dx[hit].isnan().all()


def test_gradient_against_differences():
    """The slope of sum(dy y) along random directions, by central differences of the definition in 64 bits."""
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(9)
    for D_ in (5, 100, 1024, 1100):
        x, w, b, dy = (torch.randn(s, generator=g, device="cuda") for s in ((6, D_), (D_,), (D_,), (6, D_)))
        y, m, r = D.layer_norm(x, w, b)
        grads = D.layer_norm_backward(dy, x, m, r, w)
        at = [t.double() for t in (x, w, b)]

        def value(t):
            d = t[0] - t[0].mean(1, keepdim=True)
            return float((dy.double() * (d / torch.sqrt(d.square().mean(1, keepdim=True) + 1e-5) * t[1] + t[2])).sum())
        for i in range(3):
            v = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
            e = 1e-5
            up, down = value([t + e * v if j == i else t for j, t in enumerate(at)]), value([t - e * v if j == i else t for j, t in enumerate(at)])
            slope = float((grads[i].double() * v).sum())
            # differences: e^2 of the third derivative and 1e-16 / e of the value; the gradient: fp32 errors of its entries
            assert abs((up - down) / (2 * e) - slope) <= 1e-6 * float(dy.abs().sum()) * 3


def test_recorded_for_differentiation():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(2)
    for dtype in ("float32", "bfloat16"):
        x, dy = randn(torch, g, 4, 9, 24, dtype=dtype), randn(torch, g, 4, 9, 24, dtype=dtype)
        w, b = randn(torch, g, 24, dtype="float32"), randn(torch, g, 24, dtype="float32")
        y0, m, r = D.layer_norm(x, w, b)
        want = D.layer_norm_backward(dy, x, m, r, w)
        leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
        y, m1, r1 = D.layer_norm(*leaves)
        assert torch.equal(y, y0) and y.requires_grad and not m1.requires_grad and not r1.requires_grad
        y.backward(dy)
        assert all(torch.equal(t.grad, v) for t, v in zip(leaves, want))
        p = torch.nn.Parameter(w.clone())
        D.layer_norm(x, p)[0].sum().backward()                     # an expanded gradient; only the weight
        assert torch.equal(p.grad, D.layer_norm_backward(torch.ones_like(x), x, m, r, w)[1])
        with torch.no_grad():
            assert not D.layer_norm(x, p)[0].requires_grad
        out = torch.empty_like(x)
        assert not D.layer_norm(x, p, out=out)[0].requires_grad
        t = x.clone().requires_grad_(True)
        s = t * 1.0
        y = D.layer_norm(s, p)[0]
        D.layer_norm(x, out=s.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


def test_captured_and_replayed_on_another_stream():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(3)
    shapes = [(50, 64), (700, 1024), (30, 5000), (9, 20000)]
    xs = [randn(torch, g, *s) for s in shapes]
    dys = [randn(torch, g, *s) for s in shapes]

    def all_of():
        out = []
        for x, dy in zip(xs, dys):
            y, m, r = D.layer_norm(x)
            out += [y, m, r, *D.layer_norm_backward(dy, x, m, r)]
        return out
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_of()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = all_of()
    for t in xs + dys:
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, all_of()))


def test_rows_beyond_32_bit_offsets():
    torch, D = _d()
    M, n = 70000, 32768                                             # 2.3e9 elements, 4.6 GB each
    x = torch.empty(M, n, device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(8)
    x.normal_(generator=g)
    y, m, r = D.layer_norm(x)
    last = slice(M - 4, M)
    want = D.layer_norm(x[last].contiguous())
    assert all(torch.equal(a[last], b) for a, b in zip((y, m, r), want))
    dx = D.layer_norm_backward(y, x, m, r, out=y)[0]
    assert torch.equal(dx[last], D.layer_norm_backward(want[0], x[last], m[last], r[last])[0])


def test_refusals():
    torch, D = _d()
    x, w = torch.zeros(4, 24, device="cuda"), torch.zeros(24, device="cuda")
    m = torch.zeros(4, device="cuda")
    bad = [lambda: D.layer_norm(x.double()), lambda: D.layer_norm(x.half()), lambda: D.layer_norm(x, w[:23]), lambda: D.layer_norm(x, w.bfloat16()), lambda: D.layer_norm(x, w.cpu()),
           lambda: D.layer_norm(x, eps=-1.0), lambda: D.layer_norm(x, eps="a"), lambda: D.layer_norm(x, eps=float("nan")), lambda: D.layer_norm(x, out=x.bfloat16()),
           lambda: D.layer_norm(x, out=x[:3]), lambda: D.layer_norm(x, out=x[:1].expand(4, 24)), lambda: D.layer_norm(torch.zeros(2, 65537, device="cuda")),
           lambda: D.layer_norm(x.cpu()), lambda: D.layer_norm(torch.zeros((), device="cuda")), lambda: D.layer_norm(x, torch.zeros(48, device="cuda")[::2]),
           lambda: D.layer_norm_backward(x[:3], x, m, m), lambda: D.layer_norm_backward(x.bfloat16(), x, m, m), lambda: D.layer_norm_backward(x, x, m[:3], m),
           lambda: D.layer_norm_backward(x, x, m, m.double()), lambda: D.layer_norm_backward(x, x, m, m, add=x[0]), lambda: D.layer_norm_backward(x, x, m, m, w[1:]),
           lambda: D.layer_norm_backward(x, x, m, m, out=x[:, :23])]
    for call in bad:
        with pytest.raises(D.DmxError):
            call()
    torch.cuda.synchronize()
