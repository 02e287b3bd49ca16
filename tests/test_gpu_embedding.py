"""The embedding lookup and its gradient against the definition in 64 bits.

The lookup is one fp32 product and one rounding: compared bit for bit. A row of the gradient is a sum of c terms in fp32 (at most c + 2
roundings of partial sums, each at most the sum of the terms' magnitudes), a product and one rounding to the type."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def definition(torch, dy, ids, V, scale, old=None):
    """(sums in 64 bits, their bounds without the rounding of the result)"""
    ids, dy = ids.reshape(-1).long(), dy.double().reshape(ids.numel(), -1)
    keep = (ids >= 0) & (ids < V)
    at = ids[keep]
    total = torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, dy[keep])
    size = torch.zeros_like(total).index_add_(0, at, dy[keep].abs())
    count = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones(len(at), dtype=torch.float64, device="cuda"))
    total, size = total * scale, (count[:, None] + 3) * U * size * abs(scale)
    if old is not None:
        total, size = total + old.double(), size + 2 * U * old.double().abs()
    return total, size, count


def check(torch, D, dy, ids, V, scale=1.0, out=None, accumulate=False):
    old = out.clone() if accumulate else None
    want, size, count = definition(torch, dy, ids, V, scale, old)
    got = D.embedding_backward(dy, ids, V, scale, out=out, accumulate=accumulate)
    assert got.shape == (V, dy.shape[-1]) and got.dtype == (dy.dtype if out is None else out.dtype)
    tol = size + torch.finfo(got.dtype).eps / 2 * want.abs()
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), "%d of %d off" % (int(bad.sum()), bad.numel())
    untouched = count == 0
    assert torch.equal(got[untouched], old[untouched] if accumulate else torch.zeros_like(got[untouched]))
    return got


def words(torch, g, n, V, dtype="int64"):
    k = (torch.rand(n, generator=g, device="cuda").double() * torch.log(torch.tensor(V + 1.0, dtype=torch.float64))).exp().long() - 1
    return torch.randperm(V, generator=g, device="cuda")[k.clamp(0, V - 1)].to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("scale", [1.0, 22.627417])
def test_lookup(dtype, scale):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(1)
    for V, n in ((1, 8), (7, 1), (100, 33), (1000, 771), (30522, 1024), (65537, 130), (50, 5000)):
        table = torch.randn(V, n, generator=g, device="cuda").to(getattr(torch, dtype))
        for shape, it in (((1,), "int64"), ((5, 7), "int32"), ((3, 2, 11), "int64"), ((513,), "int32"), ((), "int64")):
            ids = torch.randint(-2, V + 2, shape, generator=g, device="cuda", dtype=getattr(torch, it))
            ok = (ids >= 0) & (ids < V)
            want = ((table[ids.long().clamp(0, V - 1)].float() * scale).to(table.dtype)) * ok[..., None]
            got = D.embedding(ids, table, scale)
            assert got.dtype == table.dtype and got.shape == (*shape, n) and torch.equal(got, want)
    # far ids, both ends of the integers
    ids = torch.tensor([2 ** 62, -2 ** 63, 3, 2 ** 32 + 1, -1], device="cuda")
    got = D.embedding(ids, table, 1.0)
    assert torch.equal(got[2], table[3]) and not got[[0, 1, 3, 4]].any()


def test_lookup_strides():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(2)
    for dtype in (torch.float32, torch.bfloat16):
        for n in (24, 25):
            for slack, start in ((8, 0), (3, 0), (0, 1)):
                base = torch.randn(60 * (n + slack) + 8, generator=g, device="cuda").to(dtype)[start:]
                table = base.as_strided((60, n), (n + slack, 1))
                tokens = torch.randint(0, 60, (6, 9), generator=g, device="cuda")
                ids = tokens[:, :-1]                                 # not dense, as inputs that are their own shifted targets
                out = torch.full((6, 8, n + 5), 7.0, device="cuda", dtype=dtype)
                view = out[..., :n]
                assert D.embedding(ids, table, out=view) is view
                assert torch.equal(view, table[ids]) and (out[..., n:] == 7.0).all()
                assert torch.equal(D.embedding(ids.t(), table), table[ids.t()])
    one = torch.randn(1, 32, generator=g, device="cuda")
    assert torch.equal(D.embedding(torch.arange(9, device="cuda"), one.expand(9, 32)), one.expand(9, 32))


@pytest.mark.parametrize("dtype,out", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("V,n", [(1, 8), (2, 1), (10, 64), (255, 40), (256, 33), (257, 256), (1000, 771), (30522, 1024), (65535, 24), (65536, 16), (70001, 8), (300000, 8)])
def test_gradient(V, n, dtype, out):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(V + n)
    for N in (1, 2, 31, 32, 33, 100, 1000, 9001):
        ids = words(torch, g, N, V, "int32" if N % 2 else "int64")
        if N % 3 == 0:
            ids = torch.where(torch.rand(N, generator=g, device="cuda") < 0.3, torch.full_like(ids, -1 if N % 2 else V), ids)
        dy = torch.randn(N, n, generator=g, device="cuda").to(getattr(torch, dtype))
        check(torch, D, dy, ids, V, scale=1.0 if N % 2 else 5.5, out=torch.full((V, n), float("nan"), device="cuda", dtype=getattr(torch, out)))
        check(torch, D, dy, ids, V, out=torch.randn(V, n, generator=g, device="cuda").to(getattr(torch, out)), accumulate=True)


@pytest.mark.parametrize("N", [20000, 65536, 262144 + 77])
@pytest.mark.parametrize("kind", ["one", "two", "words", "none", "each", "runs"])
def test_how_often_a_token_comes(kind, N):
    """One token for all, halves, Zipf's law, none at all, each once, runs that end at chunk borders."""
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(N)
    V, n = 300001, 40
    ids = {"one": lambda: torch.full((N,), 77777, device="cuda"), "two": lambda: torch.arange(N, device="cuda") % 2 * 300000,
           "words": lambda: words(torch, g, N, V), "none": lambda: torch.full((N,), V, device="cuda"),
           "each": lambda: torch.randperm(V, generator=g, device="cuda")[:N], "runs": lambda: torch.arange(N, device="cuda") // 32 * 7}[kind]()
    dy = torch.randn(N, n, generator=g, device="cuda")
    a = check(torch, D, dy, ids, V, out=torch.empty(V, n, device="cuda"))
    assert torch.equal(a, D.embedding_backward(dy, ids, V))           # bitwise reproducible
    wide = torch.randn(N, 520, generator=g, device="cuda").bfloat16() if N < 70000 else dy.bfloat16()
    check(torch, D, wide, ids % 1009, 1009)


def test_gradient_strides():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(4)
    for dtype in (torch.float32, torch.bfloat16):
        for n in (24, 25):
            for slack, start in ((8, 0), (3, 0), (8, 1), (0, 1)):
                cut = lambda rows: torch.randn(rows * (n + slack) + 8, generator=g, device="cuda").to(dtype)[start:].as_strided((rows, n), (n + slack, 1))  # noqa: E731
                tokens = torch.randint(0, 60, (10, 9), generator=g, device="cuda")
                dy = cut(80)
                base = torch.full((60 * (n + slack) + 8,), 7.0, device="cuda", dtype=dtype)
                out = base[start:].as_strided((60, n), (n + slack, 1))
                check(torch, D, dy, tokens[:, 1:].reshape(-1), 60, out=out)
                if slack:
                    gaps = base[start:start + 60 * (n + slack)].view(60, n + slack)[:, n:]
                    assert (gaps == 7.0).all() and (base[:start] == 7.0).all()
                check(torch, D, torch.randn(10, 8, n, generator=g, device="cuda").to(dtype), tokens[:, 1:], 60, out=cut(60), accumulate=True)
        one = torch.randn(1, 32, generator=g, device="cuda").to(dtype)
        check(torch, D, one.expand(500, 32), torch.randint(0, 9, (500,), generator=g, device="cuda"), 9)


def test_nothing_to_do():
    torch, D = _d()
    t, none = torch.randn(5, 8, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    assert D.embedding(none, t).shape == (0, 8) and D.embedding(none.view(3, 0), t).shape == (3, 0, 8)
    assert not D.embedding(torch.zeros(4, dtype=torch.int64, device="cuda"), t[:0]).any()
    assert D.embedding(torch.zeros(4, dtype=torch.int64, device="cuda"), t[:, :0]).shape == (4, 0)
    got = D.embedding_backward(torch.empty(0, 8, device="cuda"), none, 5, out=torch.full((5, 8), 3.0, device="cuda"))
    assert not got.any()
    got = D.embedding_backward(torch.empty(0, 8, device="cuda"), none, 5, out=torch.full((5, 8), 3.0, device="cuda"), accumulate=True)
    assert (got == 3.0).all()
    assert D.embedding_backward(torch.ones(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), 0).shape == (0, 8)


def test_values_that_are_not_finite_stay_in_their_rows():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(6)
    ids = torch.randint(0, 50, (3000,), generator=g, device="cuda")
    dy = torch.randn(3000, 24, generator=g, device="cuda")
    want = D.embedding_backward(dy, ids, 50)
    ids2, dy2 = torch.cat([ids, torch.tensor([-1, 99], device="cuda")]), torch.cat([dy, torch.full((2, 24), float("nan"), device="cuda")])
    check(torch, D, dy2, ids2, 50)
    dy3 = dy.clone()
    dy3[ids == 7] = float("inf")
    got = D.embedding_backward(dy3, ids, 50)
    assert torch.equal(got[torch.arange(50, device="cuda") != 7], want[torch.arange(50, device="cuda") != 7]) and got[7].isinf().all()


def test_recorded_for_differentiation():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(7)
    for dtype in (torch.float32, torch.bfloat16):
        ids = torch.randint(-1, 40, (6, 9), generator=g, device="cuda")
        table, dy = torch.randn(40, 24, generator=g, device="cuda").to(dtype), torch.randn(6, 9, 24, generator=g, device="cuda").to(dtype)
        p = torch.nn.Parameter(table.clone())
        y = D.embedding(ids, p, 3.0)
        assert y.requires_grad and torch.equal(y, D.embedding(ids, table, 3.0))
        y.backward(dy)
        assert torch.equal(p.grad, D.embedding_backward(dy, ids, 40, 3.0))
        p.grad = None
        D.embedding(ids, p).sum().backward()
        assert torch.equal(p.grad, D.embedding_backward(torch.ones_like(dy), ids, 40))
        with torch.no_grad():
            assert not D.embedding(ids, p).requires_grad
        assert not D.embedding(ids, p, out=torch.empty_like(dy)).requires_grad


def test_captured_and_replayed_on_another_stream():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(8)
    ids = words(torch, g, 3001, 5003)
    table, dy = torch.randn(5003, 72, generator=g, device="cuda"), torch.randn(3001, 72, generator=g, device="cuda")
    grad = torch.randn(5003, 72, generator=g, device="cuda")

    def both(to):
        return D.embedding(ids, table, 2.0), D.embedding_backward(dy, ids, 5003), D.embedding_backward(dy, ids, 5003, out=to, accumulate=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(grad.clone())
    torch.cuda.current_stream().wait_stream(side)
    graph, to = torch.cuda.CUDAGraph(), grad.clone()
    with torch.cuda.graph(graph):
        kept = both(to)
    ids.copy_(words(torch, g, 3001, 5003))
    dy.normal_(generator=g)
    graph.replay()
    to.copy_(grad)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, both(grad)))


def test_offsets_beyond_32_bits():
    torch, D = _d()
    V, n = 140000, 16384                                              # 2.3e9 elements, 4.6 GB
    table = torch.empty(V, n, device="cuda", dtype=torch.bfloat16).normal_()
    ids = torch.tensor([V - 1, 0, V // 2, 131073, V - 1], device="cuda")
    y = D.embedding(ids, table)
    assert torch.equal(y, table[ids])
    got = D.embedding_backward(y, ids, V, out=table)
    assert torch.equal(got[V - 1], (y[0].float() * 2).bfloat16()) and torch.equal(got[131073], y[3]) and not got[131074:V - 1].any() and not got[1:V // 2].any()
    ids = torch.arange(V, device="cuda") % 3                          # long gradients: places beyond 32-bit offsets
    table.normal_()
    got = D.embedding_backward(table, ids, 3)
    want = torch.stack([sum(part.double().sum(0) for part in table[i::3].split(5000)) for i in range(3)])
    size = torch.stack([sum(part.double().abs().sum(0) for part in table[i::3].split(5000)) for i in range(3)])
    assert ((got.double() - want).abs() <= 2 ** -8 * want.abs() + (V / 3 + 3) * U * size).all()


def test_refusals():
    torch, D = _d()
    t, i = torch.zeros(5, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    dy = torch.zeros(3, 8, device="cuda")
    bad = [lambda: D.embedding(i, t.double()), lambda: D.embedding(i.float(), t), lambda: D.embedding(i.short(), t), lambda: D.embedding(i.cpu(), t), lambda: D.embedding(i, t.cpu()),
           lambda: D.embedding(i, t[0]), lambda: D.embedding(i, t.t()), lambda: D.embedding(i, t, "a"), lambda: D.embedding(i, t, out=dy[:2]), lambda: D.embedding(i, t, out=dy.bfloat16()),
           lambda: D.embedding(i, t, out=dy[:1].expand(3, 8)), lambda: D.embedding(i, t, out=torch.zeros(3, 9, device="cuda")), lambda: D.embedding(i, torch.zeros(2, 65537, device="cuda")),
           lambda: D.embedding_backward(dy[:2], i, 5), lambda: D.embedding_backward(dy, i, -1), lambda: D.embedding_backward(dy, i, 5, out=t[:4]), lambda: D.embedding_backward(dy, i, 2 ** 31),
           lambda: D.embedding_backward(dy, i, 5, accumulate=True), lambda: D.embedding_backward(dy.half(), i, 5), lambda: D.embedding_backward(dy, i, 5, out=t[:1].expand(5, 8)),
           lambda: D.embedding_backward(dy, i.cpu(), 5), lambda: D.embedding_backward(dy, i.view(3, 1), 5), lambda: D.embedding_backward(dy, i, "5")]
    for call in bad:
        with pytest.raises(D.DmxError):
            call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("N", [1, 1023, 1024, 1025, 4095, 4096, 4097, 131072, 1048576, 1048577])
def test_borders_between_the_sorts(N):
    """One CTA's tokens and one more; a warp's rounds of 32 in all of 128 CTAs, and what no longer stays in registers."""
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(N)
    for V in (200, 256, 65536, 70000):
        ids = words(torch, g, N, V)
        ids[torch.rand(N, generator=g, device="cuda") < 0.1] = -5
        dy = torch.randn(N, 8, generator=g, device="cuda")
        a = check(torch, D, dy, ids, V)
        assert torch.equal(a, D.embedding_backward(dy, ids, V))


def test_a_table_of_more_than_2_to_24_rows():
    """Four passes of the sort, in one CTA and in several."""
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(1)
    V = 20_000_003
    for N in (3000, 9000):
        ids = torch.randint(0, V, (N,), generator=g, device="cuda")
        ids[::3] = ids[0]
        ids[1::7] = V - 1
        dy = torch.randn(N, 4, generator=g, device="cuda")
        got = D.embedding_backward(dy, ids, V)
        rows, back = ids.unique(return_inverse=True)
        want, size, _ = definition(torch, dy, back, len(rows), 1.0)
        assert ((got[rows].double() - want).abs() <= size + U * want.abs()).all()
        got[rows] = 0
        assert not got.any()
        assert torch.equal(D.embedding(ids, got), torch.zeros(N, 4, device="cuda"))
