"""The training operators at the far end of their range: the matrix product at its largest extents (a sum so long that waits inside
the kernel last for milliseconds among them), and places in memory beyond 32-bit counts. Checks and tolerances of the former are those
of ordinary sizes; the latter are the same numbers as from small pieces, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

MOST = 4194240


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


@pytest.fixture(autouse=True)
def leave_no_memory():
    yield
    import torch
    torch.cuda.empty_cache()


@pytest.mark.parametrize("shape", [(MOST, 8, 7), (MOST, 16, 8), (8, MOST, 7), (5, 16, MOST), (64, 64, MOST), (130, 72, MOST - 1), (260, 264, MOST // 2), (MOST, 1, 1)])
def test_largest_extents(shape):
    from tests.test_gpu_linear import run
    run(*shape, act="gelu" if shape[0] < 100 else "none")


def test_product_with_rows_far_apart():
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(1)
    far, K, N = 2 ** 30 + 8, 72, 40
    room = torch.empty(3 * far, dtype=torch.bfloat16, device="cuda")          # 6.4 GB, only its rows' places written
    for odd in (0, 1):
        x, dy, y = (room.as_strided((3, n), (far, 1), odd + at) for n, at in ((K, 0), (N, 512), (N, 1024)))
        x.copy_(torch.randn(3, K, generator=g, device="cuda"))
        dy.copy_(torch.randn(3, N, generator=g, device="cuda"))
        w = torch.randn(N, K, generator=g, device="cuda").bfloat16()
        want, z = D.linear(x.contiguous(), w, act="silu", save=True)
        D.linear(x, w, act="silu", out=y)
        assert torch.equal(y, want)
        back = D.linear_backward(dy.contiguous(), x.contiguous(), w, z, act="silu")
        dx = room.as_strided((3, K), (far, 1), odd + 2048)
        got = D.linear_backward(dy, x, w, z, act="silu", out=(dx, None, None))
        assert all(torch.equal(a, b) for a, b in zip(got, back))
    assert D.linear_status() == 0


@pytest.mark.parametrize("C", [64, 63])
def test_group_norm_beyond_32_bits(C):
    torch, D = _d()
    N, L = 3, 2 ** 31 // (2 * 64)                                            # the third image starts at 2^31 elements and more
    x = torch.empty(N, L + 8, C, dtype=torch.bfloat16, device="cuda").normal_()[:, :L]
    w, b = torch.rand(C, device="cuda"), torch.rand(C, device="cuda")
    groups = C // 21 if C == 63 else 8
    y, mean, rstd = D.group_norm(x, groups, w, b, act="silu")
    dx, dw, db = D.group_norm_backward(y, x, mean, rstd, groups, w, b, act="silu")
    dws = []
    for i in range(N):
        p = D.group_norm(x[i:i + 1], groups, w, b, act="silu")
        assert torch.equal(p[0], y[i:i + 1]) and torch.equal(p[1], mean[i:i + 1]) and torch.equal(p[2], rstd[i:i + 1])
        q = D.group_norm_backward(p[0], x[i:i + 1], p[1], p[2], groups, w, b, act="silu")
        assert torch.equal(q[0], dx[i:i + 1])
        dws.append(q[1:])
        del p, q
    for k, t in enumerate((dw, db)):                                          # three images' sums, added in some order: three roundings of the largest
        s = torch.stack([v[k].double() for v in dws])
        assert torch.all((t.double() - s.sum(0)).abs() <= 4 * 2.0 ** -24 * s.abs().sum(0) + 1e-30)


@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer_beyond_32_bits(bits):
    torch, D = _d()
    n, odd = 2 ** 31 + 256 * 5 + 77, 1001
    p, g = torch.empty(n, device="cuda").normal_(), torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_()
    q, h = torch.empty(odd, device="cuda").normal_(), torch.empty(odd, dtype=torch.bfloat16, device="cuda").normal_()
    tail = 2 ** 31 - 256 * 3                                                   # a block's start: the pieces keep their blocks
    pieces = [p[:5000].clone(), p[tail:].clone(), q.clone()]
    opt, ref = D.AdamW([p, q], [g, h], state_bits=bits), D.AdamW(pieces, [g[:5000].clone(), g[tail:].clone(), h.clone()], state_bits=bits)
    st, sr = opt.new_state(), ref.new_state()
    norm = opt.grad_norm(1.0)
    total = sum(float(t.double().square().sum()) for t in (*g.split(2 ** 28), h)) ** 0.5
    assert abs(float(norm[0]) - total) <= 6 * 2.0 ** -24 * total
    for t in (1, 2):
        opt.step(*st, t=t, lr=1e-2)
        ref.step(*sr, t=t, lr=1e-2)
    whole = 5000 // 256 * 256                                                  # (the first piece's last block is cut short)
    assert torch.equal(p[:whole], pieces[0][:whole]) and torch.equal(p[tail:], pieces[1]) and torch.equal(q, pieces[2])
    for a, b in ((st[0], sr[0]), (st[1], sr[1])):
        assert torch.equal(opt.state_view(a, 0)[tail:], ref.state_view(b, 1)) and torch.equal(opt.state_view(a, 1), ref.state_view(b, 2))
