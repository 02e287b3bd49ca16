"""The training operators under torch's differentiation: gradients are those of the explicit backward calls, bit for bit, and are not
lost silently; writes to given tensors are seen by it."""
import pytest

pytestmark = pytest.mark.gpu


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def randn(g, *shape, dtype="bfloat16"):
    import torch
    return torch.randn(*shape, generator=g, device="cuda").to(getattr(torch, dtype))


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("save", [False, True])
def test_linear_is_differentiated(act, save):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(1)
    for M, N, K in ((40, 72, 64), (200, 33, 17), (1, 8, 8)):
        x, w, b, r, dy = randn(g, M, K), randn(g, N, K), randn(g, N), randn(g, M, N), randn(g, M, N)
        y0, z0 = D.linear(x, w, b, act=act, residual=r, save=True)
        want = D.linear_backward(dy, x, w, z0, act=act)
        leaves = [t.clone().requires_grad_(True) for t in (x, w, b, r)]
        y, z = D.linear(*leaves[:3], act=act, residual=leaves[3], save=save)
        assert y.requires_grad and torch.equal(y, y0) and (z is None) == (not save or act == "none")
        assert z is None or (torch.equal(z, z0) and not z.requires_grad)
        y.backward(dy)
        assert all(torch.equal(t.grad, v) for t, v in zip(leaves, (*want, dy)))
        # only some of the inputs; a gradient that is one value for every element
        w2 = torch.nn.Parameter(w.clone())
        D.linear(x, w2, act=act)[0].sum().backward()
        ones = torch.ones_like(dy)
        z1 = D.linear(x, w, act=act, save=True)[1]
        assert torch.equal(w2.grad, D.linear_backward(ones, x, w, z1, act=act)[1])


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_group_norm_is_differentiated(act, dtype):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy, w, b = randn(g, 3, 5, 7, 24, dtype=dtype), randn(g, 3, 5, 7, 24, dtype=dtype), randn(g, 24, dtype="float32"), randn(g, 24, dtype="float32")
    y0, mean, rstd = D.group_norm(x, 4, w, b, act=act)
    want = D.group_norm_backward(dy, x, mean, rstd, 4, w, b, act=act)
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    y, m, r = D.group_norm(leaves[0], 4, *leaves[1:], act=act)
    assert torch.equal(y, y0) and not m.requires_grad and not r.requires_grad
    y.backward(dy)
    assert all(torch.equal(t.grad, v) for t, v in zip(leaves, want))
    w2 = torch.nn.Parameter(w.clone())
    y = D.group_norm(x, 4, w2, act=act)[0]
    y.sum().backward()                      # an expanded gradient
    assert torch.equal(w2.grad, D.group_norm_backward(torch.ones_like(x), x, mean, rstd, 4, w, act=act)[1])
    t = x.clone().requires_grad_(True)
    D.group_norm(t, 4, act=act)[0].transpose(1, 2).contiguous().backward(dy.transpose(1, 2).contiguous())
    assert torch.equal(t.grad, D.group_norm_backward(dy, x, mean, rstd, 4, act=act)[0])


def test_what_is_not_recorded():
    torch, D = _d()
    x, w = torch.ones(4, 8, dtype=torch.bfloat16, device="cuda"), torch.nn.Parameter(torch.ones(16, 8, dtype=torch.bfloat16, device="cuda"))
    v = torch.nn.Parameter(torch.ones(8, device="cuda"))
    with torch.no_grad():
        assert not D.linear(x, w)[0].requires_grad and not D.group_norm(x.view(1, 4, 8), 2, v)[0].requires_grad
    assert not D.linear(x, w.detach())[0].requires_grad
    y, _ = D.linear(x, w, out=(out := torch.empty(4, 16, dtype=torch.bfloat16, device="cuda")))
    assert y is out and not y.requires_grad
    z = torch.empty(1, 4, 8, dtype=torch.bfloat16, device="cuda")
    assert D.group_norm(x.view(1, 4, 8), 2, v, out=z)[0] is z and not z.requires_grad
    with pytest.raises(D.DmxError):
        D.linear(x[:, :7], w)
    with pytest.raises(D.DmxError):
        D.group_norm(x.view(1, 4, 8), 3, v)
    y = D.linear(x.clone().requires_grad_(True), w, act="gelu")[0]
    (gx,) = torch.autograd.grad(y.float().square().sum(), w, create_graph=True)
    with pytest.raises(RuntimeError):
        gx.float().sum().backward()         # first derivatives only


def test_writes_are_seen():
    torch, D = _d()
    x, w = torch.ones(4, 8, dtype=torch.bfloat16, device="cuda"), torch.nn.Parameter(torch.ones(16, 8, dtype=torch.bfloat16, device="cuda"))
    # the optimizer changes a weight between forward and backward: an error, not a wrong gradient
    y = D.linear(x.clone().requires_grad_(True), w)[0]
    opt = D.AdamW([w], [torch.ones_like(w)], copies=None)
    st = opt.new_state()
    opt.step(*st, t=1, lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    n = torch.empty(2, device="cuda")
    was = [t._version for t in (w, st[0], st[1], n)]
    opt.grad_norm(1.0, out=n)
    opt.step(*st, t=2, lr=0.1, grad_scale=n[1:])
    assert all(t._version > v for t, v in zip((w, st[0], st[1], n), was))
    # copies, 8-bit states and their values; a tensor without a gradient is left alone
    p, q, c = torch.ones(300, device="cuda"), torch.ones(30, device="cuda"), torch.zeros(300, dtype=torch.bfloat16, device="cuda")
    opt = D.AdamW([p, q], [torch.ones(300, device="cuda"), None], state_bits=8, copies=[c, None])
    st = opt.new_state()
    om, ov = torch.empty(768, device="cuda"), torch.empty(768, device="cuda")
    seen = (p, c, *st)
    was = [t._version for t in seen]
    opt.step(*st, t=1, lr=0.1)
    opt.moments(*st, om, ov)
    assert all(t._version > v for t, v in zip(seen, was)) and q._version == 0 and om._version == ov._version == 1
    # given outputs
    out, dx, img = torch.empty(4, 16, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 8, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 4, 8, device="cuda")
    D.linear(x, w, out=out)
    D.linear_backward(out, x, w, need=(True, False, False), out=(dx, None, None))
    _, mean, rstd = D.group_norm(img, 2, out=img)
    D.group_norm_backward(img, img, mean, rstd, 2, out=img)
    assert out._version == 1 and dx._version == 1 and img._version == 2
    with torch.inference_mode():
        a = torch.ones(4, 8, dtype=torch.bfloat16, device="cuda")
        D.linear(a, a, out=torch.empty(4, 4, dtype=torch.bfloat16, device="cuda"))
    D.linear(a, a, out=(b := torch.empty(4, 4, dtype=torch.bfloat16, device="cuda")))
    assert (b == 8).all()
