"""The training operators under torch's differentiation: gradients are those of the explicit backward calls, bit for bit, and are not
lost silently."""
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
