"""Rows that are sure of their target: the loss is log(1 + q), q = sum over the other words of exp(z - z_target), and nothing but that.

With E = 2^-24. The sum holds a 1 for the target; the others add at most q (1 + e), where e covers the errors of the logits (2 (D + 2) E of their
magnitudes), of the distances and of the exponentials (2 ulp): below 1/4 at these sizes. An addition to the sum is off by no more than what is
added. So 0 <= loss <= 4 q: at margins of 30 and more below 4e-8 for 30522 words, where the logits' own steps are 2^-19 and more.
The gradient's entry of the target, exp(z_t - lse) - 1, has lse = z_t rounded, so it is 0 or a rounding of lse."""
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def sure(torch, N, V, n, top, seed=0):
    """Rows whose target's logit is about `top` and far above the others'."""
    g = torch.Generator(device="cuda").manual_seed(seed + N + V)
    w = torch.randn(V, n, generator=g, device="cuda").bfloat16()
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    wt = w[t].float()
    x = (wt * (top / wt.square().sum(1, keepdim=True)) * (1 + 0.3 * torch.rand(N, 1, generator=g, device="cuda"))).bfloat16()
    z = x.double() @ w.double().t()
    own = z[torch.arange(N, device="cuda"), t]
    others = z.clone()
    others[torch.arange(N, device="cuda"), t] = -float("inf")
    return x, w, t, own, torch.exp(others - own[:, None]).sum(1)


# one tile, several, pairs of CTAs, many tiles across
@pytest.mark.parametrize("N,V,n", [(64, 10, 256), (700, 60, 256), (500, 1000, 512), (300, 30522, 512), (4096, 5000, 512)])
@pytest.mark.parametrize("top", [60.0, 200.0, 1000.0, 3e4])
def test_loss_is_what_the_others_add(N, V, n, top):
    torch, D = _d()
    x, w, t, own, q = sure(torch, N, V, n, top)
    far = q < 1e-3
    assert far.sum() > N * 0.8
    loss, lse = D.linear_cross_entropy(x, w, t)
    assert (loss >= 0).all()
    assert (loss.double() <= 4 * q + 1e-37)[far].all(), float((loss.double() / (q + 1e-37))[far].max())
    assert ((lse.double() - own).abs() <= 2 * (n + 3) * E * (x.double().abs() * w[t].double().abs()).sum(1) + E * own.abs() + 4 * q)[far].all()


def test_one_word_has_no_loss():
    torch, D = _d()
    for scale in (0.01, 1.0, 50.0, 1e15):
        x = (torch.randn(300, 40, device="cuda") * scale).bfloat16()
        w = torch.randn(1, 40, device="cuda").bfloat16()
        b = torch.randn(1, device="cuda").bfloat16()
        t = torch.zeros(300, dtype=torch.int64, device="cuda")
        loss, lse = D.linear_cross_entropy(x, w, t, b)
        assert not loss.any() and lse.isfinite().all()
        dx, dw, db = D.linear_cross_entropy_backward(torch.ones(300, device="cuda"), x, w, t, lse, b)
        assert not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("top", [200.0, 3e4])
def test_their_gradient_is_nothing(top):
    """lse is then the target's logit to the last bit, and so is what backward computes again (the same products in the same order): what is left of G are
    the others' entries."""
    torch, D = _d()
    x, w, t, own, q = sure(torch, 500, 1000, 512, top)
    keep = q < 2.0 ** -60
    x, t = x[keep], t[keep]
    assert len(t) > 400
    loss, lse = D.linear_cross_entropy(x, w, t)
    dx, dw, db = D.linear_cross_entropy_backward(torch.ones(len(t), device="cuda"), x, w, t, lse, torch.zeros(1000, device="cuda", dtype=torch.bfloat16))
    # others' shares: q times the largest entries, two roundings to bf16
    assert float(dx.abs().max()) <= 2.0 ** -59 * float(w.abs().max()) and float(db.abs().max()) <= 2.0 ** -59 * len(t)
    assert float(dw.abs().max()) <= 2.0 ** -59 * len(t) * float(x.abs().max())
