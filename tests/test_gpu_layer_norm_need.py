"""Layer norm's gradient without the sums over rows, or with one of them: what is asked for comes bit for bit as with both."""
import pytest

pytestmark = pytest.mark.gpu


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


# a team of 8 lanes, a warp, a CTA, a cluster; 16-byte and single-element accesses
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,n", [(1, 1), (300, 40), (77, 63), (5000, 64), (900, 256), (90, 771), (3000, 1024), (40, 1025), (700, 4096), (9, 16384), (5, 9999)])
def test_either_or_neither(M, n, dtype):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(M + n)
    x, dy, add = (torch.randn(M, n, generator=g, device="cuda").to(getattr(torch, dtype)) for _ in range(3))
    w = torch.randn(n, generator=g, device="cuda")
    _, m, r = D.layer_norm(x, w)
    for a in (None, add):
        dx, dw, db = D.layer_norm_backward(dy, x, m, r, w, add=a)
        for need in ((False, False), (True, False), (False, True), (True, True)):
            got = D.layer_norm_backward(dy, x, m, r, w, add=a, need=need)
            assert torch.equal(got[0], dx)
            assert torch.equal(got[1], dw) if need[0] else got[1] is None
            assert torch.equal(got[2], db) if need[1] else got[2] is None


def test_nothing_to_sum_takes_no_memory():
    torch, D = _d()
    x = torch.randn(4000, 1024, device="cuda").bfloat16()
    _, m, r = D.layer_norm(x)
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    D.layer_norm_backward(x, x, m, r, out=out, need=(False, False))
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    empty = x[:0]
    assert D.layer_norm_backward(empty, empty, m[:0], r[:0], need=(False, False))[1:] == (None, None)
    assert not D.layer_norm_backward(empty, empty, m[:0], r[:0], need=(False, True))[2].any()


def test_recorded_without_the_parameters():
    """Frozen or absent parameters, only the weight, only the bias: the recorded gradient asks for what is needed."""
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = torch.randn(50, 96, generator=g, device="cuda"), torch.randn(50, 96, generator=g, device="cuda")
    w, b = torch.randn(96, generator=g, device="cuda"), torch.randn(96, generator=g, device="cuda")
    _, m, r = D.layer_norm(x, w, b)
    want = D.layer_norm_backward(dy, x, m, r, w)
    from paper_2510_08522_b200 import train_ops as T
    asked, call = [], T.layer_norm_backward

    def seen(*a, **k):
        asked.append(tuple(bool(v) for v in k["need"]))
        return call(*a, **k)
    T.layer_norm_backward = seen
    try:
        for wants in ((True, False, False), (False, True, False), (False, False, True), (True, True, False), (True, True, True)):
            leaves = [t.clone().requires_grad_(k) for t, k in zip((x, w, b), wants)]
            D.layer_norm(*leaves)[0].backward(dy)
            for leaf, k, v in zip(leaves, wants, want):
                assert torch.equal(leaf.grad, v) if k else leaf.grad is None
            assert asked[-1] == wants[1:]
        t = x.clone().requires_grad_(True)
        D.layer_norm(t)[0].backward(dy)
        assert asked[-1] == (False, False) and torch.equal(t.grad, call(dy, x, m, r)[0])
    finally:
        T.layer_norm_backward = call
