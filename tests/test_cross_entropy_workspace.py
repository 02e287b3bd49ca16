"""How much workspace the cross entropy's gradient asks for by the outputs that are wanted, and that a call with just that much keeps to it."""
import pytest

import paper_2510_08522_b200 as D
from paper_2510_08522_b200 import binding as B

# (N, V, D): several pieces, one piece, products cut into ranges, one row
SHAPES = [(65536, 20000, 1024), (70000, 5003, 40), (777, 1000, 513), (16000, 33, 24), (1, 30522, 264)]


def asked(N, V, n, outputs, ld=None):
    return B.lib().dmx_cross_entropy_backward_workspace_for(N, V, n, 256, ld or -(-n // 8) * 8, 512, ld or -(-n // 8) * 8, outputs)


@pytest.mark.parametrize("N,V,n", SHAPES)
def test_each_output_asks_for_its_own(N, V, n):
    L = B.lib()
    ld = -(-n // 8) * 8
    every = asked(N, V, n, 7)
    assert every == L.dmx_cross_entropy_backward_workspace(N, V, n, 256, ld, 512, ld)
    assert asked(N, V, n, 0) == 0
    for o in range(1, 8):
        for less in range(1, 8):
            if less & ~o == 0:
                assert 0 < asked(N, V, n, less) <= asked(N, V, n, o) <= every
    plan = (D.binding.ctypes.c_int64 * 11)()
    assert L.dmx_cross_entropy_plan(N, V, n, plan) == B.OK
    pieces, words = plan[3], min(plan[4], V)
    g, columns = 2 * N * words, -(-N // 32) * words * 4
    assert asked(N, V, n, 2) >= g and columns <= asked(N, V, n, 4) < columns + 4096
    if pieces > 1:
        assert asked(N, V, n, 3) - asked(N, V, n, 2) >= 4 * N * n and asked(N, V, n, 6) - asked(N, V, n, 2) < columns + 4096


def test_refusals():
    for outputs in (-1, 8):
        assert asked(4, 8, 8, outputs) == B.ERR_ARG
    assert asked(-1, 8, 8, 7) == asked(4, 0, 8, 7) == B.ERR_ARG and asked(0, 8, 8, 7) == 0
    # too little for what is asked for: refused on the host
    def backward(dx, dw, db, size, N=70000, V=5003, n=40):
        return B.lib().dmx_cross_entropy_backward(N, V, n, 128, 1, 256, n, 512, n, None, 4, 1024, 2048, dx, n, dw, n, db, 16384, size, None)
    for o in range(1, 8):
        assert backward(*(1 << 20 if o >> i & 1 else None for i in range(3)), asked(70000, 5003, 40, o) - 1) == B.ERR_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("N,V,n", [(70000, 5003, 40), (777, 1000, 513), (777, 1000, 512), (16000, 33, 24), (1, 30522, 264), (300, 40, 64)])
def test_a_call_keeps_to_what_it_asked_for(N, V, n):
    import torch
    L = B.lib()
    g = torch.Generator(device="cuda").manual_seed(N)
    x, w = torch.randn(N, n, generator=g, device="cuda").bfloat16(), (n ** -0.5 * torch.randn(V, n, generator=g, device="cuda")).bfloat16()
    b, t = torch.randn(V, generator=g, device="cuda").bfloat16(), torch.randint(-1, V, (N,), generator=g, device="cuda")
    dloss = torch.rand(N, generator=g, device="cuda")
    _, lse = D.linear_cross_entropy(x, w, t, b)
    want = D.linear_cross_entropy_backward(dloss, x, w, t, lse, b)
    for o in range(1, 8):
        need = tuple(bool(o >> i & 1) for i in range(3))
        size = L.dmx_cross_entropy_backward_workspace_for(N, V, n, x.data_ptr(), n, w.data_ptr(), n, o)
        ws = torch.full((size + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        out = [torch.full_like(r, float("nan")) for r in want]
        p = [v.data_ptr() if k else None for v, k in zip(out, need)]
        rc = L.dmx_cross_entropy_backward(N, V, n, dloss.data_ptr(), 1, x.data_ptr(), n, w.data_ptr(), n, b.data_ptr(), 8, t.data_ptr(), lse.data_ptr(), p[0], n, p[1], n, p[2],
                                          ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
        assert rc == B.OK
        assert (ws[size:] == 0x5a).all()
        for v, r, k in zip(out, want, need):
            assert torch.equal(v, r) if k else v.isnan().all()
        got = D.linear_cross_entropy_backward(dloss, x, w, t, lse, b, need=need)
        assert all(torch.equal(v, r) if k else v is None for v, r, k in zip(got, want, need))
    assert D.linear_status() == 0


@pytest.mark.gpu
def test_memory_of_a_head_alone():
    """Only the weight's gradient: neither dx's sums over the pieces nor the columns' are reserved."""
    import torch
    N, V, n = 70000, 5003, 512
    x, w = torch.randn(N, n, device="cuda").bfloat16(), torch.randn(V, n, device="cuda").bfloat16()
    t = torch.randint(0, V, (N,), device="cuda")
    loss, lse = D.linear_cross_entropy(x, w, t)

    def peak(need):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        out = D.linear_cross_entropy_backward(torch.ones_like(loss), x, w, t, lse, need=need)
        most = torch.cuda.max_memory_allocated() - before
        del out
        return most
    alone, both = peak((False, True, False)), peak((True, True, False))
    assert both - alone >= N * n * 6 * 0.99         # its fp32 sums and its result
