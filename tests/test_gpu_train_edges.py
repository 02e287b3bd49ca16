"""Edges of the training operators' domain that a user meets: nothing to sum over, values that overflow or underflow, images cut out
of wider ones, tensors in other dense orders, calls from several threads and streams."""
import ctypes
import gc
import math
import threading
import weakref

import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_statistics_of_no_positions_are_nan(dtype):
    # a sum of nothing over nothing: no mean and no deviation. The memory the results come from held other values before.
    torch, D = _d()
    for N, groups in ((3, 2), (1, 1), (70, 8)):
        x = torch.empty(N, 0, 8, dtype=getattr(torch, dtype), device="cuda")
        old = [torch.full((N, groups), 7.0, device="cuda") for _ in range(8)]
        del old
        y, mean, rstd = D.group_norm(x, groups)
        assert y.shape == x.shape and mean.shape == rstd.shape == (N, groups)
        assert torch.isnan(mean).all() and torch.isnan(rstd).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_a_second_moment_that_overflows_stops_its_parameter(bits, offset):
    # (1 - b2) g^2 is above fp32's range for |g| = 1e21: v' is infinite, m' is not, and m'/inf = 0 leaves the parameter to its decay.
    # 8-bit codes hold such a block at the largest scale whose square is finite, so that no value of the block is lost.
    torch, D = _d()
    n, at = 700, 300
    g0 = torch.Generator(device="cuda").manual_seed(1)
    p = torch.randn(n + offset, generator=g0, device="cuda")[offset:]
    g = torch.randn(n + offset, generator=g0, device="cuda")[offset:]
    q, clean = p.clone(), g.clone()
    g[at] = -1e21
    opt, ref = D.AdamW([p], [g], state_bits=bits), D.AdamW([q], [clean], state_bits=bits)
    st, sr = opt.new_state(), ref.new_state()
    was = p.clone()
    h = dict(lr=1e-2, beta1=0.9, beta2=0.999, weight_decay=0.1)
    opt.step(*st, t=1, **h)
    ref.step(*sr, t=1, **h)
    others = torch.arange(n, device="cuda") != at
    assert torch.equal(p[others], q[others])
    assert abs(float(p[at]) - float(was[at]) * (1 - 1e-3)) <= 2 * E * abs(float(was[at]))
    if bits == 32:
        assert torch.equal(st[0][:n][others], sr[0][:n][others]) and torch.equal(st[1][:n][others], sr[1][:n][others])
        assert math.isinf(float(st[1][at])) and abs(float(st[0][at]) + 1e20) < 1e14
    else:
        assert torch.isfinite(st[2]).all() and torch.isfinite(st[3]).all() and float(st[3][1]) > 1.8e19
        m, v = opt.moments(*st)
        assert torch.isfinite(m).all() and torch.isfinite(v).all() and float(v[at]) > 3.3e38 and (v[:n] > 0).all()
        out = torch.arange(768, device="cuda") // 256 != 1                    # the other blocks
        rm, rv = ref.moments(*sr)
        assert torch.equal(m[out], rm[out]) and torch.equal(v[out], rv[out])
    # and the next step
    g[at] = 0.5
    was = p.clone()
    opt.step(*st, t=2, **h)
    # (8 bits: v' is held at 2^128 (1 - 2^-22) at most, which lets lr * 0.9e20/0.19 / (1.84e19/0.0447) through)
    assert torch.isfinite(p).all() and abs(float(p[at]) - float(was[at]) * (1 - 1e-3)) <= 2 * E * abs(float(was[at])) + (0.012 if bits == 8 else 0)


@pytest.mark.parametrize("bits", [32, 8])
def test_tiny_second_moments_with_no_epsilon(bits):
    # the first step without eps and decay is lr * sign(g), whatever g's size. v' = (1-b2) g^2 is rounded in units of 2^-149 where
    # it is subnormal (three roundings, half of it after the root); everything else is relative: 5 e for m', 14 e for the
    # quotient, 3 e for the parameter.
    torch, D = _d()
    size = torch.logspace(-20.5, 3, 2048, dtype=torch.float64, device="cuda")
    sign = torch.where(torch.arange(2048, device="cuda") % 3 == 0, -1.0, 1.0)
    g = (size * sign).float()
    p = torch.zeros(2048, device="cuda")
    opt = D.AdamW([p], [g], state_bits=bits)
    st = opt.new_state()
    opt.step(*st, t=1, lr=1.0, eps=0.0, weight_decay=0.0, beta1=0.9, beta2=0.999)
    v = 1e-3 * g.double() ** 2
    tol = 22 * E + 1.5 * 2.0 ** -149 / v
    err = (p.double() + sign).abs()
    assert torch.all(err <= tol), float((err / tol).max())
    if bits == 8:
        want = v.view(-1, 256).amax(1).sqrt()
        assert torch.all((st[3].double() - want).abs() <= want * (8 * E + 1.5 * 2.0 ** -149 / want ** 2) + 1.2e-38)
    # a later step with a small eps of its own, moments given
    if bits == 32:
        st[0].copy_(g)
        st[1].copy_(g.square())
        q0 = p.clone()
        g0, v0 = st[0].double(), st[1].double()
        opt.bind([torch.zeros_like(g)])
        opt.step(*st, t=5, lr=1.0, eps=1e-20, weight_decay=0.0, beta1=0.9, beta2=0.999)
        want = q0.double() - 0.9 * g0 / (1 - 0.9 ** 5) / ((0.999 * v0).sqrt() / math.sqrt(1 - 0.999 ** 5) + 1e-20)
        scale = (want - q0.double()).abs()
        keep = v0 > 0
        assert torch.all(((p.double() - want).abs() <= scale * (25 * E + 2.0 ** -149 / v0) + 2 * E * (want.abs() + 1))[keep])


def test_a_block_that_is_all_tiny_keeps_its_second_moments():
    # 8-bit codes of a block whose largest sqrt(v') is 1e-19: its scale is the root, to rounding
    torch, D = _d()
    for size in (3e-21, 1e-18, 3e-17, 1e-15):
        g = torch.full((256,), size, device="cuda")
        opt = D.AdamW([torch.zeros(256, device="cuda")], [g], state_bits=8)
        st = opt.new_state()
        opt.step(*st, t=1, lr=0.0)
        v = 1e-3 * float(g[0]) ** 2
        assert abs(float(st[3][0]) - math.sqrt(v)) <= math.sqrt(v) * (8 * E + 1.5 * 2.0 ** -149 / v), size
        assert (st[1] == 255).all()


def test_channel_counts_beyond_32_bits_are_refused():
    torch, D = _d()
    x = torch.empty(1, 1, 2 ** 32 + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(D.DmxError):
        D.group_norm(x, 2)
    with pytest.raises(D.DmxError):
        D.group_norm_backward(x, x, torch.zeros(1, 2, device="cuda"), torch.ones(1, 2, device="cuda"), 2)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_images_one_position_wide_cut_out_of_wider_ones(dtype):
    torch, D = _d()
    g = torch.Generator(device="cuda").manual_seed(2)
    wide = torch.randn(3, 9, 5, 16, generator=g, device="cuda").to(getattr(torch, dtype))
    for x in (wide[:, :, 2:3], wide[:, 4:5], wide[:, 4:5, 1:2], wide[1:2, :, 2:3], wide[:, :, 2:3, 4:12], wide[:, ::2, 2:3]):
        # a dense copy that starts as x does within 16 bytes: the same accesses, so the same sums
        dense = torch.empty(x.numel() + 8, dtype=x.dtype, device="cuda")[x.storage_offset() % 8:][:x.numel()].view(x.shape).copy_(x)
        want = D.group_norm(dense, 2, act="silu")
        got = D.group_norm(x, 2, act="silu")
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        back = D.group_norm_backward(x, x, got[1], got[2], 2, act="silu")
        assert all(torch.equal(a, b) for a, b in zip(back, D.group_norm_backward(dense, dense, want[1], want[2], 2, act="silu")))
        out = x.clone(memory_format=torch.preserve_format)
        room = torch.zeros(x.shape[0], x.shape[1], x.shape[2] + 2, x.shape[3], dtype=x.dtype, device="cuda")
        if x.shape[2] == 1:
            D.group_norm(x, 2, act="silu", out=room[:, :, 1:2])
            assert torch.equal(room[:, :, 1:2], want[0]) and not room[:, :, 0].any() and not room[:, :, 2].any()
        plain = D.group_norm(x.contiguous(), 2, act="silu")[0]
        D.group_norm(out, 2, act="silu", out=out)
        assert torch.equal(out, plain)


def test_status_waits_for_work_on_every_stream():
    torch, D = _d()
    x = torch.ones(256, 256, dtype=torch.bfloat16, device="cuda")
    D.linear(x, x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)               # about a tenth of a second
        D.linear(x, x)
    assert D.linear_status() == 0
    assert side.query(), "the count was taken before the product had run"
    assert D.linear_status() == 0


def test_group_norm_from_two_threads():
    # two sizes of one kernel whose shared memory differs, launched through the C entry by two host threads
    torch, D = _d()
    from paper_2510_08522_b200 import binding as B
    L = B.lib()
    bad = {}

    def work(name, positions):
        torch.cuda.set_device(0)
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            x = torch.randn(300, positions, 32, device="cuda")
            y, mean, rstd = torch.empty_like(x), torch.empty(300, 4, device="cuda"), torch.empty(300, 4, device="cuda")
            f = L.dmx_group_norm_forward
            args = (300, positions, 32, 4, B.F32, x.data_ptr(), positions * 32, 32, None, None, ctypes.c_float(1e-5), 0, y.data_ptr(), positions * 32, 32,
                    mean.data_ptr(), rstd.data_ptr(), None, 0, s.cuda_stream)
            f(*args)
            go.wait()
            codes = [f(*args) for _ in range(4000)]
        s.synchronize()
        bad[name] = [c for c in codes if c != B.OK]

    go = threading.Barrier(2)
    ts = [threading.Thread(target=work, args=a) for a in (("large", 768), ("small", 448))]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert bad == {"large": [], "small": []}, {k: (len(v), v[:3]) for k, v in bad.items()}


def test_copies_stay_alive_whatever_becomes_of_the_callers_list():
    torch, D = _d()
    p, g = [torch.ones(300, device="cuda")], [torch.ones(300, device="cuda")]
    copies = [torch.zeros(300, dtype=torch.bfloat16, device="cuda")]
    ref = weakref.ref(copies[0])
    opt = D.AdamW(p, g, copies=copies)
    copies.clear()
    gc.collect()
    assert ref() is not None, "the step would write to memory that is someone else's"
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_model_of_empty_tensors(bits):
    torch, D = _d()
    opt = D.AdamW([torch.empty(0, device="cuda"), torch.empty(3, 0, device="cuda")], [torch.empty(0, device="cuda"), None], state_bits=bits)
    st = opt.new_state()
    n = opt.grad_norm(1.0)
    assert float(n[0]) == 0 and float(n[1]) == 1
    opt.step(*st, t=1, lr=1e-3, grad_scale=n[1:])
    if bits == 8:
        m, v = opt.moments(*st)
        assert m.numel() == v.numel() == 0


def test_gradients_that_come_later_choose_their_type():
    torch, D = _d()
    for later in (torch.bfloat16, torch.float32):
        p = [torch.ones(300, device="cuda"), torch.ones(40, device="cuda")]
        q = [x.clone() for x in p]
        g = [torch.full((300,), 0.5, dtype=later, device="cuda"), torch.full((40,), -0.25, dtype=later, device="cuda")]
        opt, ref = D.AdamW(p, [None, None]), D.AdamW(q, g)
        st, sr = opt.new_state(), ref.new_state()
        opt.step(*st, t=1, lr=0.1)
        assert float(p[0].min()) == 1.0 and not st[0].any()            # nothing to do yet
        opt.bind(g)
        opt.step(*st, t=1, lr=0.1)
        ref.step(*sr, t=1, lr=0.1)
        assert all(torch.equal(a, b) for a, b in zip(p, q)) and torch.equal(st[1], sr[1])
        other = torch.float32 if later == torch.bfloat16 else torch.bfloat16
        with pytest.raises(D.DmxError):
            opt.bind([x.to(other) for x in g])


@pytest.mark.parametrize("bits", [32, 8])
def test_dense_tensors_in_any_order(bits):
    # AdamW takes a tensor's elements as they lie; parameter, gradient and copy have to lie alike
    torch, D = _d()
    gen = torch.Generator(device="cuda").manual_seed(3)
    mk = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    a, b = mk(24, 5, 3, 3), mk(40, 30)
    p = [a.to(memory_format=torch.channels_last), b.t()]
    g = [mk(24, 5, 3, 3).to(memory_format=torch.channels_last), mk(40, 30).t()]
    c = [torch.zeros_like(x, dtype=torch.bfloat16) for x in p]
    assert c[0].stride() == p[0].stride()
    flat = lambda x: x.permute(0, 2, 3, 1).reshape(-1).clone() if x.dim() == 4 else x.t().reshape(-1).clone()  # noqa: E731  (memory order)
    q, h = [flat(x) for x in p], [flat(x) for x in g]
    opt, ref = D.AdamW(p, g, state_bits=bits, copies=c), D.AdamW(q, h, state_bits=bits)
    st, sr = opt.new_state(), ref.new_state()
    for t in (1, 2):
        opt.step(*st, t=t, lr=0.1, seed=t)
        ref.step(*sr, t=t, lr=0.1, seed=t)
    assert all(torch.equal(flat(x), y) for x, y in zip(p, q)) and all(torch.equal(x, y.bfloat16()) for x, y in zip(c, p))
    m = st[0] if bits == 32 else opt.moments(*st)[0]
    r = sr[0] if bits == 32 else ref.moments(*sr)[0]
    for i in range(2):
        v = opt.state_view(m, i)
        assert v.shape == p[i].shape and torch.equal(flat(v), ref.state_view(r, i))
    for bad in ([g[0].contiguous(), g[1]], [g[0], g[1].contiguous()], [g[0], mk(1, 1).expand(30, 40)], [g[0], mk(30, 80)[:, ::2]]):
        with pytest.raises(D.DmxError):
            opt.bind(bad, c)
    one = mk(24, 1, 1, 1)                                   # where extents of one leave the order open, any strides do
    D.AdamW([one], [torch.empty_strided((24, 1, 1, 1), (1, 24, 24, 24), device="cuda")]).close()


def test_entries_that_are_no_tensors_are_refused():
    torch, D = _d()
    p, g = torch.ones(30, device="cuda"), torch.ones(30, device="cuda")
    for params, grads, copies in (([p, None], [g, None], None), ([p], [1.0], None), ([p], ["g"], None), ([p], [g], [3])):
        with pytest.raises(D.DmxError):
            D.AdamW(params, grads, copies=copies)
    opt = D.AdamW([p], [g])
    with pytest.raises(D.DmxError):
        opt.bind([0])
