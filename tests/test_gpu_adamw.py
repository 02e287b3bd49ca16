"""AdamW over many tensors and its gradient norm against the definition in fp64: every parameter, gradient and
state type, odd sizes and starts, missing gradients, the skipped step, dithered codes, and chains of steps.

Tolerances are forward error bounds. With e = 2^-24: m' = b1 m + (1-b1) s g takes at most five roundings (two constants, s g, b1 m, the
sum), so it is within 5 e (|b1 m| + |(1-b1) s g|); v' is a sum of positive terms within 7 e of itself; the
update u = m'/(sqrt(v') c + eps) adds at most 8 e |u| (half of v's error, root, product, sum, quotient, and the
step's constant) if root and quotient are correctly rounded and 14 e |u| at the 2 ulp each that CUDA documents
for their approximate forms (the bound taken); p (1 - lr wd) - step u adds 3 e |p|. A bf16 parameter lies between
the bf16 roundings of the two ends of that interval. Codes are checked by bracketing: the code lies between the
codes of the two ends of the value's error interval."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
H = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


def _d():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2510_08522_b200 as D
    return torch, D


def mixed(idx, seed):
    """The dither hash of state indices (Murmur3 finaliser), restated in numpy: two uniforms in [0,1)."""
    h = (idx.astype(np.uint64) * np.uint64(0x9E3779B1) + np.uint64((seed * 0x85EBCA6B + 0x1B873593) & 0xFFFFFFFF)) & np.uint64(0xFFFFFFFF)
    h ^= h >> np.uint64(16)
    h = (h * np.uint64(0x85EBCA6B)) & np.uint64(0xFFFFFFFF)
    h ^= h >> np.uint64(13)
    h = (h * np.uint64(0xC2B2AE35)) & np.uint64(0xFFFFFFFF)
    h ^= h >> np.uint64(16)
    return (h & np.uint64(0xFFFF)).astype(np.float64) / 65536, (h >> np.uint64(16)).astype(np.float64) / 65536


def decode(c, scale, steps):
    c = c.astype(np.float64).reshape(-1, 256)
    return (np.sign(c) * (c / steps) ** 2 * scale.astype(np.float64)[:, None]).reshape(-1)


class Case:
    def __init__(self, sizes, pd, gd, bits, offset=0, copies=False, seed=0):
        torch, D = _d()
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.sizes, self.bits = sizes, bits
        mk = lambda n, s, d: (torch.randn(n + offset, generator=g, device="cuda") * s).to(d)[offset:]  # noqa: E731
        self.p = [mk(n, 0.5, pd) for n in sizes]
        self.g = [mk(n, 1.0, gd) for n in sizes]
        self.c = [torch.zeros(n + offset, dtype=torch.bfloat16, device="cuda")[offset:] for n in sizes] if copies else None
        self.decay = [i % 3 != 1 for i in range(len(sizes))]
        self.opt = D.AdamW(self.p, self.g, state_bits=bits, copies=self.c, decay=self.decay)
        self.state = self.opt.new_state()
        self.gen = g

    def new_grads(self):
        torch, _ = _d()
        for x in self.g:
            x.copy_(torch.randn(x.shape, generator=self.gen, device="cuda"))

    def check_step(self, t, scale=None, seed=None, skip=()):
        torch, _ = _d()
        before = [x.double().cpu().numpy() for x in self.p]
        st0 = [None if s is None else s.cpu().numpy().copy() for s in self.state]
        gs = None if scale is None else torch.tensor([scale], dtype=torch.float32, device="cuda")
        self.opt.step(*self.state, t=t, grad_scale=gs, seed=seed, **H)
        torch.cuda.synchronize()
        st1 = [None if s is None else s.cpu().numpy() for s in self.state]
        s = 1.0 if scale is None else float(np.float32(scale))
        b0 = 0
        for i, n in enumerate(self.sizes):
            nb = -(-n // 256)
            lo, pad = b0 * 256, nb * 256
            blk = slice(b0, b0 + nb)
            b0 += nb
            if n == 0:
                continue
            p1 = self.p[i].double().cpu().numpy()
            if i in skip:
                assert np.array_equal(p1, before[i])
                for a, b in zip(st0, st1):
                    if a is not None:
                        sl = slice(lo, lo + pad) if a.size > len(st0[2] if st0[2] is not None else []) else blk
                        assert np.array_equal(a[sl], b[sl])
                continue
            g = np.zeros(pad)
            g[:n] = self.g[i].double().cpu().numpy()
            if self.bits == 32:
                m, v = st0[0][lo:lo + pad].astype(np.float64), st0[1][lo:lo + pad].astype(np.float64)
                extra = 0.0
            else:
                m = decode(st0[0][lo:lo + pad], st0[2][blk], 127.0)
                v = decode(st0[1][lo:lo + pad], st0[3][blk], 255.0) ** 2
                extra = 10 * E        # decoding: constant, product, square, scale (and the square of sqrt(v))
            cm = np.abs(H["beta1"] * m) + np.abs((1 - H["beta1"]) * s * g)
            m1 = H["beta1"] * m + (1 - H["beta1"]) * s * g
            v1 = H["beta2"] * v + (1 - H["beta2"]) * (s * g) ** 2
            dm, dv = (5 * E + extra) * cm + 1e-44, (7 * E + 2 * extra) * v1 + 1e-44
            den = np.sqrt(v1) / math.sqrt(1 - H["beta2"] ** t) + H["eps"]
            u = m1 / den
            step = H["lr"] / (1 - H["beta1"] ** t)
            keep = 1 - H["lr"] * H["weight_decay"] if self.decay[i] else 1.0
            ref = before[i] * keep - step * u[:n]
            tol = 3 * E * np.abs(before[i]) + step * (dm / den + (14 * E + extra) * np.abs(u))[:n]
            lo_p, hi_p = ref - tol, ref + tol
            if self.p[i].dtype == torch.bfloat16:
                lo_p, hi_p = (torch.from_numpy(x).to(torch.bfloat16).double().numpy() for x in (lo_p, hi_p))
            assert np.all(p1 >= lo_p) and np.all(p1 <= hi_p), (i, n, np.max(np.abs(p1 - ref) / tol))
            if self.c is not None:
                assert torch.equal(self.c[i], self.p[i].to(torch.bfloat16))
            if self.bits == 32:
                assert np.all(np.abs(st1[0][lo:lo + pad] - m1) <= dm) and np.all(np.abs(st1[1][lo:lo + pad] - v1) <= dv)
                assert not st1[0][lo + n:lo + pad].any() and not st1[1][lo + n:lo + pad].any()
                continue
            um, uv = (0.5, 0.5) if seed is None else mixed(np.arange(lo, lo + pad), seed)
            r1 = np.sqrt(v1)
            for c, sc, x, dx, uu, steps in ((st1[0], st1[2], np.abs(m1), dm, um, 127), (st1[1], st1[3], r1, (6 * E + extra) * r1 + 1e-22, uv, 255)):
                big = x.reshape(-1, 256)
                S = sc[blk].astype(np.float64)
                assert np.all(np.abs(S - big.max(1)) <= dx.reshape(-1, 256).max(1) + 1.2e-38)
                for side, sign in (("lo", -1), ("hi", 1)):
                    y = np.maximum(x + sign * dx, 0).reshape(-1, 256) / np.where(S > 0, S, 1)[:, None] * (1 + sign * 4 * E)
                    code = np.floor(np.sqrt(y) * steps * (1 + sign * 4 * E) + np.reshape(uu, (-1, 256)) if np.ndim(uu) else np.sqrt(y) * steps * (1 + sign * 4 * E) + uu)
                    code = np.minimum(code, steps).reshape(-1)
                    got = np.abs(c[lo:lo + pad].astype(np.int64))
                    if steps == 255:
                        code = np.where(x > 0, np.maximum(code, 1), code)
                    assert np.all(got >= code) if side == "lo" else np.all(got <= code), (i, n, side, steps)
            signs = np.sign(st1[0][lo:lo + pad].astype(np.float64)) * np.sign(m1)
            assert np.all((signs >= 0) | (np.abs(m1) <= dm))
            assert np.all((st1[1][lo:lo + n] > 0) | (v1[:n] == 0))
            assert not st1[0][lo + n:lo + pad].any() and not st1[1][lo + n:lo + pad].any()


SIZES = [0, 1, 2, 7, 8, 9, 255, 256, 257, 511, 1000, 2048, 8191, 8192, 8193, 30011]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pd,gd", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_steps(bits, pd, gd, offset):
    torch, _ = _d()
    c = Case(SIZES, getattr(torch, pd), getattr(torch, gd), bits, offset, copies=pd == "float32", seed=offset)
    for t in range(1, 5):
        c.check_step(t, scale=[None, 0.37, 1.0, 2.5][t - 1], seed=None if t % 2 else 1000 + t)
        c.new_grads()


def test_many_blocks_take_the_long_chunks():
    torch, _ = _d()
    c = Case([3_000_001, 12_345_679, 5], torch.float32, torch.bfloat16, 8, 0, seed=5)
    for t in (1, 2):
        c.check_step(t, seed=t)
        c.new_grads()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_missing_gradient_leaves_its_tensor_alone(bits):
    torch, _ = _d()
    c = Case([700, 5000, 300], torch.float32, torch.float32, bits)
    c.check_step(1)
    c.opt.bind([c.g[0], None, c.g[2]])
    c.check_step(2, skip=(1,))
    n = c.opt.grad_norm(1.0)
    ref = math.sqrt(sum(float((x.double() ** 2).sum()) for x in (c.g[0], c.g[2])))
    assert abs(float(n[0]) - ref) <= 6 * E * ref


@pytest.mark.parametrize("bits", [32, 8])
def test_nan_factor_skips_the_step(bits):
    torch, _ = _d()
    c = Case([700, 5000], torch.float32, torch.float32, bits)
    c.check_step(1)
    p, st = [x.clone() for x in c.p], [None if s is None else s.clone() for s in c.state]
    c.g[1][17] = float("inf")
    n = c.opt.grad_norm(1.0)
    c.opt.step(*c.state, t=2, grad_scale=n[1:], **H)
    assert math.isinf(float(n[0])) and math.isnan(float(n[1]))
    assert all(torch.equal(a, b) for a, b in zip(p, c.p)) and all(a is None or torch.equal(a, b) for a, b in zip(st, c.state))


@pytest.mark.parametrize("sizes", [[1], [5, 0, 300], SIZES, [2_000_003, 17, 4_000_000]])
@pytest.mark.parametrize("gd", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset", [0, 3])
def test_grad_norm(sizes, gd, offset):
    torch, D = _d()
    c = Case(sizes, torch.float32, getattr(torch, gd), 32, offset, seed=9)
    ref = math.sqrt(sum(float((x.double() ** 2).sum()) for x in c.g))
    for cap in (0.5, 1e9):
        a = c.opt.grad_norm(cap).clone()
        b = c.opt.grad_norm(cap)
        assert torch.equal(a, b)
        # squares summed eight at a time in fp32 (at most 8 roundings of positive terms; the root halves them), then one rounding
        assert abs(float(a[0]) - ref) <= 6 * E * ref
        want = min(1.0, cap / (ref + 1e-6))
        assert abs(float(a[1]) - want) <= 8 * E * want


def test_zero_gradients_and_first_steps():
    torch, _ = _d()
    for bits in (32, 8):
        c = Case([1000], torch.float32, torch.float32, bits)
        c.g[0].zero_()
        p0 = c.p[0].clone()
        c.opt.step(*c.state, t=1, **dict(H, weight_decay=0.0))
        assert torch.equal(c.p[0], p0) and not c.state[0].any() and not c.state[1].any()
        n = c.opt.grad_norm(1.0)
        assert float(n[0]) == 0.0 and float(n[1]) == 1.0


def test_dithered_second_moment_follows_its_average():
    # v starts at 1 and its gradient is zero: after n steps it is beta2^n. Nearest codes would stay where they are.
    torch, D = _d()
    n, steps = 256 * 64, 400
    p, g = [torch.zeros(n, device="cuda")], [torch.ones(n, device="cuda")]
    end = {}
    for dither in (False, True):
        opt = D.AdamW(p, g, state_bits=8)
        st = opt.new_state()
        g[0].fill_(1.0)
        g[0][::256] = 2.0                              # keeps the block's scale above the other values
        opt.step(*st, t=1, lr=0.0, beta2=0.999, seed=1 if dither else None)
        for t in range(2, steps):
            g[0].zero_()
            g[0][::256] = 2.0
            opt.step(*st, t=t, lr=0.0, beta2=0.999, seed=t if dither else None)
        v = opt.moments(*st)[1].view(-1, 256)[:, 1:]
        end[dither] = float(v.mean() / 0.001) / 0.999 ** (steps - 2)
    assert abs(end[True] - 1) < 0.1, end               # 398 steps of dither noise: sd of one value ~0.15, of the mean of 16320 ~0.002, plus a bias from the square law
    assert end[False] > 1.2, end


def test_moments_are_the_codes_values():
    torch, D = _d()
    c = Case([1000, 256 * 40 + 3], torch.float32, torch.float32, 8, seed=3)
    c.opt.step(*c.state, t=1, **H)
    m, v = c.opt.moments(*c.state)
    cm, cv, sm, sv = (x.cpu().numpy() for x in c.state)
    rm, rv = decode(cm, sm, 127.0), decode(cv, sv, 255.0) ** 2
    assert np.all(np.abs(m.cpu().numpy() - rm) <= 5 * E * np.abs(rm)) and np.all(np.abs(v.cpu().numpy() - rv) <= 12 * E * rv)
    bm, bv = torch.empty_like(m, dtype=torch.bfloat16), torch.empty_like(m, dtype=torch.bfloat16)
    c.opt.moments(*c.state, bm, bv)
    assert torch.equal(bm, m.bfloat16()) and torch.equal(bv, v.bfloat16())
    view = c.opt.state_view(m, 1)
    assert view.shape == (256 * 40 + 3,) and torch.equal(view, m[1024:1024 + 256 * 40 + 3])


def test_other_stream_and_graph_replay():
    torch, D = _d()
    c = Case([5000, 70_001], torch.float32, torch.bfloat16, 8, seed=2)
    d = Case([5000, 70_001], torch.float32, torch.bfloat16, 8, seed=2)
    torch.cuda.synchronize()
    side, norm = torch.cuda.Stream(), torch.empty(2, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.opt.grad_norm(1.0, out=norm)
            c.opt.step(*c.state, t=3, grad_scale=norm[1:], **H)
        for _ in range(3):
            graph.replay()
    side.synchronize()
    for _ in range(3):
        n = d.opt.grad_norm(1.0)
        d.opt.step(*d.state, t=3, grad_scale=n[1:], **H)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(c.p, d.p)) and all(torch.equal(a, b) for a, b in zip(c.state, d.state))


def test_refusals_on_the_device():
    torch, D = _d()
    p, g = [torch.zeros(300, device="cuda")], [torch.zeros(300, device="cuda")]
    opt = D.AdamW(p, g, state_bits=8)
    m, v, ms, vs = opt.new_state()
    ok = dict(lr=1e-3, t=1)
    for bad in (dict(ok, t=0), dict(ok, beta1=1.0), dict(ok, beta2=-0.1), dict(ok, eps=-1.0), dict(ok, lr=float("nan")), dict(ok, weight_decay=-1.0)):
        with pytest.raises(D.DmxError):
            opt.step(m, v, ms, vs, **bad)
    with pytest.raises(D.DmxError):
        opt.step(m, v, **ok)                           # scales missing
    with pytest.raises(D.DmxError):
        opt.step(m[:256], v, ms, vs, **ok)
    for bad in ((m.float(), v, ms, vs), (m, v, ms[:1], vs), (m, v, ms, vs.double()), (m.cpu(), v, ms, vs), (m, None, ms, vs)):
        with pytest.raises(D.DmxError):
            opt.step(*bad, **ok)
    for bad in (dict(ok, grad_scale=ms), dict(ok, grad_scale=1.0), dict(ok, seed="a"), dict(ok, t="1"), dict(ok, lr=None)):
        with pytest.raises(D.DmxError):
            opt.step(m, v, ms, vs, **bad)
    for out in (torch.empty(3, device="cuda"), torch.empty(2), torch.empty(2, device="cuda", dtype=torch.float64), torch.empty(4, device="cuda")[::2]):
        with pytest.raises(D.DmxError):
            opt.grad_norm(1.0, out=out)
    assert opt.grad_norm(1.0, out=(n := torch.empty(2, device="cuda"))) is n
    with pytest.raises(D.DmxError):
        opt.grad_norm(0.0)
    with pytest.raises(D.DmxError):
        opt.bind([torch.zeros(299, device="cuda")])
    with pytest.raises(D.DmxError):
        opt.bind([torch.zeros(300, device="cuda", dtype=torch.bfloat16)])
    with pytest.raises(D.DmxError):
        D.AdamW(p, g, state_bits=16)
    with pytest.raises(D.DmxError):
        D.AdamW([torch.zeros(4)], [torch.zeros(4)])
    with pytest.raises(D.DmxError):
        D.AdamW([torch.zeros(4, device="cuda", dtype=torch.float64)], [None])
    assert torch.count_nonzero(p[0]) == 0
    opt32 = D.AdamW(p, g)
    with pytest.raises(D.DmxError):
        opt32.moments(*opt32.new_state())
    opt.close()
    with pytest.raises(D.DmxError):
        opt.step(m, v, ms, vs, **ok)
